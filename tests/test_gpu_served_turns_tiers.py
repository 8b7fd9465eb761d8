"""Served turns whose two tiers, of an fp8 cache's blocks and of its scales, do
not lose the same blocks at the same time."""
import numpy as np
import pytest
import torch

import test_gpu_cache_ops as base
import test_gpu_served_turns as served
from gpu_common import need_gpu
from paper_2609_33762_amd import api
from paper_2609_33762_amd.drivers import ServedTurns

pytestmark = pytest.mark.gpu

L, P, T, H, D, VOCAB = served.L, served.P, served.T, served.H, served.D, served.VOCAB


class Gained(served.Model):
    """A model whose keys and values come out larger or smaller, as another
    path's may: with a gain of 2 the codes stay and every scale doubles."""
    gain = 1.0

    def project(self, layer, x):
        q, k, v = super().project(layer, x)
        return q, k * self.gain, v * self.gain


@pytest.mark.parametrize("block_slots,scale_slots", [(5, 32), (32, 5)])
def test_a_block_comes_back_with_the_scales_it_was_made_with(block_slots, scale_slots):
    need_gpu()
    kv = torch.zeros((L, P, 2, T, H, D), dtype=base.FP8, device="cuda")
    scales = torch.zeros((L, P, 2, H), device="cuda")
    cache = api.Cache(kv, P, L, T, H, D, 1, head_scales=scales)
    plane = api.Cache(scales, P, L, 1, H, 1, 4)
    model = Gained()
    serve = ServedTurns(torch, cache, api.Tier(cache, block_slots * cache.slot_bytes), model, 4,
                        rope=base.rope_table(400, D).cuda(), scale_cache=plane,
                        scale_tier=api.Tier(plane, scale_slots * plane.slot_bytes))
    r = np.random.default_rng(6)
    one, other = (r.integers(0, VOCAB, 90).astype(np.int32) for _ in range(2))
    pages = r.permutation(P).astype(np.int32)
    assert serve.turn(one, 1, pages[:6])[1:] == (0, 5)
    assert serve.turn(other, 1, pages[6:12])[1:] == (0, 5)     # the smaller tier loses the first
    model.gain = 2.0
    assert serve.turn(one, 1, pages[12:18])[1:] == (0, 5)
    assert serve.turn(one, 1, pages[18:24])[1:] == (5, 0)
    torch.cuda.synchronize()
    made, back = (torch.as_tensor(pages[a:a + 5], device="cuda").long() for a in (12, 18))
    assert (scales[:, made] > 0).all()
    assert torch.equal(kv[:, made].view(torch.uint8), kv[:, back].view(torch.uint8))
    assert torch.equal(scales[:, made], scales[:, back])


@pytest.mark.parametrize("act,x_dtype", [(base.BF16, torch.float32), (base.F16, torch.bfloat16)])
def test_bounds_of_restored_blocks_go_by_the_cache_s_type(act, x_dtype):
    # x may have any type: the bounds are of what the blocks hold
    need_gpu()

    class Mixed(served.Model):
        def embed(self, tokens):
            return super().embed(tokens).to(x_dtype)

        def project(self, layer, x):
            return tuple(t.to(act) for t in super().project(layer, x.to(base.BF16)))

        def mix(self, layer, x, attention):
            return super().mix(layer, x.to(base.BF16), attention.to(base.BF16)).to(x_dtype)

    kv = torch.zeros((L, P, 2, T, H, D), dtype=act, device="cuda")
    bounds = torch.zeros((L, P, 2, H, D), dtype=torch.int8, device="cuda")
    units = torch.zeros((L, P, H), device="cuda")
    cache = api.Cache(kv, P, L, T, H, D, 2, bounds=bounds, bound_scales=units)
    serve = ServedTurns(torch, cache, api.Tier(cache, 32 * cache.slot_bytes), Mixed(), 4,
                        rope=base.rope_table(400, D).cuda())
    r = np.random.default_rng(7)
    prompt = r.integers(0, VOCAB, 90).astype(np.int32)
    pages = r.permutation(P).astype(np.int32)
    assert serve.turn(prompt, 3, pages[:6])[1] == 0
    assert serve.turn(prompt, 3, pages[6:12])[1] == 5
    torch.cuda.synchronize()
    made, back = (torch.as_tensor(pages[a:a + 5], device="cuda").long() for a in (0, 6))
    assert torch.equal(kv[:, made], kv[:, back]) and bool((units[:, made] > 0).all())
    assert torch.equal(bounds[:, made], bounds[:, back])
    assert torch.equal(units[:, made], units[:, back])


def test_pages_of_a_turn_that_failed_are_free_of_transfers():
    cache, model, serve = served.setting(False, 4)
    r = np.random.default_rng(8)
    prompt = r.integers(0, VOCAB, 90).astype(np.int32)
    pages = r.permutation(P).astype(np.int32)
    assert serve.turn(prompt, 1, pages[:6])[1:] == (0, 5)
    torch.cuda.synchronize()
    with torch.cuda.stream(serve.copy_stream):
        torch.cuda._sleep(100_000_000)  # the blocks come late
    embed = model.embed

    def fails(tokens):
        raise RuntimeError("of the model")

    model.embed = fails
    with pytest.raises(RuntimeError, match="of the model"):
        serve.turn(prompt, 1, pages[6:12])
    again = torch.as_tensor(pages[6:12], device="cuda").long()
    cache.kv[:, again] = 7.0
    torch.cuda.synchronize()
    assert bool((cache.kv[:, again] == 7.0).all())
    model.embed = embed
    assert serve.turn(prompt, 1, pages[6:12])[1:] == (5, 0)
