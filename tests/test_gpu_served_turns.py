"""Turns of a small model served from the cache and its tier: restore, append,
attention over a chunk, block selection and sparse attention together.  Every
attention result is compared with a 64-bit one over the cache as the turn left
it (bf16 blocks never change once written); bounds of the errors as in
tests/test_gpu_cache_ops.py."""
import numpy as np
import pytest
import torch

import test_gpu_cache_ops as base
from gpu_common import need_gpu
from paper_2609_33762_amd import api
from paper_2609_33762_amd.drivers import ServedTurns

pytestmark = pytest.mark.gpu

L, P, T, H, G, D, WIDTH, VOCAB = 3, 64, 16, 2, 2, 64, 96, 500


class Model:
    def __init__(self, seed=0):
        g = torch.Generator().manual_seed(seed)

        def rand(*shape):
            return (torch.randn(shape, generator=g) * shape[0] ** -0.5).to(base.BF16).cuda()

        self.table = rand(VOCAB, WIDTH) * VOCAB ** 0.5
        self.qkv = [rand(WIDTH, (G + 2) * H * D) for _ in range(L)]
        self.out = [rand(H * G * D, WIDTH) for _ in range(L)]

    def embed(self, tokens):
        return self.table[tokens.long()]

    def project(self, layer, x):
        y = (x @ self.qkv[layer]).view(len(x), (G + 2) * H, D)
        return y[:, :G * H], y[:, G * H:G * H + H], y[:, G * H + H:]

    def mix(self, layer, x, attention):
        return x + attention.reshape(len(x), -1) @ self.out[layer]

    def next(self, x):
        return int((x[-1].float() @ self.table.float().T).argmax())


class Kept(api.Cache):
    """Keeps every call's queries and selections."""

    def attend(self, layer, batch, q, out, selected=None, **kw):
        super().attend(layer, batch, q, out, selected=selected, **kw)
        if hasattr(self, "kept"):
            self.kept.append((layer, batch.n_rows, int(batch.kv_len[0]), q.clone(),
                              None if selected is None else selected.clone(), out.clone()))


def setting(fp8, budget):
    need_gpu()
    kv = torch.zeros((L, P, 2, T, H, D), dtype=base.FP8 if fp8 else base.BF16, device="cuda")
    scales = torch.zeros((L, P, 2, H), device="cuda") if fp8 else None
    bounds = torch.zeros((L, P, 2, H, D), dtype=torch.int8, device="cuda")
    units = torch.zeros((L, P, H), device="cuda")
    cache = Kept(kv, P, L, T, H, D, 1 if fp8 else 2, head_scales=scales, bounds=bounds,
                 bound_scales=units)
    tier = api.Tier(cache, 32 * cache.slot_bytes)
    extra = {}
    if fp8:
        plane = api.Cache(scales, P, L, 1, H, 1, 4)
        extra = dict(scale_cache=plane, scale_tier=api.Tier(plane, 32 * plane.slot_bytes))
    model = Model()
    return cache, model, ServedTurns(torch, cache, tier, model, budget,
                                     rope=base.rope_table(400, D).cuda(), **extra)


def check_calls(cache, pages):
    kv = cache.kv.cpu()
    idx = torch.as_tensor(pages).long()
    for layer, rows, length, q, selected, out in cache.kept:
        q, out = q.cpu().double(), out.cpu().double()
        blocks = kv[layer, idx].double()  # [n, 2, T, H, D]
        for h in range(H):
            k, v = (blocks[:, i, :, h].reshape(-1, D)[:length] for i in (0, 1))
            for r in range(rows):
                see = torch.arange(length) <= length - rows + r
                if selected is not None:
                    see &= torch.isin(torch.arange(length) // T, selected[r, h].cpu().long())
                w = torch.softmax(q[r, h * G:h * G + G] @ k[see].T * D ** -0.5, 1)
                want, mag = w @ v[see], w @ v[see].abs()
                bound = 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -14) * mag + 2.0 ** -25
                assert ((out[r, h * G:h * G + G] - want).abs() <= bound).all()


@pytest.mark.parametrize("budget", [4, 12])
def test_turns_restore_attend_select_and_store(budget):
    cache, model, serve = setting(False, budget)
    r = np.random.default_rng(5)
    prompt = r.integers(0, VOCAB, 70).astype(np.int32)
    pages = r.permutation(P).astype(np.int32)
    cache.kept = []
    made, held, stored = serve.turn(prompt, 12, pages[:6])
    torch.cuda.synchronize()
    assert len(made) == 12 and held == 0 and stored == 81 // T
    check_calls(cache, pages[:6])

    # the next turn keeps the tokens and adds some: its first blocks come back
    # into other pages, bounds and all
    longer = np.concatenate([prompt, np.asarray(made, np.int32),
                             r.integers(0, VOCAB, 30).astype(np.int32)])
    cache.kept = []
    made2, held2, stored2 = serve.turn(longer, 9, pages[10:19])
    torch.cuda.synchronize()
    assert held2 == 5 and stored2 == (len(longer) + 8) // T - 5
    old, new = (torch.as_tensor(pages[a:a + 5], device="cuda").long() for a in (0, 10))
    assert torch.equal(cache.kv[:, old], cache.kv[:, new])
    assert torch.equal(cache.bounds[:, old], cache.bounds[:, new])
    assert torch.equal(cache.bound_scales[:, old], cache.bound_scales[:, new])
    check_calls(cache, pages[10:19])
    # a repeat restores every block but the last
    made3, held3, stored3 = serve.turn(longer, 9, pages[20:29])
    assert held3 == (len(longer) - 1) // T and stored3 == 0 and len(made3) == 9


def test_fp8_blocks_come_back_with_their_scales():
    cache, model, serve = setting(True, 4)
    r = np.random.default_rng(6)
    prompt = r.integers(0, VOCAB, 90).astype(np.int32)
    pages = r.permutation(P).astype(np.int32)
    _, held, stored = serve.turn(prompt, 1, pages[:6])
    assert held == 0 and stored == 5
    made, held, _ = serve.turn(prompt, 5, pages[8:14])
    torch.cuda.synchronize()
    assert held == 5 and len(made) == 5
    old, new = (torch.as_tensor(pages[a:a + 5], device="cuda").long() for a in (0, 8))
    assert torch.equal(cache.kv[:, old].view(torch.uint8), cache.kv[:, new].view(torch.uint8))
    assert torch.equal(cache.head_scales[:, old], cache.head_scales[:, new])
    assert torch.equal(cache.bounds[:, old], cache.bounds[:, new])
    assert (cache.head_scales[:, new] > 0).all()


def test_refusals():
    cache, model, serve = setting(False, 4)
    with pytest.raises(ValueError):
        serve.turn(np.zeros(40, np.int32), 10, np.arange(3))   # too few pages
    with pytest.raises(ValueError):
        serve.turn(np.zeros(0, np.int32), 1, np.arange(3))     # nothing to start from
    with pytest.raises(ValueError):
        ServedTurns(torch, cache, serve.pairs[-1][0], model, 4, scale_cache=cache)
