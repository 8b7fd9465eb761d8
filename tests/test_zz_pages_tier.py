"""A cache of latents stored to a host tier and loaded back, whole and layer by layer:
its bytes and scales, and attention over the loaded pages, bit for bit."""
import math

import pytest
import torch

from gpu_common import need_gpu
from latent_common import F16, BF16, Latents
from paper_2609_33762_amd import _native as N
from paper_2609_33762_amd import api
from paper_2609_33762_amd import workloads as W

pytestmark = pytest.mark.gpu

KINDS = {"bf16": dict(act=BF16), "f16": dict(act=F16), "fp8": dict(act=BF16, fp8=True)}


def attend(st, handle, q, table):
    batch = api.Batch(torch.tensor(table, dtype=torch.int32, device="cuda"), st.batch.kv_len,
                      max(st.kv_lens), st.batch.row_start, st.n_rows, max(st.rows))
    out = torch.full((st.n_rows, st.H, st.C), math.nan, dtype=st.act, device="cuda")
    lse = torch.full((st.n_rows, st.H), math.nan, device="cuda")
    handle.attend_latent(st.layer, batch, q, out, scale=0.07, lse=lse)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("plan", [N.EA_PLAN_DIRECT, N.EA_PLAN_STAGED])
@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("chunk,latent,turn,page", [(1, 512, 64, 16), (2, 128, 32, 16),
                                                    (1, 384, 48, 5)])
def test_latents_come_back_from_a_tier(chunk, latent, turn, page, kind, plan):
    need_gpu()
    st = Latents([8 * page, 4 * page], [1, 2], heads=4, latent=latent, turn=turn, page=page,
                 spare=14, **KINDS[kind])
    used = [int(p) for p in st.table.flatten() if p >= 0]
    free = [p for p in range(st.P) if p not in used][:len(used)]
    q = st.rand(st.n_rows, st.H, latent + turn).cuda()
    want = attend(st, st.handle, q, st.table.tolist())
    n = len(used) // chunk
    tier = api.Tier(st.handle, (n + 2) * chunk * st.handle.slot_bytes, chunk_pages=chunk)
    tier.set_plan(N.EA_DIR_BOTH, plan)
    keys = W.rng(3).integers(0, 256, size=(n, 32)).astype("uint8")
    taken, slots = tier.alloc(keys)
    assert taken == n
    tier.store(st.handle, used, slots)
    torch.cuda.synchronize()
    tier.unpin(slots)
    hit, found = tier.lookup(keys)
    assert hit == n and (found == slots).all()
    # into other pages of the cache
    tier.load(st.handle, found, free)
    got, scales = st.d_cache.view(torch.uint8).cpu(), st.d_scales
    assert torch.equal(got[:, free], got[:, used])
    assert torch.equal(got[:, used], st.cache.view(torch.uint8)[:, used])
    if scales is not None:
        assert torch.equal(scales[:, free], scales[:, used])
    where = dict(zip(used, free))
    for a, b in zip(attend(st, st.handle, q, [[where.get(int(p), -1) for p in row]
                                              for row in st.table]), want):
        assert torch.equal(a, b)
    # layer by layer into another cache of the shape
    kv = torch.zeros_like(st.d_cache)
    other_scales = None if scales is None else torch.zeros_like(scales)
    other = api.LatentCache(kv, st.P, kv.shape[0], page, latent, turn, 1 if st.fp8 else 2,
                            scales=other_scales)
    copies, events = torch.cuda.Stream(), [torch.cuda.Event() for _ in range(kv.shape[0])]
    copies.wait_stream(torch.cuda.current_stream())
    tier.load_layered(other, found, used, copies, events)
    torch.cuda.current_stream().wait_event(events[st.layer])
    for a, b in zip(attend(st, other, q, st.table.tolist()), want):
        assert torch.equal(a, b)
    torch.cuda.synchronize()
    assert torch.equal(kv.view(torch.uint8).cpu()[:, used], got[:, used])
    tier.unpin(found)
    tier.close()
