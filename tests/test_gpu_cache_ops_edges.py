"""The cache operators where values are not finite, planes hold garbage, caches
pass 4 GiB and pages end inside a tile.  The bounds of the errors are those of
tests/test_gpu_cache_ops.py."""
import math

import pytest
import torch

import test_gpu_cache_ops as base
from gpu_common import need_gpu
from paper_2609_33762_amd import api

pytestmark = pytest.mark.gpu

BF16, F16, FP8 = base.BF16, base.F16, base.FP8
ODD = {BF16: (0x7FC0, 0x7F80, 0xFF80), F16: (0x7E00, 0x7C00, 0xFC00)}  # NaN and infinities


def plant(st, s, tokens, h, dims):
    """Values that are not finite at these tokens of a sequence and a head."""
    raw = st.cache.view(torch.uint8 if st.fp8 else torch.int16)
    for i, (t, d) in enumerate((t, d) for t in tokens for d in dims):
        page, slot = int(st.table[s, t // st.T]), t % st.T
        code = 0x7F if st.fp8 else ODD[st.act][i % 3]
        raw[st.layer, page, 1, slot, h, d] = code if code < 0x8000 else code - 0x10000
    st.d_cache.copy_(st.cache.cuda())


def check_odd(st, window=0, selected=None, weights=2.0 ** -8, scale=None):
    q = st.rand(st.H * st.G)
    out = torch.full_like(q, 7.0, device="cuda")
    lse = torch.empty((st.n_rows, st.H * st.G), device="cuda")
    scale = st.D ** -0.5 if scale is None else scale
    st.handle.attend(st.layer, st.batch, q.cuda(), out, scale=scale, window=window, lse=lse)
    o, a, want_lse = base.attention64(st, q, scale, window=window)
    got, fine = out.cpu().double(), torch.isfinite(o)
    assert 0 < int((~fine).sum()) < fine.numel() // 2
    assert torch.equal(torch.isfinite(got), fine)
    bound = base.ULP[st.act] * o.abs() + (weights + 2.0 ** -14) * a + 2.0 ** -25
    assert ((got - o).abs() <= bound)[fine].all()
    # an infinity stays one (weights that vanish in 32 bits aside)
    inf = torch.isinf(o)
    assert torch.equal(got[inf], o[inf])
    assert ((lse.cpu().double() - want_lse).abs() < 1e-4 * (1 + want_lse.abs())).all()


KINDS = [("bf16", BF16, False), ("f16", F16, False), ("fp8", BF16, True), ("fp8_f16", F16, True)]


@pytest.mark.parametrize("kind", KINDS, ids=[k[0] for k in KINDS])
@pytest.mark.parametrize("page", [16, 5])
@pytest.mark.parametrize("rows,heads,group,dim", [(4, 2, 4, 64), (5, 1, 8, 128), (60, 2, 1, 72),
                                                  (70, 1, 4, 64), (140, 2, 2, 128),
                                                  (3, 1, 2, 256), (70, 1, 2, 256)])
@pytest.mark.parametrize("window", [0, 30])
def test_values_that_are_not_finite_reach_only_the_rows_that_see_them(rows, heads, group, dim, page,
                                                                      kind, window):
    n = 260
    st = base.Setup(kv_lens=[n, 33], rows=[rows, 2], heads=heads, group=group, dim=dim, page=page,
                    act=kind[1], fp8=kind[2])
    # the newest tokens are seen by the last rows alone, the oldest of the
    # first row's window by the first rows alone
    plant(st, 0, [n - 1, n - 2], 0, [0, 7, dim - 1])
    if window:
        plant(st, 0, [n - rows + 1 - window], heads - 1, [3, 8])
    few = rows * group <= (64 if dim <= 128 else 16)
    check_odd(st, window=window, weights=2.0 ** -11 if kind[0] == "f16" or (kind[2] and not few)
              else 2.0 ** -15 if few else 2.0 ** -8)


@pytest.mark.parametrize("page", [16, 5])
@pytest.mark.parametrize("rows", [1, 4, 70])
@pytest.mark.parametrize("garbage", [math.nan, math.inf, 2.0 ** 100])
def test_scales_of_pages_that_no_row_sees(rows, page, garbage):
    # pages before the window and pages of nobody: their scales do not matter
    n, window = 200, 20
    st = base.Setup(kv_lens=[n], rows=[rows], heads=2, group=2, dim=64, page=page, fp8=True)
    lowest = n - rows + 1 - window
    seen = {int(st.table[0, t // page]) for t in range(max(lowest, 0), n)}
    for p in range(st.P):
        if p not in seen:
            st.scales[:, p] = garbage
    st.d_scales.copy_(st.scales.cuda())
    q = st.rand(4)
    out, lse = torch.empty_like(q, device="cuda"), torch.empty((st.n_rows, 4), device="cuda")
    st.handle.attend(st.layer, st.batch, q.cuda(), out, window=window, lse=lse)
    for p in range(st.P):  # (times zero in the plain form)
        if p not in seen:
            st.scales[:, p] = 1.0
    base.check_attention(st, q, out, lse, st.D ** -0.5, 2.0 ** -11 if rows > 4 else 2.0 ** -15,
                         window=window)


@pytest.mark.parametrize("fp8", [False, True])
def test_places_past_4_gib(fp8):
    # a cache of 5 GiB, the sequences' pages at its end: offsets need more than
    # 32 bits, in bytes and in elements
    need_gpu()
    T, H, D, act = 16, 2, 128, BF16
    eb = 1 if fp8 else 2
    P = 5 * 2 ** 30 // (2 * T * H * D * eb)
    kv = torch.zeros((1, P, 2, T, H, D), dtype=FP8 if fp8 else act, device="cuda")
    scales = torch.zeros((1, P, 2, H), device="cuda") if fp8 else None
    bounds = torch.zeros((1, P, 2, H, D), dtype=torch.int8, device="cuda")
    bscales = torch.zeros((1, P, H), device="cuda")
    big = api.Cache(kv, P, 1, T, H, D, eb, head_scales=scales, bounds=bounds, bound_scales=bscales)
    n, G = 90, 2
    blocks = -(-n // T)
    small = torch.zeros((1, blocks, 2, T, H, D), dtype=kv.dtype, device="cuda")
    s_scales = torch.zeros((1, blocks, 2, H), device="cuda") if fp8 else None
    s_bounds = torch.zeros((1, blocks, 2, H, D), dtype=torch.int8, device="cuda")
    s_bscales = torch.zeros((1, blocks, H), device="cuda")
    near = api.Cache(small, blocks, 1, T, H, D, eb, head_scales=s_scales, bounds=s_bounds,
                     bound_scales=s_bscales)
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn((n, H, D), generator=g).to(act).cuda() for _ in range(2))
    q = torch.randn((n, H * G, D), generator=g).to(act).cuda()
    last = torch.arange(P - blocks, P, dtype=torch.int32, device="cuda")[None]
    first = torch.arange(blocks, dtype=torch.int32, device="cuda")[None]
    kv_len = torch.tensor([n], dtype=torch.int32, device="cuda")
    got = []
    for cache, table in ((big, last), (near, first)):
        b = api.Batch(table, kv_len, n, torch.tensor([0, n], dtype=torch.int32, device="cuda"), n, n)
        cache.append_kv(0, b, k, v)
        chunk = torch.empty_like(q)
        cache.attend(0, b, q, chunk)
        one = api.Batch(table, kv_len, n)
        ids = torch.empty((1, H, 4), dtype=torch.int32, device="cuda")
        cache.select_blocks(0, one, q[-1:], ids)
        outs = [torch.empty_like(q[-1:]) for _ in range(2)]
        cache.attend(0, one, q[-1:], outs[0])
        cache.attend(0, one, q[-1:], outs[1], selected=ids)
        got.append([chunk, ids] + outs)
    torch.cuda.synchronize()
    assert torch.equal(kv[:, -blocks:].view(torch.uint8), small.view(torch.uint8))
    assert torch.equal(bounds[:, -blocks:], s_bounds) and torch.equal(bscales[:, -blocks:], s_bscales)
    assert float(small.float().abs().sum()) > 0 and float(kv[:, 0].float().abs().sum()) == 0
    for x, y in zip(*got):
        assert torch.equal(x, y)


def test_batch_of_more_sequences_than_lanes():
    lens = [(37 * i) % 90 for i in range(150)]
    base.attend_case(2.0 ** -15, kv_lens=lens, rows=[1] * 150, heads=1, group=2, dim=64)
    base.attend_case(2.0 ** -15, kv_lens=lens, rows=[i % 3 for i in range(150)], heads=1, group=2,
                     dim=64, fp8=True)
