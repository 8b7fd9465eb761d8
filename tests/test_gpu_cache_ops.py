"""The cache operators on the GPU against plain 64-bit computations from
their definitions: append (rotation, fp8 scales, bounds), attention over the
paged cache, block selection and sparse attention.

Bounds of the errors, by the roundings each result passes through (u = 2^-8
for bf16 results, 2^-11 for f16):

  attention   u |o| + (p + 2^-14) A, A = sum_j p_j |v_j|: one rounding of the
              result; p of the weights' rounding, 2^-8 (bf16) or 2^-11 (f16);
              2^-14 for scores, exponentials and sums in 32 bits (dots of up
              to 256 terms, exponents below 64)
  keys        u |k| + 2^-22 (|x_i| + |x_j|): one rounding, two products and a
              sum in 32 bits
  fp8 codes   2^-4 of the value, or half the smallest subnormal, 2^-10, times
              the scale
Values, scales, bounds and selections are exact.
"""
import math

import numpy as np
import pytest
import torch

from gpu_common import need_gpu
from paper_2609_33762_amd import api

pytestmark = pytest.mark.gpu

BF16, F16, FP8 = torch.bfloat16, torch.float16, torch.float8_e4m3fn
ULP = {BF16: 2.0 ** -8, F16: 2.0 ** -11}


class Setup:
    """A cache of one shape filled with numbers, tables of random pages, and
    NaN in every slot that no sequence holds."""

    def __init__(self, kv_lens, rows, heads=2, group=2, dim=64, page=16, act=BF16, fp8=False,
                 layers=2, layer=1, seed=0, bounds=False, pow2=True, spare=3):
        need_gpu()
        self.g = torch.Generator().manual_seed(seed)
        self.H, self.G, self.D, self.T, self.act, self.fp8 = heads, group, dim, page, act, fp8
        self.kv_lens, self.rows, self.layer = list(kv_lens), list(rows), layer
        counts = [-(-k // page) for k in kv_lens]
        self.P = sum(counts) + spare
        perm = torch.randperm(self.P, generator=self.g)
        width = max(counts + [1]) + 2
        self.table = torch.full((len(counts), width), -1, dtype=torch.int32)
        at = 0
        for s, c in enumerate(counts):
            self.table[s, :c] = perm[at:at + c].int()
            at += c
        shape = (layers, self.P, 2, page, heads, dim)
        kind = FP8 if fp8 else act
        x = torch.randn(shape, generator=self.g) * (60 if fp8 else 1)
        self.cache = x.clamp(-448, 448).to(kind)
        held = torch.zeros((self.P, page), dtype=torch.bool)
        for s, k in enumerate(self.kv_lens):
            for p in range(counts[s]):
                held[self.table[s, p].item(), :max(0, min(page, k - p * page))] = True
        raw = self.cache.view(torch.uint8 if fp8 else torch.int16)
        raw.masked_fill_(~held[None, :, None, :, None, None], 0x7f if fp8 else 0x7fff)
        self.scales = None
        if fp8:
            e = torch.rand((layers, self.P, 2, heads), generator=self.g) * 3 - 8
            self.scales = torch.exp2(e.round() if pow2 else e).float()
        self.starts = [sum(self.rows[:i]) for i in range(len(rows) + 1)]
        self.n_rows = self.starts[-1]
        dev = lambda t: None if t is None else t.cuda()  # noqa: E731
        self.d_cache, self.d_scales = dev(self.cache), dev(self.scales)
        self.d_bounds = self.d_bscales = None
        if bounds:
            self.d_bounds = torch.full((layers, self.P, 2, heads, dim), 77, dtype=torch.int8,
                                       device="cuda")
            self.d_bscales = torch.full((layers, self.P, heads), math.nan, device="cuda")
        self.handle = api.Cache(self.d_cache, self.P, layers, page, heads, dim, 1 if fp8 else 2,
                                head_scales=self.d_scales, bounds=self.d_bounds,
                                bound_scales=self.d_bscales)
        self.batch = api.Batch(self.table.cuda(), torch.tensor(self.kv_lens, dtype=torch.int32,
                                                               device="cuda"),
                               max(self.kv_lens + [1]),
                               torch.tensor(self.starts, dtype=torch.int32, device="cuda"),
                               self.n_rows, max(self.rows + [1]))

    def rand(self, heads):
        return torch.randn((self.n_rows, heads, self.D), generator=self.g).to(self.act)

    def stored(self, s, which, h, cache=None, scales=None):
        """Keys (0) or values (1) of sequence s and head h in 64 bits."""
        k = self.kv_lens[s]
        cache = self.cache if cache is None else cache
        scales = self.scales if scales is None else scales
        out = torch.zeros((k, self.D), dtype=torch.float64)
        for p in range(-(-k // self.T)):
            page, n = int(self.table[s, p]), min(self.T, k - p * self.T)
            x = cache[self.layer, page, which, :n, h].double()
            if self.fp8:
                x = x * scales[self.layer, page, which, h].double()
            out[p * self.T:p * self.T + n] = x
        return out


def attention64(st, q, scale, window=0, selected=None):
    """(output, sum of weights times |v|, log-sum-exp) in 64 bits."""
    o = torch.zeros((st.n_rows, st.H * st.G, st.D), dtype=torch.float64)
    a, lse = torch.zeros_like(o), torch.full((st.n_rows, st.H * st.G), -math.inf,
                                             dtype=torch.float64)
    for s, n in enumerate(st.rows):
        for h in range(st.H):
            k, v = st.stored(s, 0, h), st.stored(s, 1, h)
            tok = torch.arange(st.kv_lens[s])
            for r in range(n):
                pos, row = st.kv_lens[s] - n + r, st.starts[s] + r
                see = tok <= pos
                if window:
                    see &= tok > pos - window
                if selected is not None:
                    ids = selected[row, h]
                    see &= torch.isin(tok // st.T, ids[ids >= 0].long())
                if not see.any():
                    continue
                for j in range(st.G):
                    x = (k[see] @ q[row, h * st.G + j].double()) * scale
                    w = torch.softmax(x, 0)
                    o[row, h * st.G + j] = w @ v[see]
                    a[row, h * st.G + j] = w @ v[see].abs()
                    lse[row, h * st.G + j] = torch.logsumexp(x, 0)
    return o, a, lse


def check_attention(st, q, out, lse, scale, weights, **kw):
    o, a, want_lse = attention64(st, q, scale, **kw)
    got = out.cpu().double()
    assert torch.isfinite(got).all()
    bound = ULP[st.act] * o.abs() + (weights + 2.0 ** -14) * a + 2.0 ** -25
    bad = (got - o).abs() > bound
    assert not bad.any(), (int(bad.sum()), float(((got - o).abs() / bound).max()),
                           torch.nonzero(bad)[:4].tolist())
    got_lse = lse.cpu().double()
    empty = torch.isinf(want_lse)
    assert torch.equal(empty, torch.isinf(got_lse))
    assert ((got_lse - want_lse)[~empty].abs() < 1e-4 * (1 + want_lse[~empty].abs())).all()


def attend_case(weights, window=0, scale=None, strided=False, **kw):
    st = Setup(**kw)
    HQ = st.H * st.G
    if strided:  # a slice of a wider row, and an output with the heads outside
        wide = torch.randn((st.n_rows, HQ + 5, st.D), generator=st.g).to(st.act)
        d_q = wide.cuda()[:, 3:3 + HQ]
        q = wide[:, 3:3 + HQ]
        out = torch.empty((HQ, st.n_rows, st.D), dtype=st.act, device="cuda").transpose(0, 1)
    else:
        q = st.rand(HQ)
        d_q = q.cuda()
        out = torch.empty_like(d_q)
    out.fill_(math.nan)
    lse = torch.full((st.n_rows, HQ), 7.0, device="cuda")
    scale = st.D ** -0.5 if scale is None else scale
    st.handle.attend(st.layer, st.batch, d_q, out, scale=scale, window=window, lse=lse)
    check_attention(st, q, out, lse, scale, weights, window=window)


DECODE = [
    dict(kv_lens=[1, 2, 15, 16, 17, 31, 33, 100], rows=[1] * 8),
    dict(kv_lens=[40, 7], rows=[1, 1], heads=1, group=1, dim=8),
    dict(kv_lens=[0, 5, 70], rows=[1, 1, 1], heads=3, group=5, dim=80),
    dict(kv_lens=[130, 257, 64], rows=[1, 1, 1], heads=4, group=8, dim=128),
    dict(kv_lens=[700, 1500], rows=[1, 1], heads=1, group=8, dim=128),
    dict(kv_lens=[90], rows=[1], heads=1, group=16, dim=256),
    dict(kv_lens=[61, 20], rows=[1, 1], heads=2, group=3, dim=136),
    dict(kv_lens=[61, 20, 300], rows=[1, 1, 1], heads=2, group=3, dim=72, page=5),
    dict(kv_lens=[61, 20, 300], rows=[1, 1, 1], heads=1, group=4, dim=96, page=1),
    dict(kv_lens=[61, 200, 300], rows=[1, 1, 1], heads=2, group=2, dim=64, page=48),
    dict(kv_lens=[33, 50], rows=[1, 1], heads=1, group=40, dim=64),
]


@pytest.mark.parametrize("shape", DECODE)
@pytest.mark.parametrize("kind", ["bf16", "f16", "fp8", "fp8_f16"])
def test_attend_single_tokens(shape, kind):
    f16 = kind.endswith("f16") and kind != "bf16"
    attend_case(2.0 ** -11 if kind == "f16" else 2.0 ** -15, act=F16 if f16 else BF16,
                fp8=kind.startswith("fp8"), pow2=False, **shape)


@pytest.mark.parametrize("kind", ["bf16", "f16", "fp8"])
@pytest.mark.parametrize("shape", [
    dict(kv_lens=[5, 40, 33, 300], rows=[3, 4, 1, 2], heads=2, group=5, dim=128),
    dict(kv_lens=[3, 2, 90, 17], rows=[3, 2, 7, 5], heads=1, group=8, dim=64),
    dict(kv_lens=[50, 9], rows=[6, 5], heads=3, group=1, dim=80, page=7),
    # fewer cached tokens than rows: the first rows attend to nothing
    dict(kv_lens=[2, 0, 40], rows=[4, 3, 4], heads=2, group=2, dim=64),
])
@pytest.mark.parametrize("window", [0, 1, 20])
def test_attend_few_rows(shape, kind, window):
    attend_case(2.0 ** -11 if kind == "f16" else 2.0 ** -15, window=window, strided=True,
                act=F16 if kind == "f16" else BF16, fp8=kind == "fp8", **shape)


@pytest.mark.parametrize("kind", ["bf16", "f16", "fp8", "fp8_f16"])
@pytest.mark.parametrize("shape", [
    dict(kv_lens=[130], rows=[130], heads=1, group=2, dim=64),
    dict(kv_lens=[300, 65, 200], rows=[40, 65, 1], heads=2, group=4, dim=128),
    dict(kv_lens=[190, 70], rows=[33, 70], heads=1, group=5, dim=80),
    dict(kv_lens=[100, 77], rows=[20, 30], heads=1, group=3, dim=256, page=5),
    dict(kv_lens=[40, 0, 90], rows=[66, 70, 90], heads=2, group=1, dim=72),
])
@pytest.mark.parametrize("window", [0, 50])
def test_attend_chunks(shape, kind, window):
    f16 = kind in ("f16", "fp8_f16")
    attend_case(2.0 ** -8 if kind == "bf16" else 2.0 ** -11, window=window,
                act=F16 if f16 else BF16, fp8=kind.startswith("fp8"), pow2=False, **shape)


def test_attend_long_context_is_split_and_joined():
    attend_case(2.0 ** -15, kv_lens=[6000, 40, 3001], rows=[1, 1, 1], heads=1, group=4, dim=128)
    attend_case(2.0 ** -15, kv_lens=[5000, 333], rows=[2, 1], heads=1, group=4, dim=64,
                fp8=True, window=2500)
    attend_case(2.0 ** -8, kv_lens=[4100], rows=[40], heads=1, group=2, dim=64)
    attend_case(2.0 ** -11, kv_lens=[3500, 3000, 40], rows=[40, 1, 2], heads=1, group=2, dim=64,
                fp8=True)


def test_attend_scores_far_apart():
    # weights from 1 down to underflow, in both signs
    attend_case(2.0 ** -15, kv_lens=[500, 60], rows=[1, 1], heads=1, group=4, dim=64, scale=1.5)
    attend_case(2.0 ** -11, kv_lens=[500], rows=[1], heads=1, group=4, dim=64, act=F16,
                scale=1.5)
    attend_case(2.0 ** -8, kv_lens=[200], rows=[100], heads=1, group=1, dim=64, scale=1.5)


def test_attend_reads_the_cache_s_own_scales():
    # one scale for all heads of a block: the cache's plane [L][P][2]
    st = Setup(kv_lens=[70, 33], rows=[1, 1], heads=2, group=2, dim=64, fp8=True)
    plane = st.scales[..., 0].contiguous()
    st.scales = plane[..., None].expand(-1, -1, -1, st.H).contiguous()
    h = api.Cache(st.d_cache, st.P, 2, st.T, st.H, st.D, 1, scales=plane.cuda())
    q = st.rand(st.H * st.G)
    out = torch.empty_like(q, device="cuda")
    lse = torch.empty((st.n_rows, st.H * st.G), device="cuda")
    h.attend(st.layer, st.batch, q.cuda(), out, lse=lse)
    check_attention(st, q, out, lse, st.D ** -0.5, 2.0 ** -15)


@pytest.mark.parametrize("rows", [1, 40])
def test_attend_pages_outside_the_cache_hold_no_tokens(rows):
    st = Setup(kv_lens=[100], rows=[rows], heads=1, group=2, dim=64)
    q = st.rand(2)
    table = st.table.clone()
    table[0, 2], table[0, 4] = st.P, -3
    b = api.Batch(table.cuda(), st.batch.kv_len, 100, st.batch.row_start, rows, rows)
    out = torch.empty_like(q, device="cuda")
    lse = torch.empty((rows, 2), device="cuda")
    st.handle.attend(st.layer, b, q.cuda(), out, lse=lse)
    ids = torch.tensor([0, 1, 3, 5, 6]).expand(rows, 1, 5)
    check_attention(st, q, out, lse, st.D ** -0.5, 2.0 ** -8 if rows > 1 else 2.0 ** -15,
                    selected=ids)


# ------------------------------------------------------------------ append

def rope_table(n, dim):
    inv = 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
    ang = torch.arange(n, dtype=torch.float64)[:, None] * inv
    return torch.cat([ang.cos(), ang.sin()], 1).float()


def turn64(x, rope, pos, interleaved):
    """Rotated rows [n, heads, D] and the sums of magnitudes, in 64 bits."""
    x, dim = x.double().clone(), rope.shape[1]
    mag = x.abs()
    c, s = rope[pos, :dim // 2].double()[:, None], rope[pos, dim // 2:].double()[:, None]
    i = torch.arange(0, dim, 2) if interleaved else torch.arange(dim // 2)
    j = i + 1 if interleaved else i + dim // 2
    a, b = x[..., i].clone(), x[..., j].clone()
    x[..., i], x[..., j] = a * c - b * s, b * c + a * s
    both = a.abs() + b.abs()
    mag[..., i], mag[..., j] = both, both
    return x, mag


def power(amax, top):
    """The smallest power of two s >= 2^-126 with top * s >= amax."""
    e = -126
    while top * 2.0 ** e < amax:
        e += 1
    return 2.0 ** e


def append_case(rope_dim, interleaved=False, seed=0, grow=1.0, **kw):
    """Appends, then compares every byte of the cache and the planes."""
    st = Setup(seed=seed, bounds=True, **kw)
    HQ, T = st.H * st.G, st.T
    qkv = (torch.randn((st.n_rows, HQ + 2 * st.H, st.D), generator=st.g) * grow).to(st.act)
    d_qkv = qkv.cuda()
    q, k, v = qkv[:, :HQ], qkv[:, HQ:HQ + st.H], qkv[:, HQ + st.H:]
    d_q, d_k, d_v = d_qkv[:, :HQ], d_qkv[:, HQ:HQ + st.H], d_qkv[:, HQ + st.H:]
    rope = rope_table(max(st.kv_lens), rope_dim) if rope_dim else torch.cat(
        [torch.ones(max(st.kv_lens), st.D // 2), torch.zeros(max(st.kv_lens), st.D // 2)], 1)
    q_out = torch.full((st.n_rows, HQ, st.D), math.nan, dtype=st.act, device="cuda")
    st.handle.append_kv(st.layer, st.batch, d_k, d_v, rope=rope.cuda() if rope_dim else None,
                        q=d_q, q_out=q_out, interleaved=interleaved)
    torch.cuda.synchronize()
    got, raw0 = st.d_cache.cpu(), st.cache.view(torch.uint8)
    raw = got.view(torch.uint8).clone()
    scales = st.d_scales.cpu() if st.fp8 else None
    u = ULP[st.act]
    for s, n in enumerate(st.rows):
        start = st.kv_lens[s] - n
        rows = torch.arange(max(0, -start), n) + st.starts[s]
        pos = torch.arange(max(start, 0), st.kv_lens[s])
        want_q, mq = turn64(q[rows], rope, pos, interleaved)
        err = (q_out.cpu()[rows].double() - want_q).abs()
        assert (err <= u * want_q.abs() + 2.0 ** -22 * mq).all()
        want_k, mk = turn64(k[rows], rope, pos, interleaved)
        for p in sorted({int(x) // T for x in pos}):
            page = int(st.table[s, p])
            i0, i1 = max(max(start, 0) - p * T, 0), min(st.kv_lens[s] - p * T, T)
            here = (pos >= p * T) & (pos < p * T + T)
            for h in range(st.H):
                for which, want, mag in ((0, want_k[here, h], mk[here, h]),
                                         (1, v[rows][here, h].double(), None)):
                    new = got[st.layer, page, which, i0:i1, h].double()
                    if st.fp8:
                        s0 = float(st.scales[st.layer, page, which, h])
                        s1 = float(scales[st.layer, page, which, h])
                        need = power(float(want.abs().max()), 448.0)
                        need = max(need, s0) if i0 else need
                        # a rotated key on the edge of a power may go either way
                        edge = which == 0 and abs(float(want.abs().max()) / need / 448 * 2 - 1) < 1e-5
                        assert s1 == need or edge, (page, which, h, s0, s1, need)
                        if which == 1:
                            assert torch.equal(new, (want / s1).float().to(FP8).double())
                        else:
                            assert ((new * s1 - want).abs() <= 2.0 ** -4 * want.abs() +
                                    2.0 ** -10 * s1 + 2.0 ** -20 * mag).all()
                        old = st.cache[st.layer, page, which, :i0, h]
                        again = (old.float() * (s0 / s1)).to(FP8) if s1 != s0 else old
                        assert torch.equal(
                            got[st.layer, page, which, :i0, h].view(torch.uint8),
                            again.view(torch.uint8))
                    elif which == 1:
                        assert torch.equal(new, want)
                    else:
                        assert ((new - want).abs() <= u * want.abs() + 2.0 ** -22 * mag).all()
                # bounds of the block from what is stored now
                x = got[st.layer, page, 0, :i1, h].double()
                if st.fp8:
                    x = x * float(scales[st.layer, page, 0, h])
                unit = power(float(x.abs().max()), 127.0)
                assert float(st.d_bscales[st.layer, page, h]) == unit
                b = st.d_bounds[st.layer, page, :, h].cpu().double()
                assert torch.equal(b[0], (x.amin(0) / unit).floor())
                assert torch.equal(b[1], (x.amax(0) / unit).ceil())
            # checked: everything else has to be as it was
            stop = i1 if st.fp8 else None
            lo = 0 if st.fp8 else i0
            raw.view(got.dtype)[st.layer, page, :, lo:i1] = st.cache[st.layer, page, :, lo:i1]
            assert stop is None or stop == i1
    assert torch.equal(raw, raw0)


APPENDS = [
    dict(kv_lens=[1, 16, 17, 40], rows=[1, 1, 1, 1]),
    dict(kv_lens=[50, 16, 33, 5], rows=[20, 16, 33, 3], heads=3, dim=80, group=1),
    dict(kv_lens=[100, 31], rows=[37, 2], heads=1, dim=128, group=8),
    dict(kv_lens=[23, 9, 4], rows=[11, 9, 1], heads=2, dim=72, page=5),
    dict(kv_lens=[70, 64], rows=[1, 64], heads=2, dim=256, page=64, group=3),
    dict(kv_lens=[3, 30], rows=[5, 2], heads=2, dim=8, group=1, page=1),
]


@pytest.mark.parametrize("shape", APPENDS)
@pytest.mark.parametrize("kind", ["bf16", "f16", "fp8", "fp8_f16"])
@pytest.mark.parametrize("grow", [1.0, 40.0])
def test_append(shape, kind, grow):
    f16 = kind in ("f16", "fp8_f16")
    append_case(shape.get("dim", 64), act=F16 if f16 else BF16, fp8=kind.startswith("fp8"),
                grow=grow, **shape)


@pytest.mark.parametrize("rope_dim,interleaved", [(0, False), (2, False), (32, True), (48, False),
                                                  (20, True), (20, False), (64, True)])
@pytest.mark.parametrize("fp8", [False, True])
def test_append_rotations(rope_dim, interleaved, fp8):
    append_case(rope_dim, interleaved, kv_lens=[50, 16, 33], rows=[20, 1, 33], fp8=fp8)


def test_append_queries_in_place_and_keys_alone():
    st = Setup(kv_lens=[20, 33], rows=[4, 7], heads=1, group=2, dim=128)
    q, k, v = st.rand(2), st.rand(1), st.rand(1)
    rope = rope_table(33, 128).cuda()
    d_q, apart = q.cuda(), torch.empty_like(q, device="cuda")
    st.handle.append_kv(0, st.batch, k.cuda(), v.cuda(), rope=rope, q=d_q, q_out=apart)
    st.handle.append_kv(1, st.batch, k.cuda(), v.cuda(), rope=rope)
    st.handle.append_kv(0, st.batch, k.cuda(), v.cuda(), rope=rope, q=d_q, q_out=d_q)
    assert torch.equal(d_q, apart)
    c = st.d_cache.cpu().view(torch.int16)
    for s, n in enumerate(st.rows):
        for i in range(st.kv_lens[s] - n, st.kv_lens[s]):
            page = int(st.table[s, i // st.T])
            assert torch.equal(c[0, page, :, i % st.T], c[1, page, :, i % st.T])


def test_append_fp8_values_that_are_not_finite():
    st = Setup(kv_lens=[3], rows=[3], heads=1, group=1, dim=8, fp8=True, bounds=True, page=16)
    k = torch.ones((3, 1, 8), dtype=BF16)
    v = torch.zeros((3, 1, 8), dtype=BF16)
    k[0, 0, 0], k[1, 0, 1], k[2, 0, 2] = math.inf, -math.inf, math.nan
    st.handle.append_kv(1, st.batch, k.cuda(), v.cuda())
    page = int(st.table[0, 0])
    got = st.d_cache[1, page, :, :3, 0].cpu().float()
    assert torch.equal(torch.isnan(got[0]), ~torch.isfinite(k[:, 0].float()))
    sk, sv = st.d_scales[1, page, :, 0].tolist()
    assert sk == power(1.0, 448.0) and sv == 2.0 ** -126
    assert (got[1] == 0).all() and (got[0][torch.isfinite(got[0])] * sk == 1.0).all()


# --------------------------------------------------- selection, sparse attention

def select64(st, q, budget, first, last):
    """Blocks from the bounds planes in whole numbers and 64 bits."""
    bounds, units = st.d_bounds[st.layer].cpu().long(), st.d_bscales[st.layer].cpu().double()
    out = torch.full((st.n_rows, st.H, budget), -1, dtype=torch.int32)
    for s, n in enumerate(st.rows):
        for r in range(n):
            pos, row = st.kv_lens[s] - n + r, st.starts[s] + r
            held = pos // st.T + 1 if pos >= 0 else 0
            for h in range(st.H):
                score = []
                for b in range(held):
                    page = int(st.table[s, b])
                    lo, hi = bounds[page, 0, h], bounds[page, 1, h]
                    best = -math.inf
                    for j in range(st.G):
                        x = q[row, h * st.G + j].double()
                        unit = power(float(x.abs().max()), 127.0)
                        c = (x / unit).round().long()
                        best = max(best, float(torch.maximum(c * lo, c * hi).sum()) * unit *
                                   float(units[page, h]))
                    if b < first or b >= held - last:
                        best = math.inf
                    score.append(best)
                order = sorted(range(held), key=lambda b: (-score[b], b))[:budget]
                out[row, h, :len(order)] = torch.tensor(sorted(order), dtype=torch.int32)
    return out


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("shape,budget,first,last", [
    (dict(kv_lens=[200, 16, 1, 333], rows=[1, 1, 1, 1]), 4, 1, 1),
    (dict(kv_lens=[200, 90], rows=[3, 2], heads=1, group=5, dim=128), 5, 1, 2),
    (dict(kv_lens=[60, 45], rows=[1, 2], heads=3, group=1, dim=80, page=5), 3, 0, 0),
    (dict(kv_lens=[700], rows=[1], heads=1, group=20, dim=72), 11, 2, 1),
    (dict(kv_lens=[2, 0, 100], rows=[3, 1, 1], heads=1, group=2, dim=256, page=8), 6, 1, 1),
    (dict(kv_lens=[1500], rows=[1], heads=1, group=1, dim=8, page=1), 100, 0, 1),
])
def test_select_and_sparse_attention(shape, budget, first, last, fp8):
    if shape.get("dim") == 256 and shape["group"] > 16 or shape.get("dim", 64) > 128 and \
            shape.get("group", 2) > 16:
        pytest.skip("not a shape of the sparse kernel")
    st = Setup(fp8=fp8, bounds=True, **shape)
    pages = torch.arange(st.P, dtype=torch.int32, device="cuda")
    # bounds of whole blocks; the slots that hold NaN do not count
    st.handle.bound_blocks(pages)
    assert (st.d_bounds[0] != 77).any()
    q = st.rand(st.H * st.G)
    d_q = q.cuda()
    sel = torch.full((st.n_rows, st.H, budget), 9, dtype=torch.int32, device="cuda")
    st.handle.select_blocks(st.layer, st.batch, d_q, sel, first=first, last=last)
    want = select64(st, q, budget, first, last)
    assert torch.equal(sel.cpu(), want)
    out = torch.full_like(d_q, math.nan)
    lse = torch.empty((st.n_rows, st.H * st.G), device="cuda")
    st.handle.attend(st.layer, st.batch, d_q, out, selected=sel, lse=lse)
    check_attention(st, q, out, lse, st.D ** -0.5, 2.0 ** -15, selected=want)


def test_select_ties_go_to_the_lower_block():
    st = Setup(kv_lens=[40 * 16], rows=[1], heads=1, group=1, dim=64, bounds=True)
    st.d_bounds.zero_()
    st.d_bscales.fill_(1.0)
    st.d_bounds[1, st.table[0, 17].item(), 1].fill_(5)
    q = torch.ones((1, 1, 64), dtype=BF16, device="cuda")
    sel = torch.empty((1, 1, 6), dtype=torch.int32, device="cuda")
    st.handle.select_blocks(1, st.batch, q, sel, first=1, last=1)
    assert sel.flatten().tolist() == [0, 1, 2, 3, 17, 39]


def test_selections_of_another_maker():
    # unordered, short, and out of range: what is not a block of the sequence
    # is skipped
    st = Setup(kv_lens=[150], rows=[1], heads=1, group=3, dim=64)
    q = st.rand(3)
    ids = torch.tensor([[[7, 2, -1, 99, 0, 1 << 30, -5, 9]]], dtype=torch.int32)
    out = torch.empty_like(q, device="cuda")
    lse = torch.empty((1, 3), device="cuda")
    st.handle.attend(st.layer, st.batch, q.cuda(), out, selected=ids.cuda(), lse=lse)
    check_attention(st, q, out, lse, st.D ** -0.5, 2.0 ** -15,
                    selected=torch.tensor([[[7, 2, 0, 9]]]))


# ------------------------------------------------------- streams and graphs

def test_a_step_on_another_stream_and_in_a_graph():
    st = Setup(kv_lens=[600, 90, 17], rows=[1, 1, 1], heads=2, group=4, dim=128, fp8=True,
               bounds=True)
    pages = torch.arange(st.P, dtype=torch.int32, device="cuda")
    q, k, v = (st.rand(n).cuda() for n in (8, 2, 2))
    rope = rope_table(600, 128).cuda()
    q_out, out = torch.empty_like(q), torch.empty_like(q)
    sel = torch.empty((3, 2, 5), dtype=torch.int32, device="cuda")

    def step():
        st.handle.append_kv(1, st.batch, k, v, rope=rope, q=q, q_out=q_out)
        st.handle.select_blocks(1, st.batch, q_out, sel)
        st.handle.attend(1, st.batch, q_out, out, selected=sel)
        st.handle.attend(1, st.batch, q_out, full)

    full = torch.empty_like(q)
    st.handle.bound_blocks(pages)
    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in (st.d_cache.view(torch.uint8), st.d_scales, st.d_bounds, q_out, sel,
                                out, full)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t in (q_out, out, full):
        t.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    now = [st.d_cache.view(torch.uint8), st.d_scales, st.d_bounds, q_out, sel, out, full]
    for a, b in zip(now, want):
        assert torch.equal(a, b)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        step()
    for i in range(4):
        q.copy_(torch.randn(q.shape, generator=st.g).to(q.dtype).cuda())
        k.mul_(1.0 + i)
        torch.cuda.synchronize()
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in now]
        for t in (q_out, out, full):
            t.zero_()
        sel.fill_(-7)
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(now, want):
            assert torch.equal(a, b)


def test_two_streams_at_once_share_a_batch():
    st = Setup(kv_lens=[5000, 40], rows=[1, 1], heads=1, group=4, dim=128)
    q = st.rand(4).cuda()
    outs = [torch.empty_like(q) for _ in range(6)]
    st.handle.attend(1, st.batch, q, outs[0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i, o in enumerate(outs[1:]):
        st.handle.attend(1, st.batch, q, o, stream=streams[i % 2])
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert torch.equal(o, outs[0])


def test_results_do_not_change_from_call_to_call():
    st = Setup(kv_lens=[5000, 2000, 300], rows=[40, 1, 3], heads=2, group=4, dim=64, fp8=True)
    q = st.rand(8).cuda()
    outs = [torch.empty_like(q) for _ in range(4)]
    for o in outs:
        st.handle.attend(1, st.batch, q, o)
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert torch.equal(o, outs[0])


# ------------------------------------------------------------------ refusals

def test_refusals():
    st = Setup(kv_lens=[40, 20], rows=[1, 1], heads=2, group=2, dim=64, bounds=True)
    q, k = st.rand(4).cuda(), st.rand(2).cuda()
    out = torch.full_like(q, 3.0)
    c, b = st.handle, st.batch

    def refused(f, *a, **kw):
        with pytest.raises((ValueError, api.EAError)):
            f(*a, **kw)

    refused(c.attend, 2, b, q, out)                       # no such layer
    refused(c.attend, -1, b, q, out)
    refused(c.attend, 0, b, q, out.to(F16))               # two types
    refused(c.attend, 0, b, q.float(), out.float())
    refused(c.attend, 0, b, q, out, scale=0.0)
    refused(c.attend, 0, b, q, out, scale=math.nan)
    refused(c.attend, 0, b, q, out, window=-1)
    refused(c.attend, 0, b, q[:, :3], out[:, :3])         # no multiple of H
    refused(c.attend, 0, b, q[:1], out)                   # a row is missing
    refused(c.attend, 0, b, q[..., ::2], out)             # elements apart
    refused(c.attend, 0, b, q.cpu(), out)
    odd = torch.empty(2 * 4 * 64 + 8, dtype=BF16, device="cuda")[1:513].view(2, 4, 64)
    refused(c.attend, 0, b, odd, out)                     # not aligned
    sel = torch.zeros((2, 2, 4), dtype=torch.int32, device="cuda")
    refused(c.attend, 0, b, q, out, selected=sel, window=3)
    refused(c.attend, 0, b, q, out, selected=sel.long())
    refused(c.select_blocks, 0, b, q, sel, first=3, last=2)
    refused(c.append_kv, 0, b, k, k[:, :1])
    refused(c.append_kv, 0, b, k, k, rope=rope_table(39, 64).cuda())   # too short
    refused(c.append_kv, 0, b, k, k, rope=rope_table(40, 66).cuda())   # too wide
    refused(c.append_kv, 0, b, k, k, q=q)                 # no place for q
    short = api.Batch(st.table.cuda()[:, :2].contiguous(), b.kv_len, 40, b.row_start, 2, 1)
    refused(c.attend, 0, short, q, out)                   # table too narrow
    with pytest.raises(ValueError):
        api.Batch(st.table.cuda(), b.kv_len[:1], 40)
    plain = api.Cache(st.d_cache, st.P, 2, 16, 2, 64, 2)
    refused(plain.select_blocks, 0, b, q, sel)            # no bounds
    fp8 = api.Cache(st.d_cache, st.P, 2, 16, 2, 64, 1)
    refused(fp8.attend, 0, b, q, out)                     # no scales
    page = api.Cache(st.d_cache, st.P, 2, 16, 2, 64, 1,
                     scales=torch.ones((2, st.P, 2), device="cuda"))
    refused(page.append_kv, 0, b, k, k)                   # one scale for two heads
    with pytest.raises(ValueError):
        api.Cache(st.d_cache, st.P, 2, 16, 2, 64, 1,
                  head_scales=torch.ones((2, st.P, 2), device="cuda"))
    torch.cuda.synchronize()
    assert (out == 3.0).all()
    assert torch.equal(st.d_cache.cpu().view(torch.int16), st.cache.view(torch.int16))


def test_an_empty_step():
    st = Setup(kv_lens=[40, 20], rows=[0, 0], heads=2, group=2, dim=64)
    z = torch.empty((0, 4, 64), dtype=BF16, device="cuda")
    b = api.Batch(st.table.cuda(), st.batch.kv_len, 40, st.batch.row_start, 0, 0)
    st.handle.attend(0, b, z, z)
    st.handle.append_kv(0, b, z[:, :2], z[:, :2])
    np.testing.assert_equal(st.d_cache.cpu().view(torch.int16).numpy(),
                            st.cache.view(torch.int16).numpy())
