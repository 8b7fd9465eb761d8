"""Pages copied and kept tokens moved on the GPU, bit by bit or against the
definition in 64 bits; latents appended.

A moved or appended key passes through two products and a sum in 32 bits, of
magnitudes |x_i| + |x_j| (2^-22 of them), and one rounding: to 16 bits u = 2^-8
(bf16) or 2^-11 (f16) of the value (f16 values below 2^-14 are 2^-24 apart: off by
up to 2^-25, more than 2^-11 of a value below 2^-14; bf16 has the exponents of 32
bits), to fp8 2^-4 of it or half the smallest subnormal, 2^-10, times the block's
scale. Scales are the smallest powers of two that hold their block; values, 16-bit
ones and those that need no new rounding, are exact."""
import math

import pytest
import torch

from gpu_common import need_gpu
from latent_common import BF16, F16, FP8, ULP, Latents
from paper_2609_33762_amd import api

pytestmark = pytest.mark.gpu

TINY = {BF16: 0.0, F16: 2.0 ** -25}


def angles(n, dim):
    inv = 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
    ang = torch.arange(n, dtype=torch.float64)[:, None] * inv
    return torch.cat([ang.cos(), ang.sin()], 1).float()


def turn64(x, rope, by, interleaved):
    """Rows [n, ..., D], leading elements turned by `by` [n] positions, and the
    sums of magnitudes, in 64 bits."""
    x, dim = x.double().clone(), rope.shape[1]
    mag = x.abs()
    shape = (-1,) + (1,) * (x.dim() - 2) + (dim // 2,)
    c = rope[by.abs(), :dim // 2].double().reshape(shape)
    s = (rope[by.abs(), dim // 2:].double() * by.sign()[:, None]).reshape(shape)
    i = torch.arange(0, dim, 2) if interleaved else torch.arange(dim // 2)
    j = i + 1 if interleaved else i + dim // 2
    a, b = x[..., i].clone(), x[..., j].clone()
    x[..., i], x[..., j] = a * c - b * s, b * c + a * s
    both = a.abs() + b.abs()
    mag[..., i], mag[..., j] = both, both
    return x, mag


def power(amax, top=448.0):
    """The smallest power of two s >= 2^-126 with top * s >= amax."""
    e = -126
    while top * 2.0 ** e < amax:
        e += 1
    return 2.0 ** e


# ------------------------------------------------------------------ copies

@pytest.mark.parametrize("shape", [
    dict(page=16, heads=2, dim=64, elem=2, layers=3),
    dict(page=5, heads=1, dim=72, elem=2, layers=2),
    dict(page=16, heads=4, dim=128, elem=1, layers=4, planes=True),
    dict(page=64, heads=3, dim=40, elem=1, layers=2, planes=True),
    dict(page=1, heads=1, dim=24, elem=1, layers=1, planes=True),
    dict(page=300, heads=8, dim=128, elem=2, layers=1, planes=True),
    dict(page=16, heads=1, dim=288, elem=1, layers=2),
], ids=str)
def test_copied_pages_bit_by_bit(shape):
    need_gpu()
    P, L, H, D, T = 23, shape["layers"], shape["heads"], shape["dim"], shape["page"]
    g = torch.Generator(device="cuda").manual_seed(3)
    byte = lambda *s: torch.randint(0, 256, s, dtype=torch.uint8, device="cuda",  # noqa: E731
                                    generator=g)
    kv = byte(L, P, 2 * T * H * D * shape["elem"])
    scales = byte(L, P, 8)
    planes = {}
    if shape.get("planes"):
        planes = dict(head_scales=byte(L, P, 8 * H).view(torch.float32),
                      bounds=byte(L, P, 2 * H * D).view(torch.int8),
                      bound_scales=byte(L, P, 4 * H).view(torch.float32))
    c = api.Cache(kv, P, L, T, H, D, shape["elem"], scales=scales.view(torch.float32), **planes)
    src = torch.tensor([3, 0, 22, 9, -1, P, 4, 4], dtype=torch.int32, device="cuda")
    dst = torch.tensor([7, 21, 1, P + 5, 2, 5, 11, -7], dtype=torch.int32, device="cuda")
    every = [kv, scales] + [t.view(torch.uint8) for t in planes.values()]
    want = [t.clone() for t in every]
    for w in want:
        for a, b in ((3, 7), (0, 21), (22, 1), (4, 11)):  # the other pairs are skipped
            w[:, b] = w[:, a]
    c.copy_pages(src, dst)
    for got, w in zip(every, want):
        assert torch.equal(got, w)
    c.copy_pages(src[:0], dst[:0])
    c.copy_pages(src[:1], src[:1])  # onto itself
    for got, w in zip(every, want):
        assert torch.equal(got, w)


# ------------------------------------------------------------------- moves

class Moved:
    """Keys and values of sequences, lists of kept tokens, and fresh pages."""

    def __init__(self, kv_lens, kept, heads=2, dim=64, page=16, act=BF16, fp8=False, layers=2,
                 bounds=False, seed=0, firsts=None, pow2=True):
        need_gpu()
        self.g = g = torch.Generator().manual_seed(seed)
        self.H, self.D, self.T, self.act, self.fp8, self.L = heads, dim, page, act, fp8, layers
        before = [-(-k // page) for k in kv_lens]
        self.tokens = [torch.randperm(k, generator=g)[:n].sort().values
                       for k, n in zip(kv_lens, kept)]
        after = [-(-n // page) for n in kept]
        self.P = sum(before) + sum(after) + 3
        perm = torch.randperm(self.P, generator=g).int()
        n = len(kv_lens)
        self.src = torch.full((n, max(before) + 1), -1, dtype=torch.int32)
        self.dst = torch.full((n, max(after + [1]) + 2), -1, dtype=torch.int32)
        at = 0
        for table, counts in ((self.src, before), (self.dst, after)):
            for s, c in enumerate(counts):
                table[s, :c] = perm[at:at + c]
                at += c
        x = torch.randn((layers, self.P, 2, page, heads, dim), generator=g) * (60 if fp8 else 1)
        self.cache = x.clamp(-448, 448).to(FP8 if fp8 else act)
        self.scales = None
        if fp8:
            e = torch.rand((layers, self.P, 2, heads), generator=g) * 3 - 8
            self.scales = torch.exp2(e.round() if pow2 else e).float()
        self.firsts = firsts
        self.max_kv, self.kept = max(kv_lens), kept
        self.d_cache = self.cache.cuda()
        self.d_scales = None if self.scales is None else self.scales.cuda()
        self.d_bounds = self.d_bscales = None
        if bounds:
            self.d_bounds = torch.full((layers, self.P, 2, heads, dim), 77, dtype=torch.int8,
                                       device="cuda")
            self.d_bscales = torch.full((layers, self.P, heads), math.nan, device="cuda")
        self.handle = api.Cache(self.d_cache, self.P, layers, page, heads, dim, 1 if fp8 else 2,
                                head_scales=self.d_scales, bounds=self.d_bounds,
                                bound_scales=self.d_bscales)

    def move(self, **kw):
        ints = lambda x: torch.as_tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        start = [sum(len(t) for t in self.tokens[:i]) for i in range(len(self.tokens) + 1)]
        kw.setdefault("dtype", self.act)
        kw.setdefault("max_kv", self.max_kv)
        self.handle.move_tokens(self.src.cuda(), self.dst.cuda(), ints(torch.cat(self.tokens)),
                                ints(start), max_tokens=max(self.kept), dst_first=None if
                                self.firsts is None else ints(self.firsts), **kw)
        torch.cuda.synchronize()

    def check(self, rope, interleaved, layers):
        got = self.d_cache.cpu()
        raw = got.view(torch.uint8).clone()
        was = self.cache.view(torch.uint8)
        scales = None if self.scales is None else self.d_scales.cpu()
        for layer in range(self.L):
            if layer not in layers:
                continue
            for s, tokens in enumerate(self.tokens):
                if not len(tokens):
                    continue
                T = self.T
                pages = self.src[s, tokens // T].long()
                old = self.cache[layer, pages, :, tokens % T].double()  # [n, 2, H, D]
                if self.fp8:
                    old = old * self.scales[layer, pages].double()[..., None]
                first = 0 if self.firsts is None else self.firsts[s]
                by = torch.arange(len(tokens)) + first - tokens
                key, mag = old[:, 0], old[:, 0].abs()
                if rope is not None:
                    turned, m = turn64(key, rope, by, interleaved)
                    still = (by == 0)[:, None, None]
                    key, mag = torch.where(still, key, turned), torch.where(still, mag, m)
                for b in range(-(-len(tokens) // T)):
                    cut, page = slice(b * T, (b + 1) * T), int(self.dst[s, b])
                    n = len(tokens[cut])
                    for which, want, m in ((0, key[cut], mag[cut]), (1, old[cut, 1], None)):
                        new = got[layer, page, which, :n].double()
                        if not self.fp8:
                            if which == 1:
                                assert torch.equal(new, want)
                            else:
                                bound = ULP[self.act] * want.abs() + 2.0 ** -22 * m + TINY[self.act]
                                bound[(by[cut] == 0)] = 0
                                assert ((new - want).abs() <= bound).all()
                        else:
                            for h in range(self.H):
                                sc = float(scales[layer, page, which, h])
                                need = power(float(want[:, h].abs().max()))
                                edge = abs(float(want[:, h].abs().max()) / need / 448 * 2 - 1)
                                assert sc == need or (edge < 1e-5 and sc in (need / 2, need * 2))
                                w = want[:, h]
                                bound = torch.maximum(2.0 ** -4 * w.abs(),
                                                      torch.tensor(2.0 ** -10 * sc).double())
                                if m is not None:
                                    bound = bound + 2.0 ** -22 * m[:, h]
                                assert ((new[:, h] * sc - w).abs() <= bound).all()
                        raw[layer, page, which, :n] = was[layer, page, which, :n]
                    if self.d_bounds is not None:
                        self.check_bounds(layer, page, n, got, scales)
        assert torch.equal(raw, was)  # nothing else is written

    def check_bounds(self, layer, page, n, got, scales):
        for h in range(self.H):
            k = got[layer, page, 0, :n, h].double()
            if self.fp8:
                k = k * float(scales[layer, page, 0, h])
            unit = power(float(k.abs().max()), 127.0)
            assert float(self.d_bscales[layer, page, h]) == unit
            b = self.d_bounds[layer, page, :, h].cpu().double()
            assert torch.equal(b[0], (k.amin(0) / unit).floor())
            assert torch.equal(b[1], (k.amax(0) / unit).ceil())


MOVES = [
    dict(kv_lens=[200], kept=[120]),
    dict(kv_lens=[40, 1, 77, 3], kept=[17, 1, 77, 2], heads=1, dim=8),
    dict(kv_lens=[90, 33], kept=[50, 16], heads=3, dim=80, page=5),
    dict(kv_lens=[130, 64], kept=[100, 33], heads=4, dim=128, page=32),
    dict(kv_lens=[61, 50], kept=[40, 20], heads=2, dim=136, page=16),
    dict(kv_lens=[150], kept=[99], heads=1, dim=256, page=48),
    dict(kv_lens=[30, 20], kept=[9, 11], heads=2, dim=96, page=1),
]


@pytest.mark.parametrize("kind", ["bf16", "f16", "fp8"])
@pytest.mark.parametrize("shape", MOVES, ids=str)
def test_moved_tokens(shape, kind):
    st = Moved(act=F16 if kind == "f16" else BF16, fp8=kind == "fp8", bounds=True, pow2=False,
               **shape)
    rope = angles(st.max_kv, st.D)
    st.move(rope=rope.cuda())
    st.check(rope, False, range(st.L))


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("dim,interleaved", [(24, False), (32, False), (20, True), (72, False)])
def test_ways_to_turn(kind, dim, interleaved):
    st = Moved([70, 41], [30, 41], heads=2, dim=72, fp8=kind == "fp8", firsts=[25, 0], layers=3)
    rope = angles(80, dim)
    st.move(rope=rope.cuda(), interleaved=interleaved, layer_begin=1, layer_count=2)
    st.check(rope, interleaved, (1, 2))


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_tokens_that_move_on_and_those_without_angles(kind):
    # to later positions (behind a prefix that stays), and keys that stay as they are
    st = Moved([60, 60], [20, 31], fp8=kind == "fp8", firsts=[100, 7])
    rope = angles(200, 64)
    st.move(rope=rope.cuda())
    st.check(rope, False, range(2))
    st = Moved([60, 60], [20, 31], fp8=kind == "fp8", firsts=[100, 7], seed=4)
    st.move()
    st.check(None, False, range(2))


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_out_of_bounds_tokens_become_zeros(kind):
    st = Moved([100], [40], fp8=kind == "fp8")
    st.tokens[0][3], st.tokens[0][17], st.tokens[0][30] = -4, 100, 2 ** 30
    st.src[0, 2] = st.P
    rope = angles(20, 64)  # tokens that move by 20 or more too
    st.dst[0, 1] = -2      # and a block that goes nowhere
    tokens = st.tokens[0].clone()
    st.move(rope=rope.cuda())
    zero = [(i, int(t)) for i, t in enumerate(tokens)
            if not 0 <= t < 100 or t // 16 == 2 or abs(i - int(t)) >= 20]
    got = st.d_cache.cpu().float()
    for i in range(40):
        if i // 16 == 1:
            continue
        row = got[:, int(st.dst[0, i // 16]), :, i % 16]
        assert bool((row == 0).all()) == (i in [z[0] for z in zero]), i


def test_moved_values_that_are_not_finite():
    st = Moved([40], [20], heads=1, dim=64)
    page, slot = int(st.src[0, int(st.tokens[0][5]) // 16]), int(st.tokens[0][5]) % 16
    st.d_cache[0, page, 1, slot, 0, 3] = math.inf
    st.d_cache[0, page, 1, slot, 0, 9] = math.nan
    st.d_cache[0, page, 0, slot, 0, 63] = -math.inf
    st.move()
    got = st.d_cache[0, int(st.dst[0, 0])]
    assert got[1, 5, 0, 3] == math.inf and torch.isnan(got[1, 5, 0, 9])
    assert got[0, 5, 0, 63] == -math.inf


# ---------------------------------------------------------- latents: moves

@pytest.mark.parametrize("kind", ["bf16", "f16", "fp8"])
@pytest.mark.parametrize("shape", [
    dict(latent=128, turn=32), dict(latent=512, turn=64), dict(latent=384, turn=48, page=5),
    dict(latent=16, turn=16, page=1), dict(latent=256, turn=64, page=64),
], ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
def test_moved_latents(shape, kind, interleaved):
    need_gpu()
    kv, kept = [100, 37, 5], [70, 37, 2]
    act = F16 if kind == "f16" else BF16
    st = Latents(kv, [1, 1, 1], act=act, fp8=kind == "fp8", spare=80 if shape.get("page") == 5
                 else 160 if shape.get("page") == 1 else 20, pow2=False, **shape)
    T, C, R = st.T, st.C, st.R
    used = set(st.table[st.table >= 0].tolist())
    free = [p for p in range(st.P) if p not in used]
    dst = torch.full((3, max(-(-n // T) for n in kept) + 1), -1, dtype=torch.int32)
    for s, n in enumerate(kept):
        for b in range(-(-n // T)):
            dst[s, b] = free.pop()
    tokens = [torch.randperm(k, generator=st.g)[:n].sort().values for k, n in zip(kv, kept)]
    rope, first = angles(130, R), [0, 0, 30]
    ints = lambda x: torch.as_tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    st.handle.move_tokens(st.table.cuda(), dst.cuda(), ints(torch.cat(tokens)),
                          ints([0, 70, 107, 109]), max_tokens=70, max_kv=100,
                          dst_first=ints(first), rope=rope.cuda(), interleaved=interleaved,
                          dtype=act)
    got = st.d_cache.cpu()
    scales = st.d_scales.cpu() if st.fp8 else None
    raw, was = got.view(torch.uint8).clone(), st.cache.view(torch.uint8)
    for layer in range(2):
        st.layer = layer
        for s in range(3):
            old = st.stored(s)[tokens[s]]
            by = torch.arange(len(tokens[s])) + first[s] - tokens[s]
            key, mag = turn64(old[:, C:], rope, by, interleaved)
            for b in range(-(-len(tokens[s]) // T)):
                cut, page = slice(b * T, (b + 1) * T), int(dst[s, b])
                n = len(tokens[s][cut])
                for w, cols, want, m in ((0, slice(0, C), old[cut, :C], None),
                                         (1, slice(C, C + R), key[cut], mag[cut])):
                    new = got[layer, page, :n, cols].double()
                    if st.fp8:
                        sc, need = float(scales[layer, page, w]), power(float(want.abs().max()))
                        edge = abs(float(want.abs().max()) / need / 448 * 2 - 1)
                        assert sc == need or (edge < 1e-5 and sc in (need / 2, need * 2))
                        bound = torch.maximum(2.0 ** -4 * want.abs(),
                                              torch.tensor(2.0 ** -10 * sc).double())
                        new = new * sc
                    else:
                        bound = (ULP[act] * want.abs() + TINY[act]) * w
                    if m is not None:
                        bound = bound + 2.0 ** -22 * m
                    assert ((new - want).abs() <= bound).all()
                raw[layer, page, :n] = was[layer, page, :n]
    assert torch.equal(raw, was)


# --------------------------------------------------------- latents: append

@pytest.mark.parametrize("kind", ["bf16", "f16", "fp8"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", [
    dict(kv_lens=[1, 16, 17, 40], rows=[1, 1, 1, 1]),
    dict(kv_lens=[40, 100, 3], rows=[33, 1, 3], heads=16, latent=512, turn=64),
    dict(kv_lens=[50, 9, 0], rows=[20, 9, 2], heads=5, latent=384, turn=48, page=5),
    dict(kv_lens=[2, 300], rows=[4, 200], heads=1, latent=16, turn=16, page=64),
    dict(kv_lens=[9, 8], rows=[3, 0], heads=70, latent=256, turn=64, page=1),
], ids=str)
def test_appended_latents(shape, kind, interleaved):
    need_gpu()
    act = F16 if kind == "f16" else BF16
    st = Latents(act=act, fp8=kind == "fp8", pow2=True, **shape)
    C, R, T, H = st.C, st.R, st.T, st.H
    rope = angles(max(st.kv_lens), R)
    both = st.rand(st.n_rows, 1, C + R)
    wide = st.rand(st.n_rows, H, 16 + R)
    d_both, d_wide = both.cuda(), wide.cuda()
    q_out = torch.full((st.n_rows, H, R), 9.0, dtype=act, device="cuda")
    st.handle.append_latent(st.layer, st.batch, d_both[..., :C], d_both[..., C:], rope=rope.cuda(),
                            q=d_wide[..., 16:], q_out=q_out, interleaved=interleaved)
    got, out = st.d_cache.cpu(), q_out.cpu().double()
    raw, was = got.view(torch.uint8).clone(), st.cache.view(torch.uint8)
    scales = st.d_scales.cpu() if st.fp8 else None
    for s, n in enumerate(st.rows):
        start = st.kv_lens[s] - n
        for r in range(max(0, -start)):  # rows before the first position: left alone
            assert (out[st.starts[s] + r] == 9.0).all()
        rows = torch.arange(max(0, -start), n) + st.starts[s]
        pos = torch.arange(max(start, 0), st.kv_lens[s])
        if not len(pos):
            continue
        want, mag = turn64(wide[rows][..., 16:], rope, pos, interleaved)
        assert ((out[rows] - want).abs() <=
                ULP[act] * want.abs() + TINY[act] + 2.0 ** -22 * mag).all()
        key, mag = turn64(both[rows, 0, C:], rope, pos, interleaved)
        new = torch.cat([both[rows, 0, :C].double(), key], 1)
        mag = torch.cat([torch.zeros_like(new[:, :C]), mag], 1)
        for p in sorted({int(x) // T for x in pos}):
            page, here = int(st.table[s, p]), pos // T == p
            i0, i1 = max(max(start, 0) - p * T, 0), min(st.kv_lens[s] - p * T, T)
            for w, cols in ((0, slice(0, C)), (1, slice(C, C + R))):
                want, m = new[here][:, cols], mag[here][:, cols]
                stored = got[st.layer, page, i0:i1, cols].double()
                if not st.fp8:
                    bound = (ULP[act] * want.abs() + TINY[act]) * w + 2.0 ** -22 * m
                    assert ((stored - want).abs() <= bound).all()
                    continue
                s0, s1 = float(st.scales[st.layer, page, w]), float(scales[st.layer, page, w])
                need = power(float(want.abs().max()))
                edge = abs(float(want.abs().max()) / need / 448 * 2 - 1) < 1e-5
                need = max(need, s0) if i0 else need
                assert s1 == need or (edge and s1 in (need / 2, need * 2))
                bound = torch.maximum(2.0 ** -4 * want.abs(),
                                      torch.tensor(2.0 ** -10 * s1).double()) + 2.0 ** -22 * m
                assert ((stored * s1 - want).abs() <= bound).all()
                old = st.cache[st.layer, page, :i0, cols].double() * s0
                again = got[st.layer, page, :i0, cols].double() * s1
                bound = torch.where(old.abs() < 2.0 ** -6 * s1, 2.0 ** -10 * s1, 0.0) * (s1 != s0)
                assert ((again - old).abs() <= bound).all()
                raw[st.layer, page, :i0, cols] = was[st.layer, page, :i0, cols]
            raw[st.layer, page, i0:i1] = was[st.layer, page, i0:i1]
    assert torch.equal(raw, was)


def test_appended_without_angles_and_queries_in_place():
    need_gpu()
    st = Latents(kv_lens=[20, 5], rows=[3, 5], heads=4, latent=128, turn=32)
    both, q = st.rand(8, 1, 160), st.rand(8, 4, 32).cuda()
    d = both.cuda()
    st.handle.append_latent(st.layer, st.batch, d[..., :128], d[..., 128:])
    got = st.d_cache.cpu()
    for s, r, p in ((0, 0, 17), (0, 2, 19), (1, 3, 4), (1, 7, 4)):
        if s == 1 and r == 3:
            p = 0
        assert torch.equal(got[st.layer, int(st.table[s, p // 16]), p % 16], both[r, 0])
    rope, q0 = angles(20, 32), q.cpu()
    st.handle.append_latent(st.layer, st.batch, d[..., :128], d[..., 128:], rope=rope.cuda(), q=q,
                            q_out=q)
    pos = torch.tensor([17, 18, 19, 0, 1, 2, 3, 4])
    want, mag = turn64(q0, rope, pos, False)
    assert ((q.cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -22 * mag).all()


@pytest.mark.parametrize("turn", [16, 32, 48, 64])
@pytest.mark.parametrize("heads", [11, 24, 128])
def test_queries_of_many_heads_in_place(turn, heads):
    # heads whose pieces are no whole part of a wave's lanes
    need_gpu()
    st = Latents(kv_lens=[20, 5, 70], rows=[3, 5, 1], heads=heads, latent=128, turn=turn)
    both, q = st.rand(9, 1, 128 + turn).cuda(), st.rand(9, heads, turn).cuda()
    rope, q0 = angles(70, turn), q.cpu()
    st.handle.append_latent(st.layer, st.batch, both[..., :128], both[..., 128:], rope=rope.cuda(),
                            q=q, q_out=q)
    want, mag = turn64(q0, rope, torch.tensor([17, 18, 19, 0, 1, 2, 3, 4, 69]), False)
    assert ((q.cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -22 * mag).all()
