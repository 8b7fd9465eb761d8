"""Latents, copied pages and moved tokens as a server calls them: refused calls,
captured ones, other streams, padded steps, a tier, and a run of all of them."""
import ctypes as C
import math

import pytest
import torch

from gpu_common import need_gpu
from latent_common import BF16, F16, Latents, check_attention
from paper_2609_33762_amd import _native as N
from paper_2609_33762_amd import api
from test_zz_pages_moves import Moved, angles, turn64

pytestmark = pytest.mark.gpu

WEIGHTS = {False: 2.0 ** -8, True: 2.0 ** -11}  # rounding of the weights: bf16 latents, fp8 ones
SCALE = 0.07


def ints(x):
    return torch.as_tensor(x, dtype=torch.int32, device="cuda")


def attend(st, q, batch=None, **kw):
    out = torch.full((q.shape[0], st.H, st.C), math.nan, dtype=st.act, device="cuda")
    lse = torch.full((q.shape[0], st.H), math.nan, device="cuda")
    st.handle.attend_latent(st.layer, batch or st.batch, q, out, scale=SCALE, lse=lse, **kw)
    return out, lse


# ------------------------------------------------------------------ refusals

def test_refusals():
    need_gpu()
    st = Latents([20, 7], [1, 2], heads=4, latent=128, turn=32)
    c, b, act = st.handle, st.batch, st.act
    q, out = st.rand(3, 4, 160).cuda(), torch.empty((3, 4, 128), dtype=act, device="cuda")
    lat, key = st.rand(3, 1, 128).cuda(), st.rand(3, 1, 32).cuda()
    rope = angles(20, 32).cuda()

    def refused(f, *a, **kw):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            f(*a, **kw)

    for layer in (-1, 2):
        refused(c.attend_latent, layer, b, q, out, scale=1.0)
        refused(c.append_latent, layer, b, lat, key)
    for scale in (0.0, -1.0, math.nan, math.inf):
        refused(c.attend_latent, 0, b, q, out, scale=scale)
    refused(c.attend_latent, 0, b, q[..., :128], out, scale=1.0)
    refused(c.attend_latent, 0, b, q, q, scale=1.0)
    refused(c.attend_latent, 0, b, q, out.to(F16), scale=1.0)
    refused(c.attend_latent, 0, b, q.float(), out.float(), scale=1.0)
    refused(c.attend_latent, 0, b, q[:2], out, scale=1.0)
    refused(c.attend_latent, 0, b, q.cpu(), out, scale=1.0)
    refused(c.attend_latent, 0, b, q, out, scale=1.0, lse=torch.empty((3, 4), device="cuda").half())
    refused(c.append_latent, 0, b, lat, key, rope=rope[:, :16].contiguous())
    refused(c.append_latent, 0, b, lat, key, rope=rope[:10])
    refused(c.append_latent, 0, b, lat, key, rope=rope.double())
    refused(c.append_latent, 0, b, lat, lat)
    refused(c.append_latent, 0, b, lat, key.to(F16))
    refused(c.append_latent, 0, b, lat, key, q=q[..., 128:])
    far = api.Batch(st.table[:, :1].contiguous().cuda(), ints([20, 7]), 20)
    refused(c.attend_latent, 0, far, q, out, scale=1.0)
    # sizes that the kernels do not have
    for latent, turn in ((520, 64), (528, 64), (512, 80), (24, 32), (32, 24)):
        kv = torch.zeros((1, 4, 16, latent + turn), dtype=act, device="cuda")
        other = api.LatentCache(kv, 4, 1, 16, latent, turn, 2)
        t = api.Batch(ints([[0]]), ints([3]), 16)
        refused(other.attend_latent, 0, t, torch.zeros((1, 4, latent + turn), dtype=act,
                device="cuda"), torch.zeros((1, 4, latent), dtype=act, device="cuda"), scale=1.0)
    no_scales = api.LatentCache(torch.zeros((1, 4, 16, 160), dtype=torch.uint8, device="cuda"),
                                4, 1, 16, 128, 32, 1)
    refused(no_scales.attend_latent, 0, b, q, out, scale=1.0)
    # moves and copies
    src, dst = st.table.cuda(), ints([[0, 1], [2, 3]])
    kw = dict(max_tokens=20, max_kv=20)
    ok = (src, dst, ints([1, 2, 3]), ints([0, 2, 3]))
    refused(c.move_tokens, src, dst[:1], *ok[2:], **kw)
    refused(c.move_tokens, src, dst, ok[2], ints([0, 3]), **kw)
    refused(c.move_tokens, src.long(), *ok[1:], **kw)
    refused(c.move_tokens, src.cpu(), *ok[1:], **kw)
    refused(c.move_tokens, *ok, max_tokens=33, max_kv=20)
    refused(c.move_tokens, *ok, max_tokens=2, max_kv=16 * src.shape[1] + 1)
    refused(c.move_tokens, *ok, max_tokens=-1, max_kv=20)
    refused(c.move_tokens, *ok, rope=rope[:, :16].contiguous(), **kw)
    refused(c.move_tokens, *ok, dst_first=ints([0]), **kw)
    refused(c.move_tokens, *ok, layer_begin=1, layer_count=2, **kw)
    refused(c.move_tokens, *ok, layer_begin=-1, layer_count=1, **kw)
    refused(c.move_tokens, *ok, dtype=torch.float32, **kw)
    refused(c.copy_pages, ints([0, 1]), ints([2]))
    with pytest.raises(AttributeError):  # host lists, as in every call of device arrays
        c.copy_pages([0], [1])
    refused(c.copy_pages, ints([0]).cpu(), ints([1]))
    # one scale for all heads of a block
    two = api.Cache(torch.zeros((1, 4, 2, 16, 2, 64), dtype=torch.uint8, device="cuda"), 4, 1, 16,
                    2, 64, 1, scales=torch.ones((1, 4, 2), device="cuda"))
    refused(two.move_tokens, ints([[0]]), ints([[1]]), ints([0]), ints([0, 1]), 16, 16)
    torch.cuda.synchronize()
    raw = st.d_cache.cpu().view(torch.uint8)
    assert torch.equal(raw, st.cache.view(torch.uint8))  # nothing was written


def test_a_workspace_that_is_too_small_is_refused():
    need_gpu()
    st = Latents([900], [1], heads=4, latent=128, turn=32)
    q, out = st.rand(1, 4, 160).cuda(), torch.zeros((1, 4, 128), dtype=BF16, device="cuda")
    lib, ref = N.load(), C.byref
    a = N.LatentAttention(*(N.Rows(t.data_ptr(), t.stride(0), t.stride(1)) for t in (q, out)))
    a.latent_dim, a.rope_dim, a.q_heads, a.dtype, a.scale = 128, 32, 4, N.EA_BF16, SCALE
    need = lib.ea_attend_latent_workspace(st.handle.handle, st.batch.ref, ref(a))
    assert need > 0
    ws = torch.full((need + 16,), 0xff, dtype=torch.uint8, device="cuda")
    for ptr, n in ((None, need), (ws.data_ptr(), need - 1), (ws.data_ptr() + 4, need)):
        assert lib.ea_attend_latent(st.handle.handle, st.layer, st.batch.ref, ref(a), ptr, n,
                                    api.current_stream()) == -1
    # a workspace holds whatever it held
    assert lib.ea_attend_latent(st.handle.handle, st.layer, st.batch.ref, ref(a), ws.data_ptr(),
                                need, api.current_stream()) == 0
    torch.cuda.synchronize()
    assert (ws[need:] == 0xff).all()
    lse = torch.empty((1, 4), device="cuda")
    st.handle.attend_latent(st.layer, st.batch, q, out2 := torch.empty_like(out), scale=SCALE,
                            lse=lse)
    assert torch.equal(out, out2)
    check_attention(st, q.cpu(), out2, lse, SCALE, WEIGHTS[False])


# ------------------------------------------------------------ empty calls

def test_calls_of_nothing():
    st = Latents([5], [1])
    none = api.Batch(st.table[:0].cuda(), ints([]), 0)
    empty = torch.empty((0, 2, 160), dtype=BF16, device="cuda")
    st.handle.attend_latent(0, none, empty, empty[..., :128], scale=1.0)
    st.handle.append_latent(0, none, empty[:, :1, :128], empty[:, :1, 128:])
    st.handle.copy_pages(ints([]), ints([]))
    st.handle.move_tokens(st.table.cuda(), ints([[1]]), ints([]), ints([0, 0]), 0, 0)
    torch.cuda.synchronize()
    assert torch.equal(st.d_cache.cpu().view(torch.uint8), st.cache.view(torch.uint8))


# --------------------------------------------------- streams and captures

@pytest.mark.parametrize("fp8", [False, True])
def test_captured_calls_beside_eager_ones(fp8):
    # a graph that appends and attends, and another one on another stream; replays
    # with eager work of both forms between them
    need_gpu()
    st = Latents([700, 45, 3000], [1, 1, 1], heads=8, latent=512, turn=64, fp8=fp8, pow2=True)
    rope = angles(3000, 64).cuda()
    both, q = st.rand(3, 1, 576).cuda(), st.rand(3, 8, 576).cuda()
    chunk = Latents([400, 90], [300, 60], heads=8, latent=512, turn=64, fp8=fp8, seed=2)
    cq = chunk.rand(360, 8, 576).cuda()

    def step(out, lse):
        st.handle.append_latent(st.layer, st.batch, both[..., :512], both[..., 512:], rope=rope)
        st.handle.attend_latent(st.layer, st.batch, q, out, scale=SCALE, lse=lse)

    def new():
        return (torch.full((3, 8, 512), math.nan, dtype=BF16, device="cuda"),
                torch.full((3, 8), math.nan, device="cuda"))

    want, (out, lse) = new(), new()
    step(*want)
    big = attend(chunk, cq)
    torch.cuda.synchronize()
    state = [t.clone() for t in (st.d_cache, st.d_scales) if t is not None]
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    ga, gb = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(ga, stream=a):
        step(out, lse)
    cout, clse = torch.empty_like(big[0]), torch.empty_like(big[1])
    with torch.cuda.graph(gb, stream=b):
        chunk.handle.attend_latent(chunk.layer, chunk.batch, cq, cout, scale=SCALE, lse=clse)
    for _ in range(4):
        for t in (out, lse, cout, clse):
            t.fill_(math.nan)
        torch.cuda.synchronize()
        with torch.cuda.stream(a):
            ga.replay()
        with torch.cuda.stream(b):  # at the same time
            gb.replay()
        again = attend(chunk, cq)
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        assert torch.equal(cout, big[0]) and torch.equal(clse, big[1])
        assert torch.equal(again[0], big[0])
        eager = new()
        step(*eager)
        torch.cuda.synchronize()
        assert torch.equal(eager[0], want[0]) and torch.equal(eager[1], want[1])
        for t, was in zip((st.d_cache, st.d_scales), state):
            assert torch.equal(t.view(torch.uint8), was.view(torch.uint8))


def test_captured_moves_and_copies():
    st = Moved([90, 33], [50, 16], fp8=True)
    rope = angles(90, st.D).cuda()
    src, dst = ints([int(st.src[0, 0])]), ints([st.P - 1])
    free = [p for p in range(st.P) if p not in st.src and p not in st.dst]
    dst = ints([free[0]])
    args = (st.src.cuda(), st.dst.cuda(), ints(torch.cat(st.tokens)), ints([0, 50, 66]))

    def edit():
        st.handle.move_tokens(*args, max_tokens=50, max_kv=90, rope=rope)
        st.handle.copy_pages(src, dst)

    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        edit()
    first = [st.d_cache.clone(), st.d_scales.clone()]
    edit()
    want = [st.d_cache.clone(), st.d_scales.clone()]
    for _ in range(3):
        for t, was in zip((st.d_cache, st.d_scales), first):
            t.copy_(was)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for t, w in zip((st.d_cache, st.d_scales), want):
            assert torch.equal(t.view(torch.uint8), w.view(torch.uint8))


def test_calls_on_a_given_stream():
    st = Latents([1000, 3], [1, 1], heads=4)
    q = st.rand(2, 4, 160).cuda()
    want = attend(st, q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = attend(st, q, stream=s)
    s.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("rows", [[1, 1], [0, 3], [40, 0], [7, 30]])
def test_a_step_padded_to_its_largest_form(kind, rows):
    # n_rows, max_rows and max_kv are bounds; rows of nobody stay as they are
    need_gpu()
    st = Latents([60, 200], rows, heads=5, fp8=kind == "fp8", pow2=True)
    n = 96
    batch = api.Batch(st.table.cuda(), ints(st.kv_lens), 208, ints(st.starts), n, 48)
    q = st.rand(n, 5, 160)
    out, lse = attend(st, q.cuda(), batch)
    there = st.n_rows
    assert torch.isnan(out[there:]).all() and torch.isnan(lse[there:]).all()
    check_attention(st, q[:there], out[:there], lse[:there], SCALE, WEIGHTS[kind == "fp8"])
    both, turn = st.rand(n, 1, 160).cuda(), st.rand(n, 5, 32).cuda()
    q_out = torch.full_like(turn, 9.0)
    st.handle.append_latent(st.layer, batch, both[..., :128], both[..., 128:],
                            rope=angles(208, 32).cuda(), q=turn, q_out=q_out)
    assert (q_out[there:] == 9.0).all() and (q_out[:there] != 9.0).any(-1).all()


def test_more_rows_than_the_host_was_told_are_not_reached():
    # row_start beyond n_rows: the rest has no memory behind it
    need_gpu()
    st = Latents([60, 60], [4, 4], heads=3)
    q = st.rand(8, 3, 160)
    full = attend(st, q.cuda())
    short = api.Batch(st.table.cuda(), ints(st.kv_lens), 60, ints(st.starts), 6, 4)
    out = torch.full((8, 3, 128), 7.0, dtype=BF16, device="cuda")
    st.handle.attend_latent(st.layer, short, q.cuda()[:6], out[:6], scale=SCALE)
    assert torch.equal(out[:4], full[0][:4]) and (out[6:] == 7.0).all()


# ----------------------------------------------------- long caches

def test_offsets_beyond_32_bits():
    # a plane of more than 4 GiB: the last pages hold the sequence
    need_gpu()
    latent, turn, page = 512, 64, 64
    pages = 65536  # 4.8 GB of bf16 rows
    kv = torch.zeros((1, pages, page, 576), dtype=BF16, device="cuda")
    g = torch.Generator().manual_seed(5)
    ids = [pages - 1, 3, pages - 700, pages - 2, 60000]
    x = torch.randn((5, page, 576), generator=g).to(BF16)
    kv[0, torch.tensor(ids, device="cuda")] = x.cuda()
    cache = api.LatentCache(kv, pages, 1, page, latent, turn, 2)
    batch = api.Batch(ints([ids]), ints([300]), 320)
    q = torch.randn((1, 16, 576), generator=g).to(BF16)
    out, lse = torch.empty((1, 16, 512), dtype=BF16, device="cuda"), torch.empty((1, 16), device="cuda")
    cache.attend_latent(0, batch, q.cuda(), out, scale=SCALE, lse=lse)
    st = object.__new__(Latents)
    st.kv_lens, st.rows, st.starts, st.n_rows, st.H, st.C, st.R = [300], [1], [0, 1], 1, 16, 512, 64
    st.act, st.stored = BF16, lambda s: x.reshape(-1, 576)[:300].double()
    check_attention(st, q, out, lse, SCALE, WEIGHTS[False])
    # copied there, and moved there
    cache.copy_pages(ints([pages - 1, 3]), ints([pages - 5, pages - 6]))
    assert torch.equal(kv[0, pages - 5].cpu(), x[0]) and torch.equal(kv[0, pages - 6].cpu(), x[1])
    cache.move_tokens(ints([ids]), ints([[pages - 9, pages - 8]]), ints(range(100, 200)),
                      ints([0, 100]), 100, 320)
    want = x.reshape(-1, 576)[100:200]
    got = torch.cat([kv[0, pages - 9], kv[0, pages - 8, :36]]).cpu()
    assert torch.equal(got, want)
    # appended there
    new = torch.randn((1, 1, 576), generator=g).to(BF16)
    cache.append_latent(0, batch, new.cuda()[..., :512], new.cuda()[..., 512:])
    assert torch.equal(kv[0, 60000, 299 - 256].cpu(), new[0, 0])


# ----------------------------------------------------- as they are used

@pytest.mark.parametrize("fp8", [False, True])
def test_a_context_is_written_forked_edited_and_goes_on(fp8):
    """A prompt in two chunks, a fork of its last block, a step of both contexts,
    an edit that drops tokens, and a step of the edited context: each attention
    against 64 bits over what the cache then holds, and the cache against what
    was appended."""
    need_gpu()
    C_, R, T, H = 128, 32, 16, 6
    act, scale = BF16, SCALE
    P = 40
    rope = angles(128, R)
    d_rope = rope.cuda()
    kv = torch.zeros((1, P, T, C_ + R), dtype=torch.float8_e4m3fn if fp8 else act, device="cuda")
    scales = torch.ones((1, P, 2), device="cuda") if fp8 else None
    cache = api.LatentCache(kv, P, 1, T, C_, R, 1 if fp8 else 2, scales=scales)
    g = torch.Generator().manual_seed(8)

    def view(tables, lens, rows):
        st = object.__new__(Latents)
        st.kv_lens, st.rows, st.layer, st.H, st.C, st.R, st.T = lens, rows, 0, H, C_, R, T
        st.act, st.fp8, st.table = act, fp8, torch.tensor(tables, dtype=torch.int32)
        st.starts = [sum(rows[:i]) for i in range(len(rows) + 1)]
        st.n_rows = st.starts[-1]
        return st

    def step(tables, lens, rows):
        st = view(tables, lens, rows)
        batch = api.Batch(st.table.cuda(), ints(lens), max(lens), ints(st.starts), st.n_rows,
                          max(rows))
        new = torch.randn((st.n_rows, 1, C_ + R), generator=g).to(act)
        q = torch.randn((st.n_rows, H, C_ + R), generator=g).to(act)
        d_new, d_q = new.cuda(), q.cuda()
        cache.append_latent(0, batch, d_new[..., :C_], d_new[..., C_:], rope=d_rope,
                            q=d_q[..., C_:], q_out=d_q[..., C_:])
        out = torch.full((st.n_rows, H, C_), math.nan, dtype=act, device="cuda")
        lse = torch.empty((st.n_rows, H), device="cuda")
        cache.attend_latent(0, batch, d_q, out, scale=scale, lse=lse)
        st.cache, st.scales = kv.cpu(), None if scales is None else scales.cpu()
        check_attention(st, d_q.cpu(), out, lse, scale, WEIGHTS[fp8])
        # what was appended is there: a rounding to the cache's type, and 16-bit
        # rows' one
        for s, n in enumerate(rows):
            pos = torch.arange(lens[s] - n, lens[s])
            x = new[st.starts[s]:st.starts[s + 1], 0].double()
            x[:, C_:] = turn64(x[:, C_:], rope, pos, False)[0]
            got = st.stored(s)[pos]
            for cols in (slice(0, C_), slice(C_, C_ + R)):
                top = float(st.stored(s)[:, cols].abs().max())
                # fp8: half a step of the value, or of the smallest subnormal of a
                # scale that is at most twice what the block's largest value needs
                bound = 2.0 ** -8 * x[:, cols].abs() + 2.0 ** -20 if not fp8 else \
                    2.0 ** -4 * x[:, cols].abs() + 2.0 ** -10 * top / 448 * 4
                # a later token's larger scale may round a value once more
                assert ((got[:, cols] - x[:, cols]).abs() <= bound * (2 if fp8 else 1)).all()
        return st

    step([[3, 9, 1, 0]], [30], [30])
    step([[3, 9, 1, 0]], [37], [7])
    cache.copy_pages(ints([1]), ints([22]))  # the fork writes its own last block
    before = view([[3, 9, 1]], [37], [1])
    before.cache, before.scales = kv.cpu(), None if scales is None else scales.cpu()
    fork = view([[3, 9, 22]], [37], [1])
    fork.cache, fork.scales = before.cache, before.scales
    assert torch.equal(before.stored(0), fork.stored(0))
    st = step([[3, 9, 1, 30], [3, 9, 22, 31]], [40, 45], [3, 8])
    # the fork drops positions 5 .. 19 and goes on
    kept = [t for t in range(45) if not 5 <= t < 20]
    old = st.stored(1)
    cache.move_tokens(ints([[3, 9, 22, 31]]), ints([[12, 13, -1, -1]]), ints(kept), ints([0, 30]),
                      max_tokens=30, max_kv=45, rope=d_rope)
    edited = view([[12, 13]], [30], [1])
    edited.cache, edited.scales = kv.cpu(), None if scales is None else scales.cpu()
    by = torch.arange(30) - torch.tensor(kept)
    x = old[kept]
    x[:, C_:] = turn64(x[:, C_:], rope, by, False)[0]
    off = (edited.stored(0) - x).abs()
    if fp8:
        assert (off <= 2.0 ** -4 * x.abs() + 2.0 ** -10 * x.abs().max() / 448 * 4).all()
    else:
        assert (off <= 2.0 ** -8 * x.abs() + 2.0 ** -20).all()
    step([[3, 9, 1, 30], [12, 13, 14, -1]], [41, 33], [1, 3])


def test_a_cache_of_latents_through_a_tier():
    # gathered to slots and scattered to other pages, as any cache
    st = Latents([64, 20], [1, 1], heads=2, fp8=True, spare=8)
    used = [int(p) for p in st.table.flatten() if p >= 0]
    free = [p for p in range(st.P) if p not in used][:len(used)]
    buf = torch.empty((len(used), st.handle.slot_bytes), dtype=torch.uint8, device="cuda")
    q = st.rand(2, 2, 160).cuda()
    want = attend(st, q)
    st.handle.gather(used, buf)
    st.handle.scatter(buf, free)
    where = dict(zip(used, free))
    table = torch.tensor([[where.get(int(p), -1) for p in row] for row in st.table],
                         dtype=torch.int32, device="cuda")
    moved = api.Batch(table, ints(st.kv_lens), 64, ints(st.starts), 2, 1)
    got = attend(st, q, moved)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
