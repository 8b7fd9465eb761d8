"""Moved, appended and attended tokens on the GPU where a block, a batch or its
memory is out of the ordinary."""
import ctypes as C
import math

import pytest
import torch

from gpu_common import need_gpu
from latent_common import BF16, F16, FP8, Latents, check_attention
from paper_2609_33762_amd import _native as N
from paper_2609_33762_amd import api
from test_gpu_cache_ops import Setup
from test_zz_pages_moves import Moved, angles, turn64

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.as_tensor(x, dtype=torch.int32, device="cuda")


# ------------------------------------------------ fp8 blocks of zeros, moved

def zeros_and_few(where):
    """Codes of blocks 0 and 1 (zeros), 2 (zeros but where `where` says so), and
    scales that hold values up to 448 * 2^20, or, of block 2, the least ones."""
    scales = torch.tensor([4.0, 2.0 ** 20, 2.0 ** -126])
    codes = torch.zeros((3, *where.shape))
    codes[2] = where * torch.tensor([1.0, -448.0, 0.5, 2.0 ** -9]).repeat(
        -(-where.numel() // 4))[:where.numel()].view(where.shape)
    codes[0].view(-1)[::3] = -0.0
    return codes.to(FP8), scales


@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("page", [16, 48])
@pytest.mark.parametrize("dim,pairs", [(64, 64), (128, 128), (256, 256), (72, 72), (64, 20)])
def test_moved_zeros_stay_zeros(dim, pairs, page, turned):
    # a factor from an old block's scale to a new one's may pass 32 bits where all
    # codes are zeros; tokens of such blocks alone, and beside very small ones
    need_gpu()
    heads = 2
    where = (torch.arange(page) % 2 == 0)[:, None, None] * torch.ones(heads, dim)
    codes, scales = zeros_and_few(where)
    kv = torch.zeros((1, 8, 2, page, heads, dim), dtype=FP8)
    kv[0, :3] = codes[:, None].expand(3, 2, page, heads, dim)
    plane = torch.ones((1, 8, 2, heads))
    plane[0, :3] = scales[:, None, None]
    d_kv, d_plane = kv.cuda(), plane.cuda()
    bounds = torch.full((1, 8, 2, heads, dim), 77, dtype=torch.int8, device="cuda")
    unit = torch.full((1, 8, heads), 7.0, device="cuda")
    cache = api.Cache(d_kv, 8, 1, page, heads, dim, 1, head_scales=d_plane, bounds=bounds,
                      bound_scales=unit)
    # new block 4: zeros of both kinds; 5: of the second kind beside the small values
    half = page // 2
    tokens = list(range(half)) + list(range(page, page + half)) + \
        list(range(page + half, 2 * page)) + list(range(2 * page, 2 * page + half))
    rope = angles(3 * page, pairs).cuda() if turned else None
    cache.move_tokens(ints([[0, 1, 2]]), ints([[4, 5]]), ints(tokens), ints([0, len(tokens)]),
                      max_tokens=len(tokens), max_kv=3 * page, rope=rope)
    got, sc = d_kv.cpu().float(), d_plane.cpu()
    assert (got[0, 4] == 0).all()
    assert (sc[0, 4] == 2.0 ** -126).all()
    assert (bounds[0, 4] == 0).all()
    assert (got[0, 5, :, :page - half] == 0).all()
    small = got[0, 5, :, page - half:page - half + half]
    assert torch.isfinite(small).all() and (small[:, ::2] != 0).any(-1).all()
    assert torch.equal(small[1], codes[2, :half].float())  # values, whose scale stays


@pytest.mark.parametrize("latent,turn,page", [(128, 32, 16), (512, 64, 16), (384, 48, 5),
                                              (256, 64, 40)])
@pytest.mark.parametrize("turned", [False, True])
def test_moved_latents_of_zeros_stay_zeros(latent, turn, page, turned):
    need_gpu()
    where = (torch.arange(page) % 2 == 0)[:, None] * torch.ones(latent + turn)
    codes, scales = zeros_and_few(where)
    kv = torch.zeros((1, 8, page, latent + turn), dtype=FP8)
    kv[0, :3] = codes
    plane = torch.ones((1, 8, 2))
    plane[0, :3] = scales[:, None]
    d_kv, d_plane = kv.cuda(), plane.cuda()
    cache = api.LatentCache(d_kv, 8, 1, page, latent, turn, 1, scales=d_plane)
    half = page // 2
    tokens = list(range(half)) + list(range(page, page + page - half)) + \
        list(range(page + half, 2 * page)) + list(range(2 * page, 2 * page + half))
    rope = angles(3 * page, turn).cuda() if turned else None
    cache.move_tokens(ints([[0, 1, 2]]), ints([[4, 5]]), ints(tokens), ints([0, len(tokens)]),
                      max_tokens=len(tokens), max_kv=3 * page, rope=rope)
    got = d_kv.cpu().float()
    assert (got[0, 4] == 0).all()
    assert (d_plane[0, 4] == 2.0 ** -126).all()
    assert (got[0, 5, :page - half] == 0).all()
    small = got[0, 5, page - half:page]
    assert torch.isfinite(small).all()
    assert torch.equal(small[:, :latent], codes[2, :half, :latent].float())


# --------------------------------------- sequences without rows in a step

@pytest.mark.parametrize("scale", [math.nan, 0.0, 2.0 ** -140, -1.0, math.inf, 0.375])
@pytest.mark.parametrize("page", [16, 40])
def test_appended_latents_of_others_leave_a_sequence_without_rows_alone(page, scale):
    # its last block is filled in part; whatever its scales are they stay
    need_gpu()
    st = Latents([20, 60, 17], [0, 5, 0], heads=2, fp8=True, pow2=True, page=page)
    mine = [int(st.table[s, 20 // page if s == 0 else 17 // page]) for s in (0, 2)]
    st.scales[st.layer, mine] = scale
    st.to_device()
    new = st.rand(5, 1, 160).cuda()
    st.handle.append_latent(st.layer, st.batch, new[..., :128], new[..., 128:],
                            rope=angles(60, 32).cuda())
    theirs = [int(p) for p in st.table[1] if p >= 0]
    rest = [p for p in range(st.P) if p not in theirs]
    for got, was in ((st.d_cache, st.cache), (st.d_scales, st.scales)):
        assert torch.equal(got.cpu()[:, rest].view(torch.uint8), was[:, rest].view(torch.uint8))
    assert not torch.equal(st.d_cache.cpu()[:, theirs].view(torch.uint8),
                           st.cache[:, theirs].view(torch.uint8))


def test_appended_latents_take_no_heed_of_a_free_place_s_old_table():
    # a place of the batch that is free now, its length and table those of an earlier
    # step: the block that another sequence goes on writing
    need_gpu()
    results = []
    for stale in (False, True):
        st = Latents([40, 60], [0, 3], heads=2, fp8=True, pow2=True)
        if stale:
            st.table[0, 2] = st.table[1, 3]
        st.scales[st.layer] = 2.0 ** -20  # grows for any new token
        st.to_device()
        new = st.rand(3, 1, 160).cuda()
        st.handle.append_latent(st.layer, st.batch, new[..., :128], new[..., 128:])
        results.append([t.cpu().view(torch.uint8) for t in (st.d_cache, st.d_scales)])
    for a, b in zip(*results):
        assert torch.equal(a, b)


@pytest.mark.parametrize("scale", [math.nan, 0.0, 2.0 ** -140, -1.0, math.inf, 0.375, None])
@pytest.mark.parametrize("page", [16, 40])
def test_appended_keys_of_others_leave_a_sequence_without_rows_alone(page, scale):
    # None: a 16-bit cache; bounds of the block stay too, which may hold more tokens
    # than an earlier step's length says
    need_gpu()
    st = Setup([20, 60, 17], [0, 5, 0], heads=2, dim=64, fp8=scale is not None, bounds=True,
               page=page)
    mine = [int(st.table[s, 20 // page if s == 0 else 17 // page]) for s in (0, 2)]
    if scale is not None:
        st.scales[st.layer, mine] = scale
        st.d_scales[st.layer, mine] = scale
    st.d_bscales.fill_(3.0)
    k, v = st.rand(2).cuda(), st.rand(2).cuda()
    st.handle.append_kv(st.layer, st.batch, k, v, rope=angles(60, 64).cuda())
    theirs = [int(p) for p in st.table[1] if p >= 0]
    rest = [p for p in range(st.P) if p not in theirs]
    for got, was in ((st.d_cache, st.cache), (st.d_scales, st.scales)):
        if was is None:
            continue
        assert torch.equal(got.cpu()[:, rest].view(torch.uint8), was[:, rest].view(torch.uint8))
    assert (st.d_bounds[:, rest] == 77).all() and (st.d_bscales[:, rest] == 3.0).all()
    assert (st.d_bscales[st.layer, theirs[-1]] != 3.0).all()


def test_appended_keys_take_no_heed_of_a_free_place_s_old_table():
    need_gpu()
    results = []
    for stale in (False, True):
        st = Setup([40, 60], [0, 3], heads=2, dim=64, fp8=True, bounds=True)
        if stale:
            st.table[0, 2] = st.table[1, 3]
        batch = api.Batch(st.table.cuda(), ints(st.kv_lens), 60, ints(st.starts), 3, 3)
        st.d_scales[st.layer] = 2.0 ** -20  # grows for any new token
        st.d_bscales.fill_(3.0)
        k, v = st.rand(2).cuda(), st.rand(2).cuda()
        st.handle.append_kv(st.layer, batch, k, v)
        results.append([t.cpu().view(torch.uint8) for t in (st.d_cache, st.d_scales, st.d_bounds,
                                                            st.d_bscales)])
    for a, b in zip(*results):
        assert torch.equal(a, b)


# ------------------------------------------------------ starts that decrease

@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("held", [(0x7f7f7f7f, 0x7f7f7f7f), (1 << 30, 2), (-5, 3), (809, 2)])
def test_starts_that_decrease_stay_within_the_workspace(held, fp8):
    # 200 of 400 sequences claim all 40 rows, 1,000 units where the host counts and
    # launches fewer; the workspace holds numbers that are no units' places.  All
    # sequences are one, so whoever writes a row writes the same.
    need_gpu()
    n, seqs, heads = 40, 400, 16
    st = Latents([1000], [n], heads=heads, latent=512, turn=64, fp8=fp8)
    q = st.rand(n, heads, 576)
    d_q, guard = q.cuda(), 5
    out = torch.full((n + guard, heads, 512), 7.0, dtype=st.act, device="cuda")
    lse = torch.full((n + guard, heads), 7.0, device="cuda")
    batch = api.Batch(st.table.repeat(seqs, 1).cuda(), ints([1000] * seqs), 1000,
                      ints([0, n] * (seqs // 2) + [0]), n, n)
    lib, ref = N.load(), C.byref
    a = N.LatentAttention(*(N.Rows(t.data_ptr(), t.stride(0), t.stride(1)) for t in (d_q, out)))
    a.lse, a.latent_dim, a.rope_dim, a.q_heads = lse.data_ptr(), 512, 64, heads
    a.dtype, a.scale = N.EA_BF16, 0.07
    need = lib.ea_attend_latent_workspace(st.handle.handle, batch.ref, ref(a))
    assert need > 1 << 20
    ws = ints(held).repeat((need + 15) // 8 + 512)
    assert lib.ea_attend_latent(st.handle.handle, st.layer, batch.ref, ref(a), ws.data_ptr(), need,
                                api.current_stream()) == 0
    torch.cuda.synchronize()
    assert torch.equal(ws[-1024:], ints(held).repeat(512))
    assert (out[n:] == 7.0).all() and (lse[n:] == 7.0).all()
    check_attention(st, q, out[:n], lse[:n], 0.07, 2.0 ** -11 if fp8 else 2.0 ** -8)


# ------------------------------------------------- types of 16-bit caches

@pytest.mark.parametrize("act", [F16, BF16])
def test_a_cache_s_own_type_is_the_one_its_tokens_turn_in(act):
    # no dtype given; and one given for a cache held in bytes
    for held in (act, torch.uint8):
        st = Moved([100, 37], [70, 37], act=act, bounds=True)
        if held == torch.uint8:
            raw = st.d_cache.view(torch.uint8)
            st.handle = api.Cache(raw, st.P, st.L, st.T, st.H, st.D, 2, bounds=st.d_bounds,
                                  bound_scales=st.d_bscales)
        rope = angles(st.max_kv, st.D)
        st.move(rope=rope.cuda(), dtype=None if held == act else act)
        st.check(rope, False, range(st.L))


def test_latents_of_16_bit_turn_in_their_own_type():
    st = Latents([60], [1], act=F16, latent=128, turn=32)
    rope = angles(60, 32)
    free = [p for p in range(st.P) if p not in st.table]
    st.handle.move_tokens(st.table.cuda(), ints([free[:1]]), ints(range(40, 56)), ints([0, 16]),
                          max_tokens=16, max_kv=60, rope=rope.cuda())
    old = st.stored(0)[40:56]
    want, mag = turn64(old[:, 128:], rope, torch.full((16,), -40), False)
    got = st.d_cache[st.layer, free[0]].cpu().double()
    assert torch.equal(got[:, :128], old[:, :128])
    assert ((got[:, 128:] - want).abs() <=
            2.0 ** -11 * want.abs() + 2.0 ** -25 + 2.0 ** -22 * mag).all()


@pytest.mark.parametrize("act", [F16, BF16])
def test_bounds_of_blocks_go_by_the_cache_s_own_type(act):
    st = Moved([100], [16], act=act, bounds=True)
    pages = [int(p) for p in st.src[0] if p >= 0][:6]
    st.handle.bound_blocks(ints(pages))
    for page in pages:
        st.check_bounds(0, page, st.T, st.cache, None)
