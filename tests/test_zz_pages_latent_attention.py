"""Attention over a cache of latents on the GPU against its definition in 64
bits: single tokens, drafted rows, chunks, one token to long contexts, odd
sizes, strides, and what rows must not see."""
import math

import pytest
import torch

from gpu_common import need_gpu
from latent_common import BF16, F16, Latents, check_attention
from paper_2609_33762_amd import api

pytestmark = pytest.mark.gpu

KINDS = ["bf16", "f16", "fp8", "fp8_f16"]


def kind_args(kind):
    return dict(act=F16 if kind.endswith("f16") and kind != "bf16" else BF16,
                fp8=kind.startswith("fp8"))


def weights_of(kind, st):
    """Rounding of the weights: 11 bits beside f16 and fp8 latents, 8 beside
    bf16 ones."""
    return 2.0 ** -8 if kind == "bf16" else 2.0 ** -11


def attend(st, q, out=None, scale=None):
    scale = (st.C // 4 + st.R) ** -0.5 if scale is None else scale
    d_q = q.cuda()
    if out is None:
        out = torch.empty((st.n_rows, st.H, st.C), dtype=st.act, device="cuda")
    out.fill_(math.nan)
    lse = torch.full((st.n_rows, st.H), 7.0, device="cuda")
    st.handle.attend_latent(st.layer, st.batch, d_q, out, scale=scale, lse=lse)
    return out, lse, scale


def case(kind, scale=None, **kw):
    need_gpu()
    st = Latents(**kind_args(kind), **kw)
    q = st.rand(st.n_rows, st.H, st.C + st.R)
    out, lse, scale = attend(st, q, scale=scale)
    check_attention(st, q, out, lse, scale, weights_of(kind, st))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", [
    dict(kv_lens=[1, 2, 15, 16, 17, 31, 33, 100], rows=[1] * 8),
    dict(kv_lens=[40, 7], rows=[1, 1], heads=1, latent=16, turn=16),
    dict(kv_lens=[0, 5, 70], rows=[1, 1, 1], heads=5, latent=256, turn=64),
    dict(kv_lens=[130, 257, 64], rows=[1, 1, 1], heads=16, latent=512, turn=64),
    dict(kv_lens=[300, 65], rows=[1, 1], heads=40, latent=512, turn=64),
    dict(kv_lens=[200, 1, 90], rows=[1, 1, 1], heads=128, latent=512, turn=64),
    dict(kv_lens=[61, 20, 300], rows=[1, 1, 1], heads=3, latent=384, turn=48, page=5),
    dict(kv_lens=[61, 20, 300], rows=[1, 1, 1], heads=70, latent=272, turn=16, page=1),
    dict(kv_lens=[61, 200, 300], rows=[1, 1, 1], heads=33, latent=512, turn=64, page=48),
], ids=str)
def test_single_tokens(shape, kind):
    case(kind, **shape)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", [
    dict(kv_lens=[5, 40, 33, 300], rows=[3, 4, 1, 2], heads=16, latent=512, turn=64),
    dict(kv_lens=[3, 2, 90, 17], rows=[3, 2, 7, 5], heads=4, latent=128, turn=64),
    dict(kv_lens=[50, 9], rows=[6, 5], heads=1, latent=160, turn=32, page=7),
    # fewer cached tokens than rows: the first rows attend to nothing
    dict(kv_lens=[2, 0, 40], rows=[4, 3, 4], heads=8, latent=512, turn=64),
    dict(kv_lens=[20, 70, 5], rows=[9, 0, 5], heads=7, latent=512, turn=48, page=3),
], ids=str)
def test_few_rows(shape, kind):
    case(kind, **shape)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", [
    dict(kv_lens=[130], rows=[130], heads=2),
    dict(kv_lens=[300, 65, 200], rows=[40, 65, 1], heads=16, latent=512, turn=64),
    dict(kv_lens=[100, 77], rows=[20, 30], heads=5, latent=256, turn=16, page=5),
    dict(kv_lens=[40, 0, 90], rows=[66, 70, 90], heads=3, latent=512, turn=64),
], ids=str)
def test_chunks(shape, kind):
    case(kind, **shape)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_long_contexts_are_split_and_joined(kind):
    case(kind, kv_lens=[6000, 40, 3001], rows=[1, 1, 1], heads=4, latent=128, turn=32)
    case(kind, kv_lens=[7000], rows=[1], heads=128, latent=512, turn=64)
    case(kind, kv_lens=[5000, 333], rows=[2, 1], heads=16, latent=512, turn=64, page=20)
    case(kind, kv_lens=[4100], rows=[17], heads=9, latent=256, turn=64)


@pytest.mark.parametrize("kind", KINDS)
def test_scores_far_apart(kind):
    # weights from 1 down to underflow; references that grow along the tokens
    case(kind, kv_lens=[500, 60], rows=[1, 2], heads=4, scale=1.5)
    case(kind, kv_lens=[300], rows=[40], heads=4, latent=512, turn=64, scale=1.0)


@pytest.mark.parametrize("rows,heads", [(1, 16), (1, 128), (9, 16)])
def test_references_that_grow_with_every_token(rows, heads):
    # each token's score lies some 12 above the last one's, from far below 0 on
    need_gpu()
    st = Latents(kv_lens=[150], rows=[rows], heads=heads, latent=512, turn=64)
    x = st.cache[st.layer]
    for j in range(150):
        row = x[int(st.table[0, j // 16]), j % 16]
        row[0] = (j - 120) * 2.0
    st.to_device()
    q = torch.zeros((rows, heads, 576))
    q[..., 0] = 6.0
    q[..., 1:] = torch.randn((rows, heads, 575), generator=st.g) * 0.01
    q = q.to(BF16)
    out, lse, scale = attend(st, q, scale=1.0)
    check_attention(st, q, out, lse, scale, 2.0 ** -8)


def test_strides():
    # a slice of a wider row, and an output with the heads outside
    need_gpu()
    st = Latents(kv_lens=[100, 41], rows=[3, 1], heads=6, latent=256, turn=64)
    wide = st.rand(st.n_rows, 11, 336)
    q = wide[:, 3:9, 8:328]
    out = torch.empty((6, st.n_rows, 256), dtype=BF16, device="cuda").transpose(0, 1)
    lse = torch.empty((st.n_rows, 6), device="cuda")
    st.handle.attend_latent(st.layer, st.batch, wide.cuda()[:, 3:9, 8:328], out, scale=0.1, lse=lse)
    check_attention(st, q, out, lse, 0.1, 2.0 ** -8)


@pytest.mark.parametrize("page", [16, 5])
@pytest.mark.parametrize("rows,heads", [(1, 16), (4, 16), (40, 4)])
def test_pages_outside_the_cache_hold_no_tokens(rows, heads, page):
    need_gpu()
    st = Latents(kv_lens=[100], rows=[rows], heads=heads, latent=512, turn=64, page=page)
    q = st.rand(rows, heads, 576)
    table = st.table.clone()
    table[0, 2], table[0, 4] = st.P, -3
    b = api.Batch(table.cuda(), st.batch.kv_len, 100, st.batch.row_start, rows, rows)
    out = torch.empty((rows, heads, 512), dtype=BF16, device="cuda")
    lse = torch.empty((rows, heads), device="cuda")
    st.handle.attend_latent(st.layer, b, q.cuda(), out, scale=0.08, lse=lse)
    hidden = [p * page + i for p in (2, 4) for i in range(page)]
    check_attention(st, q, out, lse, 0.08, 2.0 ** -8, hidden=hidden)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("rows,heads", [(4, 5), (4, 16), (30, 16)])
def test_what_is_not_finite_reaches_only_rows_that_attend_to_it(rows, heads, value, kind):
    # in the last row's own token, which the rows before it do not see
    need_gpu()
    st = Latents(kv_lens=[200], rows=[rows], heads=heads, latent=512, turn=64, **kind_args(kind))
    if kind == "fp8":
        value = math.nan
    q = st.rand(rows, heads, 576)
    clean = [t.clone() for t in attend(st, q)[:2]]
    st.cache[st.layer, int(st.table[0, 199 // 16]), 199 % 16, 7] = value
    st.to_device()
    out, lse, scale = attend(st, q)
    assert torch.equal(out[:-1], clean[0][:-1]) and torch.equal(lse[:-1], clean[1][:-1])
    for h in range(heads):  # the row's own score decides how far it goes
        if math.isinf(value) and math.copysign(1.0, value) * float(q[-1, h, 7]) < 0:
            assert torch.isnan(out[-1, h, 7])  # a weight of zero times infinity
            rest = torch.cat([out[-1, h, :7], out[-1, h, 8:]])
            assert torch.isfinite(rest).all() and torch.isfinite(lse[-1, h])
        else:
            assert torch.isnan(out[-1, h]).all()


def test_scales_of_blocks_far_apart():
    need_gpu()
    st = Latents(kv_lens=[300, 64], rows=[2, 1], heads=16, latent=512, turn=64, fp8=True)
    g = torch.Generator().manual_seed(5)
    st.scales[..., 0] = torch.exp2(-torch.randint(4, 40, st.scales[..., 0].shape,
                                                  generator=g).float())
    st.to_device()
    q = st.rand(3, 16, 576)
    out, lse, scale = attend(st, q)
    check_attention(st, q, out, lse, scale, 2.0 ** -11)


def test_scales_of_blocks_of_zeros():
    # the smallest scale there is: such tokens take weight and add nothing
    need_gpu()
    st = Latents(kv_lens=[100, 40], rows=[1, 1], heads=16, latent=512, turn=64, fp8=True)
    pages = [int(st.table[0, p]) for p in (0, 2, 3)] + [int(st.table[1, p]) for p in range(3)]
    st.cache[st.layer, pages, :, :512] = 0
    st.scales[st.layer, pages, 0] = 2.0 ** -126
    st.to_device()
    q = st.rand(2, 16, 576)
    out, lse, scale = attend(st, q)
    check_attention(st, q, out, lse, scale, 2.0 ** -11)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("n,most,heads", [(70, 900, 3), (270, 500, 2), (300, 1300, 33), (530, 200, 2)])
def test_many_sequences(n, most, heads, kind):
    # more than a wave's lanes; more units than compute units, whole or in parts
    lens = [(i * 37) % most for i in range(n)]
    lens[n // 2], lens[n - 1] = most, 2 * most
    case(kind, kv_lens=lens, rows=[1 + (i % 7 == 0) for i in range(n)], heads=heads, latent=64,
         turn=16)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("length", [129, 1000, 2100, 9000])
@pytest.mark.parametrize("latent", [16, 48, 512])
def test_parts_of_one_sequence(length, latent, kind):
    # two parts, some, as many as one wave joins, and more
    case(kind, kv_lens=[length], rows=[1], heads=6, latent=latent, turn=16)
