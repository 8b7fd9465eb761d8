"""Latent attention that shows every token: equal scores, so that each weight is
one over the tokens seen, and latents of a single one, so that an output element is
the share of the tokens that have it.  A token that is lost or taken twice, in
the steps of a part or between parts, changes a share by more than its rounding.

Bounds: scores are zeros and weights powers of two, so sums are exact; 1 / total
and its product are off by 2^-22, the result's rounding by u; log2 and its product
by 2^-22 of it each, the sum with the reference by 2^-24 of both."""
import math

import pytest
import torch

from gpu_common import need_gpu
from latent_common import BF16, F16, ULP, Latents


def columns_of(tokens, pattern, latent):
    return tokens % latent if pattern == "tokens" else tokens // 32 % latent


def shares(length, pattern, latent, drop=(), twice=()):
    """Counts of the first `length` tokens' columns over their number, and its
    logarithm; for tests of the check, with tokens lost or taken twice."""
    weight = torch.ones(length, dtype=torch.float64)
    weight[list(drop)] = 0
    weight[list(twice)] = 2
    n = torch.zeros(latent, dtype=torch.float64)
    n.index_add_(0, columns_of(torch.arange(length), pattern, latent), weight)
    return n / weight.sum(), math.log(weight.sum())


def check_shares(length, pattern, out, lse, act):
    """Outputs [heads, latent] and lse [heads] of a row that sees `length` tokens."""
    want, want_lse = shares(length, pattern, out.shape[-1])
    assert ((out.double() - want).abs() <= (ULP[act] + 2.0 ** -22) * want).all(), length
    assert ((lse.double() - want_lse).abs() <= 2.0 ** -20 * max(want_lse, 1.0)).all(), length


@pytest.mark.parametrize("pattern", ["tokens", "steps"])
@pytest.mark.parametrize("latent", [128, 512])
@pytest.mark.parametrize("length", [3, 129, 2100, 9000, 20000])
def test_lost_and_doubled_tokens_are_seen(length, latent, pattern):
    out, lse = shares(length, pattern, latent)
    check_shares(length, pattern, out.to(BF16)[None], torch.tensor([lse]).float(), BF16)
    for at in (0, length // 2, length - 1):
        step = range(at // 32 * 32, min(at // 32 * 32 + 32, length))
        for wrong in (dict(drop=[at]), dict(twice=[at]), dict(drop=step), dict(twice=step)):
            (some,) = wrong.values()
            if "drop" in wrong and len(some) == length:
                continue
            bad, bad_lse = shares(length, pattern, latent, **wrong)
            with pytest.raises(AssertionError):  # of the logarithm
                check_shares(length, pattern, out.to(BF16)[None],
                             torch.tensor([bad_lse]).float(), BF16)
            # and of the outputs, but where all tokens count twice, or 8 bits are too few
            fine = len(some) == 32 if pattern == "steps" else latent == 512
            if fine and len(some) < length:
                with pytest.raises(AssertionError):
                    check_shares(length, pattern, bad.to(BF16)[None],
                                 torch.tensor([lse]).float(), BF16)


KINDS = ["bf16", "f16", "fp8"]


def run(kv_lens, rows, heads, latent, pattern, kind, turn=64, page=16):
    need_gpu()
    st = Latents(kv_lens, rows, heads=heads, latent=latent, turn=turn, page=page,
                 act=F16 if kind == "f16" else BF16, fp8=kind == "fp8")
    lay = torch.zeros((st.P, page, latent))
    power = torch.ones(st.P)
    if st.fp8:  # ones as codes of 1 to 64 under scales that differ from block to block
        power = torch.exp2(torch.randint(0, 7, (st.P,), generator=st.g).float())
        st.scales[st.layer, :, 0] = 1.0 / power
    for s, n in enumerate(kv_lens):
        j = torch.arange(n)
        pages = st.table[s].long()[j // page]
        lay[pages, j % page, columns_of(j, pattern, latent)] = power[pages]
    held = torch.isfinite(st.cache[st.layer].float()).all(-1, keepdim=True)
    raw = st.cache.view(torch.uint8 if st.fp8 else torch.int16)
    new = lay.to(st.cache.dtype).view(raw.dtype)
    raw[st.layer, :, :, :latent] = torch.where(held, new, raw[st.layer, :, :, :latent])
    st.to_device()
    q = torch.zeros((st.n_rows, heads, latent + turn), dtype=st.act, device="cuda")
    out = torch.full((st.n_rows, heads, latent), math.nan, dtype=st.act, device="cuda")
    lse = torch.full((st.n_rows, heads), math.nan, device="cuda")
    st.handle.attend_latent(st.layer, st.batch, q, out, scale=0.1, lse=lse)
    out, lse = out.cpu(), lse.cpu()
    for s, n in enumerate(rows):
        for r in range(n):
            check_shares(kv_lens[s] - n + r + 1, pattern, out[st.starts[s] + r],
                         lse[st.starts[s] + r], st.act)


# columns (rows times heads) that one, two and four waves take, and more tiles
@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,heads", [(1, 6), (1, 40), (1, 128), (3, 16), (9, 16)])
@pytest.mark.parametrize("length", [
    31, 32, 33, 127, 128, 129, 511, 512, 513, 545, 1024, 2100, 4095, 4097, 9000, 16385])
def test_every_token_of_one_sequence_counts_once(length, rows, heads, kind):
    run([length], [rows], heads, 512, "tokens", kind)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("latent,turn,page", [(256, 64, 16), (384, 48, 16), (512, 64, 5),
                                              (128, 32, 64), (512, 64, 48)])
@pytest.mark.parametrize("rows,heads", [(1, 6), (2, 20), (4, 16), (1, 128)])
def test_every_token_counts_once_in_other_forms(rows, heads, latent, turn, page, kind):
    for length in (70, 1000, 2100):
        run([length], [rows], heads, latent, "tokens", kind, turn, page)
    run([9000], [rows], heads, latent, "steps", kind, turn, page)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,most,heads,rows", [(5, 4000, 16, 1), (64, 2000, 4, 2), (70, 900, 3, 1),
                                               (270, 300, 2, 1), (24, 1500, 16, 4)])
def test_every_token_of_many_sequences_counts_once(n, most, heads, rows, kind):
    lens = [max(rows, (i * 37 * 17) % most) for i in range(n)]
    lens[n // 2], lens[n - 1] = most, 2 * most + 1
    run(lens, [rows] * n, heads, 512, "tokens", kind)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
def test_every_token_of_a_chunk_counts_once(kind):
    run([700], [300], 3, 512, "tokens", kind)
    run([5000, 90], [40, 90], 16, 256, "steps", kind)
