"""Weights of the latent attention beside bf16 latents.  Values of both signs whose
weights are nearly alike leave little of a sum, so that what a weight is rounded
by shows; scores come from the turned parts alone and are small, so they are exact
to 2^-20.  A weight as the sum of two bf16 is off by half a step of the second,
2^-8 of at most 2^-8 of the weight."""
import math

import pytest
import torch

from gpu_common import need_gpu
from latent_common import Latents, check_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,heads", [(1, 1), (1, 16), (4, 16), (1, 64), (2, 17)])
@pytest.mark.parametrize("latent,turn,page", [(128, 32, 16), (512, 64, 16), (384, 48, 5)])
@pytest.mark.parametrize("length", [8, 40, 301, 2500])
def test_weights_of_few_rows_are_two_bf16(length, latent, turn, page, rows, heads):
    need_gpu()
    st = Latents([length], [rows], heads=heads, latent=latent, turn=turn, page=page)
    j = torch.arange(length)
    pages = st.table[0].long()[j // page]
    x = st.cache[st.layer, pages, j % page]
    x[:, :latent] = torch.where((j % 2 == 0)[:, None], 1.0, -1.0).to(st.act)
    st.cache[st.layer, pages, j % page] = x
    st.to_device()
    q = torch.zeros((rows, heads, latent + turn))
    q[..., latent:] = torch.randn((rows, heads, turn), generator=st.g) * 0.1
    q = q.to(st.act)
    out = torch.full((rows, heads, latent), math.nan, dtype=st.act, device="cuda")
    lse = torch.empty((rows, heads), device="cuda")
    st.handle.attend_latent(st.layer, st.batch, q.cuda(), out, scale=0.1, lse=lse)
    check_attention(st, q, out, lse, 0.1, 2.0 ** -16)
