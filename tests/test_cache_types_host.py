"""The type that a 16-bit cache's elements are taken in, without a GPU."""
import pytest
import torch

from paper_2609_33762_amd import _native as N
from paper_2609_33762_amd import api


@pytest.mark.parametrize("cls", [api.Cache, api.LatentCache])
def test_elements_are_of_the_type_given_or_of_the_tensor_s(cls):
    c = object.__new__(cls)  # no memory, no handle
    c._h = None
    for held, given, want in (
            (torch.float16, None, N.EA_F16), (torch.bfloat16, None, N.EA_BF16),
            (torch.uint8, None, N.EA_BF16), (torch.uint8, torch.float16, N.EA_F16),
            (torch.int16, torch.bfloat16, N.EA_BF16), (torch.float16, torch.float16, N.EA_F16)):
        c.kv = torch.zeros(4, dtype=held)
        assert c._held(given) == want, (held, given)
    with pytest.raises(ValueError, match="bfloat16 or float16"):
        c._held(torch.float32)
