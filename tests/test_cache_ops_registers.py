"""Registers of the attention kernels: those of heads of 64 and 128 elements and
of pages of whole 16 tokens, the ones that serving runs, keep everything in them."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_33762_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# template arguments: activation type, fp8, a head's size, whether pages are whole tiles
@pytest.mark.parametrize("src,kernel,most", [
    ("ea_attend_split.hip", r"attend_splitILi\dELb[01]ELi(\d+)ELi\dELb1E", 8),
    ("ea_attend_chunk.hip", r"attend_chunkILi\dELb[01]ELi(\d+)ELb1E", 4)])
def test_no_scratch_in_the_main_attention_kernels(src, kernel, most, tmp_path):
    cc = "/opt/rocm/bin/hipcc" if os.path.exists("/opt/rocm/bin/hipcc") else shutil.which("hipcc")
    if cc is None:
        pytest.skip("hipcc not available")
    out = str(tmp_path / "k.s")
    subprocess.run([cc] + build.COMMON + ["-x", "hip", "--cuda-device-only", "-S",
                                          os.path.join(build.CSRC, src), "-o", out],
                   check=True, capture_output=True)
    text = open(out).read()
    found = re.findall(r"\.name:\s+(\S+)\n(?:.*\n)*?\s+\.private_segment_fixed_size:\s+(\d+)", text)
    main = {}
    for name, size in found:
        m = re.search(kernel, name)
        if m and int(m.group(1)) <= most:
            main[name] = int(size)
    assert len(main) >= 8
    assert not any(main.values()), {n: s for n, s in main.items() if s}
