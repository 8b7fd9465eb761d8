"""The cache operators' entry points without a GPU: refusals of the C entry
points, of the binding's classes, and the device code's instruction rules (no
packed FP32, only vector stores, a bound on scratch memory)."""
import ctypes as C
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_33762_amd import _native as N
from paper_2609_33762_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EA_EINVAL = -1


@pytest.fixture(scope="module")
def lib():
    return N.load()


def test_null_arguments_are_refused(lib):
    b, rows = N.BatchDesc(), (None, 0, 0)
    planes = N.CachePlanes(None, None, None)
    att, sel, app = N.Attention(rows, rows), N.Selection(rows), N.Append(rows, rows)
    r = C.byref
    assert lib.ea_append_kv(None, r(planes), 0, r(b), r(app), None) == EA_EINVAL
    assert lib.ea_bound_blocks(None, r(planes), 0, 1, None, 0, 0, None) == EA_EINVAL
    assert lib.ea_attend_workspace(None, r(b), r(att)) == EA_EINVAL
    assert lib.ea_attend(None, r(planes), 0, r(b), r(att), None, 0, None) == EA_EINVAL
    assert lib.ea_select_workspace(None, r(b), r(sel)) == EA_EINVAL
    assert lib.ea_select_blocks(None, r(planes), 0, r(b), r(sel), None, 0, None) == EA_EINVAL
    assert lib.ea_append_kv(None, None, 0, None, None, None) == EA_EINVAL
    assert lib.ea_attend_workspace(None, None, None) == EA_EINVAL


def test_structures_have_the_header_s_sizes():
    # the header's structures, compiled by a C compiler, against the binding's
    cc = shutil.which("gcc")
    if cc is None:
        pytest.skip("no C compiler")
    names = {"ea_cache_planes": N.CachePlanes, "ea_batch": N.BatchDesc, "ea_rows": N.Rows,
             "ea_append": N.Append, "ea_attention": N.Attention, "ea_selection": N.Selection}
    src = '#include <stdio.h>\n#include "ea.h"\nint main(void){' + "".join(
        f'printf("{n} %zu\\n", sizeof({n}));' for n in names) + "return 0;}"
    import tempfile
    with tempfile.TemporaryDirectory() as d:
        exe = os.path.join(d, "sizes")
        subprocess.run([cc, "-x", "c", "-", "-D__HIP_PLATFORM_AMD__", "-I",
                        os.path.join(ROOT, "include"), "-I", "/opt/rocm/include", "-o", exe],
                       input=src.encode(), check=True)
        out = subprocess.run([exe], capture_output=True, check=True).stdout.decode()
    for line in out.split("\n")[:-1]:
        name, size = line.split()
        assert int(size) == C.sizeof(names[name]), name


# ------------------------------------------------------------- device code

SCALAR_WRITES = re.compile(r"^\s+s_(" + "st" + "ore|buffer_st" + "ore|atomic|dcache_" + "wb|scratch_st"
                           + "ore)")
PACKED_F32 = re.compile(r"^\s+v_pk_(add|mul|fma)_" + "f32")
SOURCES = ["ea_append_kernels.hip", "ea_select_kernels.hip", "ea_attend_split.hip",
           "ea_attend_chunk.hip"]


@pytest.mark.parametrize("src", SOURCES)
def test_device_code(src, tmp_path):
    cc = "/opt/rocm/bin/hipcc" if os.path.exists("/opt/rocm/bin/hipcc") else shutil.which("hipcc")
    if cc is None:
        pytest.skip("hipcc not available")
    path = os.path.join(ROOT, "paper_2609_33762_amd", "csrc", src)
    out = str(tmp_path / "k.s")
    subprocess.run([cc] + build.COMMON + ["-x", "hip", "--cuda-device-only", "-S", path, "-o", out],
                   check=True, capture_output=True)
    text = open(out).read()
    bad = [x for x in text.split("\n") if SCALAR_WRITES.match(x) or PACKED_F32.match(x)]
    assert not bad, bad[:3]
    found = re.findall(r"\.name:\s+(\S+)\n(?:.*\n)*?\s+\.private_segment_fixed_size:\s+(\d+)", text)
    kernels = {n: int(s) for n, s in found if n.startswith("_Z")}
    assert kernels
    # no kernel keeps an array in scratch; heads of 256 and pages that are no
    # whole tiles spill a few registers
    most = {n: s for n, s in kernels.items() if s > 160}
    assert not most, most
    wide = {n: s for n, s in kernels.items() if s and "attend" not in n}
    assert not wide, wide
