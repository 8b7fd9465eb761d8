"""Latents, copied pages and moved tokens without a GPU: what the C entry points
refuse, and that the header's structures and the binding's have one size."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from paper_2609_33762_amd import _native as N
from paper_2609_33762_amd import api

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EA_EINVAL = -1


def test_null_arguments_are_refused():
    lib, r = N.load(), C.byref
    b, planes = N.BatchDesc(), N.CachePlanes(None, None, None)
    app, att, move = N.LatentAppend(), N.LatentAttention(), N.Move()
    app.latent_dim = att.latent_dim = move.latent_dim = 512
    app.rope_dim = att.rope_dim = move.rope_dim = 64
    fake = C.c_void_p(0x10000)  # never read
    assert lib.ea_append_latent(None, 0, r(b), r(app), None) == EA_EINVAL
    assert lib.ea_append_latent(None, 0, r(b), None, None) == EA_EINVAL
    assert lib.ea_attend_latent_workspace(None, r(b), r(att)) == EA_EINVAL
    assert lib.ea_attend_latent_workspace(None, None, None) == EA_EINVAL
    assert lib.ea_attend_latent(None, 0, r(b), r(att), None, 0, None) == EA_EINVAL
    assert lib.ea_attend_latent(None, 0, None, None, fake, 1 << 20, None) == EA_EINVAL
    assert lib.ea_copy_pages(None, r(planes), fake, fake, 1, None) == EA_EINVAL
    assert lib.ea_copy_pages(None, None, None, None, 0, None) == EA_EINVAL
    assert lib.ea_move_tokens(None, r(planes), 0, 1, r(move), None) == EA_EINVAL
    move.latent_dim = 0
    assert lib.ea_move_tokens(None, r(planes), 0, 1, r(move), None) == EA_EINVAL
    assert lib.ea_move_tokens(None, None, 0, 1, None, None) == EA_EINVAL


def test_structures_have_the_header_s_layout(tmp_path):
    cc = shutil.which("gcc")
    if cc is None:
        pytest.skip("no C compiler")
    names = {"ea_latent_append": N.LatentAppend, "ea_latent_attention": N.LatentAttention,
             "ea_move": N.Move}
    lines = [f'printf("{n} {f} %zu\\n", offsetof({n}, {f}));' for n, t in names.items()
             for f, _ in t._fields_]
    lines += [f'printf("{n} - %zu\\n", sizeof({n}));' for n in names]
    src = '#include <stdio.h>\n#include <stddef.h>\n#include "ea.h"\nint main(void){' + \
        "".join(lines) + "return 0;}"
    exe = str(tmp_path / "sizes")
    subprocess.run([cc, "-x", "c", "-", "-D__HIP_PLATFORM_AMD__", "-I",
                    os.path.join(ROOT, "include"), "-I", "/opt/rocm/include", "-o", exe],
                   input=src.encode(), check=True)
    out = subprocess.run([exe], capture_output=True, check=True).stdout.decode()
    for line in out.split("\n")[:-1]:
        name, field, n = line.split()
        got = C.sizeof(names[name]) if field == "-" else getattr(names[name], field).offset
        assert got == int(n), line


def test_a_cache_of_latents_needs_whole_pairs():
    with pytest.raises(ValueError, match="even"):
        api.LatentCache(None, 4, 1, 16, 511, 64, 2)


def test_operators_of_keys_and_values_are_refused():
    c = object.__new__(api.LatentCache)  # no memory, no handle
    c._h = None
    for name in ("append_kv", "attend", "select_blocks", "bound_blocks"):
        with pytest.raises(TypeError, match="append_latent"):
            getattr(c, name)(0)
