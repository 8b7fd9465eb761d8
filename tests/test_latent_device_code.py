"""Device code of the latent attention, the appended latents and the pages' copies
and moves: instruction rules, bounds on scratch memory, and the waits around
matrix instructions whose operands the compiler does not know of."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_33762_amd import build
from test_cache_ops_host import PACKED_F32, SCALAR_WRITES

SOURCES = ["ea_attend_latent.hip", "ea_latent_append.hip", "ea_page_kernels.hip"]
AFTER = 12   # wait states from a matrix instruction (8 passes) to a read of its results
BEFORE = 2   # from a vector instruction's write to a matrix instruction's read


@pytest.fixture(scope="module")
def device_code(tmp_path_factory):
    cc = "/opt/rocm/bin/hipcc" if os.path.exists("/opt/rocm/bin/hipcc") else shutil.which("hipcc")
    if cc is None:
        pytest.skip("hipcc not available")
    out = {}
    for src in SOURCES:
        path = str(tmp_path_factory.mktemp("s") / "k.s")
        subprocess.run([cc] + build.COMMON + ["-x", "hip", "--cuda-device-only", "-S",
                                              os.path.join(build.CSRC, src), "-o", path],
                       check=True, capture_output=True)
        out[src] = open(path).read()
    return out


@pytest.mark.parametrize("src", SOURCES)
def test_instructions(src, device_code):
    bad = [x for x in device_code[src].split("\n") if SCALAR_WRITES.match(x) or PACKED_F32.match(x)]
    assert not bad, bad[:3]


def bodies(text):
    for m in re.finditer(r"^(_Z\w+):.*?\n(.*?)^\.Lfunc_end", text, re.M | re.S):
        yield m[1], m[2]


def scratch(text):
    found = re.findall(r"\.name:\s+(\S+)\n(?:.*\n)*?\s+\.private_segment_fixed_size:\s+(\d+)", text)
    return {n: int(s) for n, s in found if n.startswith("_Z")}


def test_scratch(device_code):
    append = scratch(device_code["ea_latent_append.hip"])
    assert append and not any(append.values())
    moves = scratch(device_code["ea_page_kernels.hip"])
    assert moves and max(moves.values()) <= MOVES
    latent = scratch(device_code["ea_attend_latent.hip"])
    assert latent and max(latent.values()) <= ATTENTION, latent


def test_scratch_in_the_steps_of_the_attention(device_code):
    # what is spilled is spilled once, before the steps: a step has thousands of
    # instructions and reloads a few of those registers, or none
    seen = 0
    for name, body in bodies(device_code["ea_attend_latent.hip"]):
        lines = body.split("\n")
        products = [i for i, x in enumerate(lines) if "v_mfma" in x]
        if not products:
            continue
        loops = [i for i, x in enumerate(lines) if "Loop Header: Depth=1" in x and i < products[-1]]
        steps = lines[loops[-1]:products[-1] + 40]
        loads, stores = (sum("scratch_" + x in y for y in steps) for x in ("load", "store"))
        assert loads <= 16 and stores <= 2, (name, loads, stores)
        seen += 1
    assert seen


# most bytes a lane: heads that are no whole lanes, moved; rows of 512 elements in registers
MOVES, ATTENTION = 256, 448


# ------------------------------------------------- waits around matrix instructions

def registers(operand):
    """{("v", 3), ...} of an operand such as v3, a[4:7] or -v2."""
    m = re.match(r"^[-|]*([va])(?:(\d+)|\[(\d+):(\d+)\])", operand.strip())
    if not m:
        return set()
    lo, hi = (int(m[2]), int(m[2])) if m[2] else (int(m[3]), int(m[4]))
    return {(m[1], i) for i in range(lo, hi + 1)}


class Code:
    """A kernel's instructions: (name, registers written, registers read, waits), and
    what can follow each."""

    def __init__(self, lines):
        self.ins, self.next, labels, jumps = [], [], {}, []
        for line in lines:
            line = line.split(";")[0].split("//")[0].rstrip()
            m = re.match(r"^(\S+):$", line.strip())
            if m:
                labels[m[1]] = len(self.ins)
                continue
            m = re.match(r"^\s+([a-z]\w+)\s*(.*)$", line)
            if not m or line.strip().startswith("."):
                continue
            name, ops = m[1], [x for x in re.split(r",(?![^\[]*\])", m[2])]
            regs = [registers(x) for x in ops]
            store = re.match(r"(global|buffer|flat|scratch)_store|ds_write|.*_lds_|s_", name)
            wrote = set() if store or not regs else regs[0]
            read = set().union(*(regs if store else regs[1:])) if regs else set()
            if name.startswith("v_permlane") and "swap" in name or name.startswith("v_swap"):
                wrote, read = regs[0] | regs[1], regs[0] | regs[1]
            waits = int(ops[0], 0) + 1 if name == "s_nop" else 1
            if name.startswith("s_cbranch") or name == "s_branch":
                jumps.append((len(self.ins), ops[0].strip()))
            self.ins.append((name, wrote, read, waits))
        for i, (name, *_) in enumerate(self.ins):
            self.next.append([i + 1] if i + 1 < len(self.ins) and
                             name not in ("s_branch", "s_endpgm") else [])
        for i, label in jumps:
            if label in labels and labels[label] < len(self.ins):
                self.next[i].append(labels[label])

    def after(self, i, states):
        """Instructions that can run fewer than `states` wait states after i."""
        best, todo = {}, [(j, 0) for j in self.next[i]]
        while todo:
            j, waited = todo.pop()
            if waited >= states or best.get(j, states) <= waited:
                continue
            best[j] = waited
            todo += [(k, waited + self.ins[j][3]) for k in self.next[j]]
        return best


def hazards(code):
    out = []
    for i, (name, wrote, read, _) in enumerate(code.ins):
        if name.startswith("v_mfma"):
            for j in code.after(i, AFTER):
                other, w, r, _ = code.ins[j]
                # sums that go on in the same registers need no wait
                if other.startswith("v_mfma"):
                    if w == wrote or not (r | w) & wrote:
                        continue
                elif not other.startswith(("v_", "global", "buffer", "flat", "scratch", "ds_")):
                    continue
                if (r | w) & wrote:
                    out.append((name, i, other, j))
        elif name.startswith("v_"):
            for j in code.after(i, BEFORE):
                other, w, r, _ = code.ins[j]
                if other.startswith("v_mfma") and r & wrote:
                    out.append((name, i, other, j))
    return out


def kernels(text):
    for name, body in bodies(text):
        yield name, Code(body.split("\n"))


def test_missing_waits_are_seen():
    mfma = "\tv_mfma_f32_32x32x16_bf16 v[0:15], v[16:19], v[20:23], 0\n"
    lines = lambda s: hazards(Code(s.split("\n")))  # noqa: E731
    assert lines(mfma + "\tv_mov_b32_e32 v30, v3\n")
    assert lines(mfma + "\ts_nop 10\n\tv_mov_b32_e32 v30, v3\n")
    assert not lines(mfma + "\ts_nop 11\n\tv_mov_b32_e32 v30, v3\n")
    assert not lines(mfma + mfma.replace(" 0\n", " v[0:15]\n"))
    assert lines(mfma + mfma.replace("v[0:15]", "v[40:55]").replace("v[16:19]", "v[12:15]"))
    assert lines("\tv_mov_b32_e32 v17, v3\n\ts_nop 0\n" + mfma)
    assert not lines("\tv_mov_b32_e32 v17, v3\n\ts_nop 1\n" + mfma)
    loop = ".LBB0_1:\n\tv_mov_b32_e32 v30, v3\n\ts_nop 1\n" + mfma + "\ts_cbranch_scc1 .LBB0_1\n"
    assert lines(loop)


def test_waits_around_matrix_instructions(device_code):
    seen = 0
    for name, code in kernels(device_code["ea_attend_latent.hip"]):
        if "attend_latent" not in name:
            continue
        seen += any(x[0].startswith("v_mfma") for x in code.ins)
        bad = hazards(code)
        assert not bad, (name, len(bad), bad[:3], [code.ins[k] for k in range(
            max(0, bad[0][1] - 1), bad[0][3] + 1)][:24])
    assert seen
