"""The cache operators call by call: calls of many units, calls that share a
workspace, captured calls, steps whose rows only the device knows, selections
in any order.  Compared with 64-bit computations; the bounds of the errors are
those of tests/test_gpu_cache_ops.py."""
import ctypes as C
import math

import pytest
import torch

import test_gpu_cache_ops as base
from gpu_common import need_gpu
from paper_2609_33762_amd import _native as N
from paper_2609_33762_amd import api

pytestmark = pytest.mark.gpu

BF16, F16, FP8 = base.BF16, base.F16, base.FP8
FEW, MANY = 2.0 ** -15, 2.0 ** -8  # rounding of bf16 kernels' weights: few rows, a chunk's


class Step:
    """Sequences over one small cache of random pages, which they share."""

    def __init__(self, lens, rows, heads, group, dim, page=16, pages=96, seed=0, max_kv=None,
                 n_rows=None, max_rows=None):
        need_gpu()
        self.g = torch.Generator().manual_seed(seed)
        self.H, self.G, self.D, self.T = heads, group, dim, page
        self.lens, self.rows = list(lens), list(rows)
        self.starts = [0]
        for n in self.rows:
            self.starts.append(self.starts[-1] + n)
        self.n_rows = self.starts[-1] if n_rows is None else n_rows
        self.kv = torch.randn((1, pages, 2, page, heads, dim), generator=self.g).to(BF16).cuda()
        self.max_kv = max(self.lens + [1]) if max_kv is None else max_kv
        self.table = torch.randint(pages, (len(self.lens), -(-self.max_kv // page)),
                                   generator=self.g, dtype=torch.int32).cuda()
        self.cache = api.Cache(self.kv, pages, 1, page, heads, dim, 2)
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        self.kv_len, self.row_start = ints(self.lens), ints(self.starts)
        self.max_rows = max(self.rows + [1]) if max_rows is None else max_rows
        self.batch = self.new_batch()
        self.q = torch.randn((self.n_rows, heads * group, dim), generator=self.g).to(BF16).cuda()

    def new_batch(self):
        return api.Batch(self.table, self.kv_len, self.max_kv, self.row_start, self.n_rows,
                         self.max_rows)

    def choose(self, budget):
        """Distinct random blocks for every row and head, among the blocks up
        to its sequence's last one, -1 after them."""
        sel = torch.full((self.n_rows, self.H, budget), -1, dtype=torch.int32)
        for s, n in enumerate(self.rows):
            held = -(-self.lens[s] // self.T)
            take = min(held, budget)
            some = torch.rand((n, self.H, held), generator=self.g).argsort(-1)[..., :take]
            sel[self.starts[s]:self.starts[s + 1], :, :take] = some.sort(-1).values.int()
        return sel.cuda()

    def exact(self, selected=None):
        """(output, sum of weights times |v|, log-sum-exp) in 64 bits."""
        H, G, D, T = self.H, self.G, self.D, self.T
        kv = self.kv[0].double()
        o = torch.zeros((self.n_rows, H * G, D), dtype=torch.float64, device="cuda")
        a, lse = torch.zeros_like(o), torch.full((self.n_rows, H * G), -math.inf,
                                                 dtype=torch.float64, device="cuda")
        for s, n in enumerate(self.rows):
            length, at = self.lens[s], self.starts[s]
            if n == 0 or length == 0:
                continue
            pages = self.table[s, :-(-length // T)].long()
            k, v = (kv[pages, i].reshape(-1, H, D)[:length].transpose(0, 1).contiguous()
                    for i in (0, 1))
            tok = torch.arange(length, device="cuda")
            see = tok <= length - n + torch.arange(n, device="cuda")[:, None]
            see = see.expand(H, n, length)
            if selected is not None:
                ids = selected[at:at + n].transpose(0, 1).long()  # [H, n, budget]
                ok = (ids >= 0) & (ids < len(pages))
                held = torch.zeros((H, n, len(pages) + 1), dtype=torch.bool, device="cuda")
                held.scatter_(2, torch.where(ok, ids, len(pages)), True)
                see = see & held[:, :, tok // T]
            q = self.q[at:at + n].double().view(n, H, G, D).permute(1, 0, 2, 3)
            x = torch.matmul(q.reshape(H, n * G, D), k.transpose(1, 2).contiguous())
            x = x.view(H, n, G, length) * D ** -0.5
            x = x.masked_fill(~see[:, :, None], -math.inf)
            w = torch.softmax(x, -1).nan_to_num(0.0).view(H, n * G, length)
            for y, u in ((o, v), (a, v.abs())):
                y[at:at + n] = torch.matmul(w, u).view(H, n, G, D).permute(1, 0, 2, 3).reshape(
                    n, H * G, D)
            lse[at:at + n] = torch.logsumexp(x, -1).permute(1, 0, 2).reshape(n, H * G)
        return o, a, lse

    def attend(self, batch=None, **kw):
        out = torch.full_like(self.q, math.nan)
        lse = torch.full((self.n_rows, self.H * self.G), math.nan, device="cuda")
        self.cache.attend(0, self.batch if batch is None else batch, self.q, out, lse=lse, **kw)
        return out, lse

    def check(self, got, weights, selected=None, rows=slice(None)):
        o, a, want = self.exact(selected)
        o, a, want = o[rows], a[rows], want[rows]
        out, lse = got[0][rows].double(), got[1][rows].double()
        assert torch.isfinite(out).all()
        bound = base.ULP[BF16] * o.abs() + (weights + 2.0 ** -14) * a + 2.0 ** -25
        assert ((out - o).abs() <= bound).all()
        empty = torch.isinf(want)
        assert torch.equal(empty, lse == -math.inf)
        assert ((lse - want)[~empty].abs() < 1e-4 * (1 + want[~empty].abs())).all()


# ---------------------------------------------------------- many units of work

def spread(lo, hi, n):
    return [lo + (i * 37) % (hi - lo + 1) for i in range(n)]


@pytest.mark.parametrize("n,heads,group,hi", [(4200, 1, 2, 700), (1100, 8, 1, 400), (530, 8, 2, 900)])
def test_more_sequences_and_heads_than_are_split(n, heads, group, hi):
    # a unit is a sequence and one or two heads; several steps each
    st = Step(spread(1, hi, n), [1] * n, heads, group, 64)
    st.check(st.attend(), FEW)


@pytest.mark.parametrize("n,rows,heads,budget,hi", [
    (1, 1100, 4, 20, 1500),   # one sequence, several steps
    (1, 4200, 1, 4, 4200),    # one step each
    (40, 30, 4, 20, 600),
    (600, 3, 4, 20, 400),     # more sequences than lanes, and ragged rows
])
def test_more_selected_rows_and_heads_than_are_split(n, rows, heads, budget, hi):
    rows = [rows] * n if n < 600 else [1 + i % rows for i in range(n)]
    lens = [max(a, r) for a, r in zip(spread(hi // 2, hi, n), rows)]
    st = Step(lens, rows, heads, 2, 64)
    sel = st.choose(budget)
    st.check(st.attend(selected=sel), FEW, selected=sel)


# ------------------------------------------------- calls that share a workspace

COUNTERS = 32 << 10  # bytes at a workspace's start that every call leaves zero


class OneWorkspace:
    """The C entry point on a workspace of the caller's."""

    def __init__(self, nbytes):
        self.memory = torch.full((nbytes,), 0x55, dtype=torch.uint8, device="cuda")
        self.memory[:COUNTERS] = 0

    def attend(self, st, window=0, selected=None):
        lib, ref = N.load(), C.byref
        out = torch.full_like(st.q, math.nan)
        lse = torch.full((st.n_rows, st.H * st.G), math.nan, device="cuda")
        rows = [N.Rows(t.data_ptr(), t.stride(0), t.stride(1)) for t in (st.q, out)]
        a = N.Attention(*rows, lse.data_ptr(), None if selected is None else selected.data_ptr(),
                        0 if selected is None else selected.shape[2], window, st.H * st.G, N.EA_BF16,
                        st.D ** -0.5, 0)
        b = st.batch.ref
        need = lib.ea_attend_workspace(st.cache.handle, b, ref(a))
        assert 0 <= need <= self.memory.numel()
        planes = N.CachePlanes(None, None, None)
        N.check("ea_attend", lib.ea_attend(st.cache.handle, ref(planes), 0, b, ref(a),
                                           self.memory.data_ptr() if need else None, need,
                                           api.current_stream()))
        torch.cuda.synchronize()
        assert not self.memory[:COUNTERS].any(), "counters are left zero by every call"
        return (out, lse), need


def test_chunks_decodes_and_selections_share_a_workspace():
    chunk = Step([6000], [40], 1, 4, 64)                 # the chunk kernel alone, in parts
    ragged = Step([3000, 2500, 40], [40, 1, 2], 1, 4, 64)  # both kernels
    decode = Step([5000, 333], [1, 1], 1, 4, 64)         # the split kernel alone, in parts
    sel = chunk.choose(40)
    ws = OneWorkspace(64 << 20)
    for order in ("cdsr", "rscd", "dcrs"):
        for what in order:
            st = {"c": chunk, "s": chunk, "d": decode, "r": ragged}[what]
            got, need = ws.attend(st, selected=sel if what == "s" else None)
            assert need > COUNTERS  # parts, or this shows nothing
            st.check(got, FEW if what in "ds" else MANY, selected=sel if what == "s" else None)


def test_a_batch_s_calls_of_two_shapes():
    # one batch, one stream: dense in the chunk kernel's parts, then the selection in the
    # split kernel's
    st = Step([9000], [100], 1, 8, 128)
    sel = st.choose(64)
    for _ in range(2):
        st.check(st.attend(), MANY)
        st.check(st.attend(selected=sel), FEW, selected=sel)


# ------------------------------------------------- selections in any order

@pytest.mark.parametrize("lead", [1, 2, 40, 300])
@pytest.mark.parametrize("page", [16, 5])
def test_blocks_that_follow_entries_that_are_none(lead, page):
    # more skipped entries before the blocks than the sequence has blocks
    st = Step([20, 70, 3, 150], [1, 2, 1, 3], 2, 3, 64, page=page)
    blocks = st.choose(4)
    none = torch.tensor([-1, 1 << 30, -7, 5000], dtype=torch.int32, device="cuda")
    sel = none.repeat(lead)[:lead].expand(st.n_rows, st.H, lead)
    sel = torch.cat([sel, blocks.flip(-1)], -1).contiguous()
    st.check(st.attend(selected=sel), FEW, selected=sel)


# ------------------------------------------------- captured calls

def test_a_captured_call_keeps_its_scratch_when_a_larger_one_comes():
    st = Step([9000], [100], 1, 8, 128)
    sel = st.choose(64)
    side = torch.cuda.Stream()
    out, lse = torch.empty_like(st.q), torch.empty((100, 8), device="cuda")

    def selected():
        st.cache.attend(0, st.batch, st.q, out, selected=sel, lse=lse)

    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        selected()
    side.synchronize()
    (small,) = (t.numel() for t in st.batch._scratch.values())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        selected()
    with torch.cuda.stream(side):
        st.check(st.attend(), MANY)  # needs more
        assert max(t.numel() for t in st.batch._scratch.values()) > small
        # what the allocator has of the first buffer's size
        others = [torch.zeros(small, dtype=torch.uint8, device="cuda") for _ in range(8)]
    for _ in range(3):
        out.fill_(math.nan)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        st.check((out, lse), FEW, selected=sel)
        with torch.cuda.stream(side):
            st.check(st.attend(), MANY)
        torch.cuda.synchronize()
        assert not any(bool(t.any()) for t in others)


def test_scratch_of_a_call_that_was_captured_first():
    # the clearing of a buffer that a capture made is recorded, not done
    st = Step([9000, 300], [1, 1], 2, 4, 128)
    out, lse = torch.empty_like(st.q), torch.empty((2, 8), device="cuda")
    sel, ids = st.choose(100), torch.empty((2, 2, 7), dtype=torch.int32, device="cuda")
    bounds = torch.randint(-9, 10, (1, 96, 2, 2, 128), dtype=torch.int8, device="cuda")
    cache = api.Cache(st.kv, 96, 1, 16, 2, 128, 2, bounds=bounds.sort(2).values.contiguous(),
                      bound_scales=torch.ones((1, 96, 2), device="cuda"))

    def step():
        cache.select_blocks(0, st.batch, st.q, ids)
        cache.attend(0, st.batch, st.q, out, selected=sel, lse=lse)
        cache.attend(0, st.batch, st.q, out, lse=lse)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        step()
    for t in st.batch._scratch.values():  # what fresh memory may hold
        t.fill_(0x55)
    torch.cuda.synchronize()
    out.fill_(math.nan)
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    st.check((out, lse), FEW)
    want = ids.clone()
    for _ in range(3):
        out.fill_(math.nan)
        ids.fill_(9)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        st.check((out, lse), FEW)
        assert torch.equal(ids, want)
        with torch.cuda.stream(side):
            step()
        torch.cuda.synchronize()
        st.check((out, lse), FEW)


# ------------------------------------------------- rows that only the device knows

@pytest.mark.parametrize("rows,most", [([5], 128), ([0], 128), ([1], 300), ([3, 0, 100], 100),
                                       ([2, 150, 60], 150)])
def test_fewer_rows_than_the_host_was_told(rows, most):
    # a step padded to its largest form: n_rows and max_rows are bounds
    lens = [900 + 70 * i for i in range(len(rows))]
    st = Step(lens, rows, 1, 8, 64, n_rows=most * len(rows), max_rows=most)
    there = slice(0, sum(rows))
    got = st.attend()
    st.check(got, MANY, rows=there)
    assert torch.isnan(got[0][sum(rows):]).all()  # rows of nobody are left as they are


# ------------------------------------------------- scales of blocks that some rows see

@pytest.mark.parametrize("rows,group,dim", [(70, 4, 64), (100, 2, 128), (140, 1, 80), (40, 2, 256)])
@pytest.mark.parametrize("page", [16, 5])
@pytest.mark.parametrize("window", [0, 20])
@pytest.mark.parametrize("far", [2.0 ** 12, 2.0 ** 60])
def test_a_large_scale_that_other_rows_of_a_chunk_see(rows, group, dim, page, window, far):
    # values of the last block, and of one in the middle, are far larger than
    # the others: rows that attend to neither lose nothing
    n = rows + 30
    st = base.Setup(kv_lens=[n, 90], rows=[rows, 3], heads=2, group=group, dim=dim, page=page,
                    fp8=True)
    for token in (n - 1, n - rows // 2):
        st.scales[st.layer, int(st.table[0, token // page]), 1] *= far
    st.d_scales.copy_(st.scales.cuda())
    q = st.rand(2 * group)
    out = torch.full_like(q, math.nan, device="cuda")
    lse = torch.empty((st.n_rows, 2 * group), device="cuda")
    st.handle.attend(st.layer, st.batch, q.cuda(), out, window=window, lse=lse)
    base.check_attention(st, q, out, lse, st.D ** -0.5, 2.0 ** -11, window=window)


# ------------------------------------------------- appends without queries

def test_an_append_without_queries_asks_nothing_of_their_number():
    lib, ref = N.load(), C.byref
    st = Step([40], [20], 2, 2, 64)
    k, v = (torch.randn((20, 2, 64), generator=st.g).to(BF16).cuda() for _ in range(2))
    rows = [N.Rows(t.data_ptr(), t.stride(0), t.stride(1)) for t in (k, v)]
    a = N.Append(*rows)
    a.q_heads, a.dtype = 0x7FFFFFFF, N.EA_BF16  # q.data is NULL
    st.table[0] = torch.arange(3, dtype=torch.int32)
    N.check("ea_append_kv", lib.ea_append_kv(st.cache.handle, ref(N.CachePlanes(None, None, None)), 0,
                                             st.batch.ref, ref(a), api.current_stream()))
    torch.cuda.synchronize()
    got = st.kv[0, :3].transpose(0, 1).reshape(2, 48, 2, 64)[:, 20:40]
    assert torch.equal(got[0], k) and torch.equal(got[1], v)


# ------------------------------------------------- selections of many blocks

@pytest.mark.parametrize("blocks,budget,first,last", [
    (1024, 100, 1, 1), (1025, 1000, 1, 2), (4096, 64, 0, 0), (4097, 300, 2, 1), (16384, 77, 1, 1),
    (16385, 5000, 1, 1), (65536, 128, 1, 1)])
@pytest.mark.parametrize("spread", [100, 2])  # few values: many ties
def test_selections_of_many_blocks(blocks, budget, first, last, spread):
    need_gpu()
    g = torch.Generator().manual_seed(blocks + spread)
    H, G, D = 2, 3, 24
    lens = [blocks, blocks - 3, min(blocks, budget + 1), max(1, budget // 2)]
    P = 500
    kv = torch.zeros((1, P, 2, 1, H, D), dtype=BF16, device="cuda")
    lo, hi = (torch.randint(0, spread + 1, (1, P, H, D), generator=g) * (1 if spread > 2 else 40)
              for _ in range(2))
    bounds = torch.stack([-lo, hi], 2).to(torch.int8).cuda()
    units = torch.exp2(torch.randint(-2, 3, (1, P, H), generator=g).float()).cuda()
    table = torch.randint(-1, P + 1, (len(lens), blocks), generator=g, dtype=torch.int32)
    cache = api.Cache(kv, P, 1, 1, H, D, 2, bounds=bounds, bound_scales=units)
    batch = api.Batch(table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), blocks)
    q = torch.randn((len(lens), H * G, D), generator=g).to(BF16)
    got = torch.full((len(lens), H, budget), 9, dtype=torch.int32, device="cuda")
    cache.select_blocks(0, batch, q.cuda(), got, first=first, last=last)

    b, u = bounds[0].cpu().double(), units[0].cpu().double()
    for s, held in enumerate(lens):
        ids = table[s, :held].long()
        there = (ids >= 0) & (ids < P)
        pages = torch.where(there, ids, 0)
        for h in range(H):
            best = torch.full((held,), -math.inf, dtype=torch.float64)
            for j in range(G):
                x = q[s, h * G + j].double()
                unit = base.power(float(x.abs().max()), 127.0)
                c = (x / unit).round()
                score = torch.maximum(c * b[pages, 0, h], c * b[pages, 1, h]).sum(-1)
                best = torch.maximum(best, score * unit * u[pages, h])
            # pages that are not there come last, forced blocks first
            best = torch.where(there, best, -math.inf)
            at = torch.arange(held)
            best = torch.where((at < first) | (at >= held - last), math.inf, best)
            order = torch.sort(best, descending=True, stable=True).indices[:budget]
            want = torch.full((budget,), -1, dtype=torch.int32)
            want[:len(order)] = order.sort().values.int()
            assert torch.equal(got[s, h].cpu(), want), (s, h)
