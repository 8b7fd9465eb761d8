"""The cache operators of paper_2609_33762_amd as measurable cases.

Three kinds, each the call (or the two calls) a serving step makes on one layer:

  append   new tokens' keys rotated and written, with their values, into the
           pages of a cache (16-bit, or fp8 with a scale for each block and
           head), the queries rotated beside them, the blocks' bounds brought
           up to date where the cache keeps them;
  attend   attention of the new tokens' queries over the paged cache;
  sparse   blocks selected for each query and KV head by their bounds, and
           attention over the selected blocks.

With `own` false `run` is the plain form, elementary torch operations in 32
bits; with `own` true it is the library's calls.
"""
import math

import torch

own = False

ACT = {"bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    tp8 = dict(heads=1, group=8, head_dim=128, page_tokens=16, act="bf16")
    moe = dict(tp8, heads=4)
    dense = dict(tp8, heads=8, group=5)
    tiny = dict(heads=2, group=2, head_dim=64, page_tokens=16, act="bf16")
    return [
        # a decode step of a tiny model: four sequences, where launches and
        # latency are all there is
        dict(name="append_tiny", kind="append", fp8=False, bounds=False, seqs=4, rows_lo=1,
             rows_hi=1, kv_lo=512, kv_hi=512, **tiny),
        # the agent pool's decode step: one new token of 64 agents into fp8
        # pages, their scales and bounds updated
        dict(name="append_agents_fp8", kind="append", fp8=True, bounds=True, seqs=64, rows_lo=1,
             rows_hi=1, kv_lo=8192, kv_hi=65536, **moe),
        # a dense model's chunked prefill: ragged pieces of five prompts, fp8
        dict(name="append_chunks_fp8", kind="append", fp8=True, bounds=True, seqs=5, rows_lo=301,
             rows_hi=2900, kv_lo=3001, kv_hi=16383, **dense),
        # a whole 32k-token refill of a 16-bit cache
        dict(name="append_refill", kind="append", fp8=False, bounds=False, seqs=1, rows_lo=32000,
             rows_hi=32000, kv_lo=32000, kv_hi=32000, **moe),
        # decode steps: the tiny model's; the agent pool's ragged fp8 contexts
        # on a rank of TP8; one agent alone at the longest context, 16-bit
        dict(name="attend_tiny", kind="attend", fp8=False, seqs=4, rows_lo=1, rows_hi=1,
             kv_lo=512, kv_hi=512, window=0, **tiny),
        dict(name="attend_agents_fp8", kind="attend", fp8=True, seqs=64, rows_lo=1, rows_hi=1,
             kv_lo=8192, kv_hi=65536, window=0, **tp8),
        dict(name="attend_long", kind="attend", fp8=False, seqs=1, rows_lo=1, rows_hi=1,
             kv_lo=65536, kv_hi=65536, window=0, **moe),
        # drafted tokens checked: up to four rows of each of 16 sequences
        dict(name="attend_drafts_fp8", kind="attend", fp8=True, seqs=16, rows_lo=2, rows_hi=4,
             kv_lo=500, kv_hi=16000, window=0, **dense),
        # a prompt's last 2,048 tokens behind a restored 24k-token prefix, and
        # ragged chunks of six prompts over fp8 on a rank of TP8
        dict(name="attend_chunk", kind="attend", fp8=False, seqs=1, rows_lo=2048, rows_hi=2048,
             kv_lo=26624, kv_hi=26624, window=0, **moe),
        dict(name="attend_chunks_fp8", kind="attend", fp8=True, seqs=6, rows_lo=97, rows_hi=1400,
             kv_lo=1500, kv_hi=16001, window=0, **tp8),
        # sparse decode: the agent pool over 128 blocks of each context, and
        # one agent at the longest context over 64
        dict(name="sparse_agents_fp8", kind="sparse", fp8=True, seqs=64, rows_lo=1, rows_hi=1,
             kv_lo=8192, kv_hi=65536, budget=128, **moe),
        dict(name="sparse_long", kind="sparse", fp8=False, seqs=1, rows_lo=1, rows_hi=1,
             kv_lo=65536, kv_hi=65536, budget=64, **tp8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    c = dict(kind=rng.choice(["append", "attend", "attend", "sparse"]),
             fp8=rng.random() < 0.6, act=rng.choice(["bf16", "bf16", "f16"]),
             heads=rng.choice([1, 2, 3, 4, 8]), group=rng.choice([1, 2, 4, 5, 7, 8, 16]),
             head_dim=rng.choice([64, 80, 96, 128, 128, 128]),
             page_tokens=rng.choice([16, 16, 16, 32, 64]))
    width = c["heads"] * c["head_dim"]
    if c["kind"] == "append":
        rows = _log(rng, 1, 8192 * 512 // max(512, width * (c["group"] + 2) // 8))
        c["seqs"] = _log(rng, 1, min(rows, 256))
        c["rows_hi"] = max(1, rows // c["seqs"])
        c["rows_lo"] = max(1, c["rows_hi"] // rng.choice([1, 2, 9]))
        c["kv_hi"] = max(c["rows_hi"], _log(rng, 1, 60000))
        c["bounds"] = rng.random() < 0.5
    else:
        # cached values of all sequences, queries times keys
        tokens = _log(rng, 16, 250_000_000 // (width * (c["group"] + 8) // 16))
        c["seqs"] = _log(rng, 1, min(tokens, 200))
        c["kv_hi"] = min(65536, tokens // c["seqs"])
        c["rows_hi"] = 1
        if c["kind"] == "attend" and rng.random() < 0.6:
            most = int(1.5e9 / (c["seqs"] * c["heads"] * c["group"] * c["kv_hi"]))
            c["rows_hi"] = _log(rng, 1, max(1, min(c["kv_hi"], 2048, most)))
        elif c["kind"] == "sparse":
            c["rows_hi"] = rng.choice([1, 1, 1, 2, 3])
        c["rows_lo"] = max(1, c["rows_hi"] // rng.choice([1, 2, 9]))
        if c["kind"] == "sparse":
            most = 150_000_000 // (c["seqs"] * c["rows_hi"] * width * c["page_tokens"])
            c["budget"] = _log(rng, 4, max(4, min(256, most)))
        else:
            c["window"] = rng.choice([0, 0, 0, _log(rng, 1, 8192)])
    c["kv_hi"] = max(c["kv_hi"], c["rows_hi"])
    c["kv_lo"] = max(1, c["kv_hi"] // rng.choice([1, 3, 8]))
    return c


# ---------------------------------------------------------------- the cases' shapes

def _spread(lo, hi, n, step):
    """n whole numbers over lo..hi, hi among them, the same for every seed."""
    return [hi - int((hi - lo) * ((i * step) % 1.0)) for i in range(n)]


def _lengths(c):
    """(new tokens, cached tokens with them) of each sequence."""
    rows = _spread(c["rows_lo"], c["rows_hi"], c["seqs"], 0.618034)
    kv = _spread(c["kv_lo"], c["kv_hi"], c["seqs"], 0.754878)
    return rows, [max(r, k) for r, k in zip(rows, kv)]


def _visible(c):
    """Pairs of a query row and a cached token it attends to."""
    rows, kv = _lengths(c)
    total = 0
    for n, length in zip(rows, kv):
        for pos in range(length - n, length):
            if c["kind"] == "sparse":
                T = c["page_tokens"]
                blocks = pos // T + 1
                total += pos + 1 if blocks <= c["budget"] else (c["budget"] - 1) * T + pos % T + 1
            else:
                total += min(pos + 1, c["window"]) if c["window"] else pos + 1
    return total


def work(c):
    rows, kv = _lengths(c)
    H, G, D, T = c["heads"], c["group"], c["head_dim"], c["page_tokens"]
    elem = 1 if c["fp8"] else 2
    n = sum(rows)
    if c["kind"] == "append":
        byts = n * (H * G + 2 * H) * D * 2 + n * H * G * D * 2 + n * 2 * H * D * elem + n * D * 4
        tail = [(length - r) % T for r, length in zip(rows, kv)]
        if c["fp8"]:
            byts += sum(-(-(t + r) // T) for t, r in zip(tail, rows)) * 2 * H * 4
        if c["bounds"]:  # the part of a block that was there is read for its bounds
            byts += sum(tail) * H * D * elem
            byts += sum(-(-(t + r) // T) for t, r in zip(tail, rows)) * H * (2 * D + 4)
        return {"bytes": byts, "flops": 6 * n * (H * G + H) * D}
    io = 2 * n * H * G * D * 2
    flops = 4 * D * H * G * _visible(c)
    if c["kind"] == "attend":
        seen = sum(min(length, c["window"] + r) if c["window"] else length
                   for r, length in zip(rows, kv))
        byts = io + seen * H * 2 * D * elem + sum(-(-k // T) for k in kv) * 4
        if c["fp8"]:
            byts += -(-seen // T) * H * 8
        return {"bytes": byts, "flops": flops}
    blocks = sum(-(-k // T) for k in kv)
    byts = io + blocks * (4 + H * (2 * D + 4)) + _visible(c) * H * 2 * D * elem
    byts += n * H * c["budget"] * 4
    if c["fp8"]:
        byts += -(-_visible(c) // T) * H * 8
    scored = sum((length - r + j) // T + 1 for r, length in zip(rows, kv) for j in range(r))
    return {"bytes": byts, "flops": flops + 2 * 2 * D * H * G * scored}


# ---------------------------------------------------------------- inputs

def _normal(shape, g, dtype, spread=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * spread).clamp(-448, 448).to(dtype)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    H, G, D, T = c["heads"], c["group"], c["head_dim"], c["page_tokens"]
    rows, kv = _lengths(c)
    n, n_rows, L, layer = c["seqs"], sum(rows), 2, 1
    act = ACT[c["act"]]
    width = -(-max(kv) // T)
    count = [-(-k // T) for k in kv]
    first = [(k - r) // T for r, k in zip(rows, kv)]  # first page the new tokens touch
    if c["kind"] == "append":
        # pages with new tokens are the sequence's own; the ones before lie in
        # a prefix that the sequences share
        fresh = sum(a - b for a, b in zip(count, first))
        shared = 64
    else:
        fresh, shared, first = sum(count), 0, [0] * n
    P = fresh + shared + 5
    perm = torch.randperm(P, generator=g, device="cuda", dtype=torch.int32)
    index = torch.full((n, width), -1, dtype=torch.int64)
    at = 0
    for i in range(n):
        if shared:
            index[i, :first[i]] = fresh + torch.arange(first[i]) % shared
        index[i, first[i]:count[i]] = torch.arange(at, at + count[i] - first[i])
        at += count[i] - first[i]
    index = index.cuda()
    table = torch.where(index >= 0, perm[index.clamp(min=0)], 0).to(torch.int32)
    st = dict(c=c, layer=layer, pages=P, table=table, max_rows=max(rows), max_kv=max(kv),
              kv_len=torch.tensor(kv, dtype=torch.int32, device="cuda"),
              row_start=torch.tensor([sum(rows[:i]) for i in range(n + 1)], dtype=torch.int32,
                                     device="cuda"),
              n_rows=n_rows, scales=None, bounds=None, bound_scales=None)
    kind = torch.float8_e4m3fn if c["fp8"] else act
    cache = torch.zeros((L, P, 2, T, H, D), dtype=kind, device="cuda")
    step = max(1, (1 << 27) // (2 * T * H * D))
    for a in range(0, P, step):  # in parts: the numbers are drawn in 32 bits
        b = min(P, a + step)
        cache[layer, a:b] = _normal((b - a, 2, T, H, D), g, kind, 60.0 if c["fp8"] else 1.0)
    st["cache"] = cache
    if c["fp8"]:  # values of about one; scales as the append writes them are powers of two,
        # another writer's are not
        e = torch.rand((L, P, 2, H), generator=g, device="cuda") * 3 - 8
        st["scales"] = torch.exp2(e if c["kind"] == "attend" else e.round()).contiguous()
    if c["kind"] == "append":
        # one row of a token holds its queries, keys and values side by side
        qkv = _normal((n_rows, H * G + 2 * H, D), g, act)
        st["q"], st["k"], st["v"] = qkv[:, :H * G], qkv[:, H * G:H * G + H], qkv[:, H * G + H:]
        st["q_out"] = torch.empty((n_rows, H * G, D), dtype=act, device="cuda")
        inv = 10000.0 ** (-torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D)
        ang = torch.arange(max(kv), device="cuda", dtype=torch.float64)[:, None] * inv
        st["rope"] = torch.cat([ang.cos(), ang.sin()], 1).float()
    else:
        st["q"] = _normal((n_rows, H * G, D), g, act)
        st["out"] = torch.empty_like(st["q"])
    if c["kind"] == "sparse" or c.get("bounds"):
        st["bounds"] = torch.zeros((L, P, 2, H, D), dtype=torch.int8, device="cuda")
        st["bound_scales"] = torch.ones((L, P, H), device="cuda")
    if c["kind"] == "sparse":  # in parts, as above
        for a in range(0, P, step):
            ids = torch.arange(a, min(P, a + step), device="cuda")
            lo, hi, s = _bounds_of(_values(st, ids, 0), None)
            st["bounds"][layer, ids, 0], st["bounds"][layer, ids, 1] = lo, hi
            st["bound_scales"][layer, ids] = s
        st["selected"] = torch.empty((n_rows, H, c["budget"]), dtype=torch.int32, device="cuda")
    if own:
        _prepare_own(st)
    return st


def _prepare_own(st):
    from paper_2609_33762_amd import api
    c = st["c"]
    st["handle"] = api.Cache(st["cache"], st["pages"], st["cache"].shape[0], c["page_tokens"],
                             c["heads"], c["head_dim"], 1 if c["fp8"] else 2,
                             head_scales=st["scales"], bounds=st["bounds"],
                             bound_scales=st["bound_scales"])
    st["batch"] = api.Batch(st["table"], st["kv_len"], st["max_kv"], st["row_start"],
                            st["n_rows"], st["max_rows"])


# ---------------------------------------------------------------- one pass

def run(st):
    kind = st["c"]["kind"]
    if own:
        h, b, layer = st["handle"], st["batch"], st["layer"]
        if kind == "append":
            h.append_kv(layer, b, st["k"], st["v"], rope=st["rope"], q=st["q"], q_out=st["q_out"])
            return _appended(st)
        if kind == "attend":
            h.attend(layer, b, st["q"], st["out"], window=st["c"]["window"])
            return st["out"]
        h.select_blocks(layer, b, st["q"], st["selected"], first=1, last=1)
        h.attend(layer, b, st["q"], st["out"], selected=st["selected"])
        return {"out": st["out"], "selected": st["selected"]}
    return {"append": _append, "attend": _attend, "sparse": _sparse}[kind](st)


def _appended(st):
    out = {"cache": st["cache"][st["layer"]], "q": st["q_out"]}
    if st["scales"] is not None:
        out["scales"] = st["scales"][st["layer"]]
    if st["bounds"] is not None:
        out["bounds"] = st["bounds"][st["layer"]]
        out["bound_scales"] = st["bound_scales"][st["layer"]]
    return out


def _rows_of(st):
    """Sequence and position of each row."""
    start = st["row_start"].long()
    r = torch.arange(st["n_rows"], device="cuda")
    seq = torch.searchsorted(start[1:].contiguous(), r, right=True)
    return seq, st["kv_len"].long()[seq] - (start[seq + 1] - r)


def _values(st, pages, kv):
    """Keys (0) or values (1) of pages as stored, [..., T, H, D] in 32 bits."""
    x = st["cache"][st["layer"], pages, kv].float()
    if st["scales"] is not None:
        x = x * st["scales"][st["layer"], pages, kv][..., None, :, None]
    return x


def _power(amax, log2_top, mantissa_top):
    """The smallest power of two s >= 2^-126 with top * s >= amax, where
    top = 2 * mantissa_top * 2^log2_top."""
    m, e = torch.frexp(amax)
    e = torch.where(amax > 0, e - 1 - log2_top + (m > mantissa_top), -126).clamp(-126, 127)
    return ((e + 127).int() << 23).view(torch.float32)


def _bounds_of(keys, there):
    """Whole-number bounds of blocks of keys [..., T, H, D]: lowest and
    highest, and the block's scale; `there` [..., T]: the tokens that count."""
    lo = hi = keys
    if there is not None:
        lo = torch.where(there[..., None, None], keys, math.inf)
        hi = torch.where(there[..., None, None], keys, -math.inf)
    lo, hi = lo.amin(-3), hi.amax(-3)
    s = _power(torch.maximum(lo.abs(), hi.abs()).amax(-1), 6, 127 / 128)
    return ((lo / s[..., None]).floor().to(torch.int8), (hi / s[..., None]).ceil().to(torch.int8),
            s)


def _rotated(x, rope, pos):
    half = x.shape[-1] // 2
    cos, sin = rope[pos][:, None, :half], rope[pos][:, None, half:]
    a, b = x[..., :half].float(), x[..., half:].float()
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _append(st):
    c, layer, T = st["c"], st["layer"], st["c"]["page_tokens"]
    seq, pos = _rows_of(st)
    st["q_out"].copy_(_rotated(st["q"], st["rope"], pos))
    page, slot = st["table"][seq, pos // T].long(), pos % T
    new = torch.stack([_rotated(st["k"], st["rope"], pos), st["v"].float()], 1)
    if st["scales"] is None:
        st["cache"][layer][page, :, slot] = new.to(st["cache"].dtype)
    else:
        scales = st["scales"][layer]
        P = scales.shape[0]
        amax = torch.zeros_like(scales).index_reduce_(0, page, new.abs().amax(-1), "amax")
        need = _power(amax, 8, 0.875)
        # each sequence's first touched page may hold older tokens
        start = (st["kv_len"] - st["row_start"].diff()).long()
        ids = torch.arange(len(start), device="cuda")
        tail = st["table"][ids, (start // T).clamp(max=st["table"].shape[1] - 1)].long()
        older = torch.arange(T, device="cuda") < (start % T)[:, None]
        keep = older[:, 0]
        s0 = scales[tail]
        s1 = torch.where(keep[:, None, None], torch.maximum(s0, need[tail]), need[tail])
        old = st["cache"][layer, tail]
        again = (old.float() * (s0 / s1)[:, :, None, :, None]).to(old.dtype)
        again = torch.where((older & keep[:, None])[:, None, :, None, None],
                            again.view(torch.uint8), old.view(torch.uint8))
        st["cache"][layer].view(torch.uint8)[tail] = again
        touched = torch.zeros(P, dtype=torch.bool, device="cuda").index_fill_(0, page, True)
        s = need.index_copy(0, tail, s1)
        scales.copy_(torch.where(touched[:, None, None], s, scales))
        code = (new / scales[page][..., None]).to(st["cache"].dtype)
        st["cache"][layer].view(torch.uint8)[page, :, slot] = code.view(torch.uint8)
    if st["bounds"] is not None:
        first = (st["kv_len"] - st["row_start"].diff()) // T
        most = (st["max_rows"] + T - 2) // T + 1
        blk = first[:, None] + torch.arange(most, device="cuda")
        held = st["kv_len"][:, None] - blk * T  # tokens from the block's start on
        pages = st["table"].gather(1, blk.clamp(max=st["table"].shape[1] - 1).long())
        pages = torch.where(held > 0, pages, pages[:, :1]).long()
        held = torch.where(held > 0, held, held[:, :1])
        there = torch.arange(T, device="cuda") < held[..., None]
        lo, hi, s = _bounds_of(_values(st, pages, 0), there)
        st["bounds"][layer][pages] = torch.stack([lo, hi], 2)
        st["bound_scales"][layer][pages] = s
    return _appended(st)


def _softmax_times(score, mask, v):
    """Softmax of `score` over the places that `mask` leaves, times v."""
    score = torch.where(mask, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / torch.where(total > 0, total, 1.0)


def _attend(st):
    c = st["c"]
    H, G, D, T = c["heads"], c["group"], c["head_dim"], c["page_tokens"]
    seq, pos = _rows_of(st)
    n, R = st["table"].shape[0], st["max_rows"]
    place = torch.arange(st["n_rows"], device="cuda") - st["row_start"].long()[seq]
    q = torch.zeros((n, R, H * G, D), device="cuda")
    q[seq, place] = st["q"].float()
    q = q.view(n, R, H, G, D).permute(0, 2, 1, 3, 4).reshape(n, H, R * G, D)
    pages = st["table"].long()
    kv = pages.shape[1] * T
    token = torch.arange(kv, device="cuda")
    there = token < st["kv_len"][:, None]
    k = _values(st, pages, 0).view(n, kv, H, D).permute(0, 2, 3, 1).contiguous()
    score = torch.matmul(q, k).mul_(1.0 / math.sqrt(D))
    del k
    v = _values(st, pages, 1).view(n, kv, H, D).permute(0, 2, 1, 3)
    v = torch.where(there[:, None, :, None], v, 0.0)
    at = torch.full((n, R), -1, device="cuda")
    at[seq, place] = pos
    mask = token <= at[..., None]
    if c["window"]:
        mask &= token > at[..., None] - c["window"]
    mask = (mask & there[:, None])[:, None, :, None].expand(n, 1, R, G, kv)
    out = _softmax_times(score, mask.reshape(n, 1, R * G, kv), v)
    out = out.view(n, H, R, G, D).permute(0, 2, 1, 3, 4).reshape(n, R, H * G, D)
    return out[seq, place].to(st["q"].dtype)


def _sparse(st):
    c = st["c"]
    H, G, D, T, layer, B = (c["heads"], c["group"], c["head_dim"], c["page_tokens"], st["layer"],
                            c["budget"])
    seq, pos = _rows_of(st)
    N = st["n_rows"]
    q = st["q"].float().view(N, H, G, D)
    sq = _power(q.abs().amax(-1), 6, 127 / 128)
    code = (q / sq[..., None]).round()
    pages = st["table"].long()
    W = pages.shape[1]
    bounds = st["bounds"][layer, pages].float()  # [n, W, 2, H, D]
    bounds = bounds.permute(0, 3, 2, 4, 1).reshape(-1, H, 2 * D, W)
    both = torch.cat([code.clamp(max=0), code.clamp(min=0)], -1)
    dot = torch.matmul(both, bounds[seq])  # [N, H, G, W], whole numbers below 2^24
    score = (dot * sq[..., None] * st["bound_scales"][layer, pages].permute(0, 2, 1)[seq][:, :, None]
             ).amax(2)
    held = (pos // T + 1)[:, None, None]
    block = torch.arange(W, device="cuda")
    score = torch.where((block < 1) | (block >= held - 1), math.inf, score)
    score = torch.where(block < held, score, -math.inf)
    top = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :B]
    if top.shape[-1] < B:
        top = torch.nn.functional.pad(top, (0, B - top.shape[-1]), value=W)
    top = torch.where(top < held, top, W + 1).sort(-1).values
    selected = torch.where(top < held, top, -1).to(torch.int32)
    page = pages[seq][:, None].expand(N, H, W).gather(2, selected.clamp(min=0).long())
    token = (selected[..., None] * T + torch.arange(T, device="cuda"))
    mask = ((token <= pos[:, None, None, None]) & (selected >= 0)[..., None]).view(N, H, 1, B * T)
    head = torch.arange(H, device="cuda")[:, None]

    def values(which):
        x = st["cache"][layer].permute(1, 0, 3, 2, 4)[which][page, head].float()  # [N, H, B, T, D]
        if st["scales"] is not None:
            x = x * st["scales"][layer][page, which, head][..., None, None]
        return x.view(N, H, B * T, D)

    k = values(0).transpose(2, 3).contiguous()
    score = torch.matmul(q, k) * (1.0 / math.sqrt(D))
    v = torch.where(mask.transpose(2, 3), values(1), 0.0)
    out = _softmax_times(score, mask, v)
    return {"out": out.view(N, H * G, D).to(st["q"].dtype), "selected": selected}


# ---------------------------------------------------------------- 64 bits

def exact(case, seed):
    """The outputs from the definitions, in 64 bits, sequence by sequence.
    Nothing for an appended cache's whole numbers and codes beyond the new
    tokens' own: they are returned as stored values."""
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    rows, kv = _lengths(case)
    if case["kind"] == "append":
        return _exact_append(st, rows, kv)
    H, G, D, T = case["heads"], case["group"], case["head_dim"], case["page_tokens"]
    out = torch.zeros((st["n_rows"], H * G, D), dtype=torch.float64, device="cuda")
    if case["kind"] == "sparse":
        picked = _sparse(st)["selected"].long()  # whole numbers; what is attended follows them
    scale, at = 1.0 / math.sqrt(D), 0
    for s in range(case["seqs"]):
        pages = st["table"][s, :-(-kv[s] // T)].long()
        for h in range(H):
            both = []
            for which in (0, 1):
                x = st["cache"][st["layer"], pages, which, :, h].double()
                if st["scales"] is not None:
                    x = x * st["scales"][st["layer"], pages, which, h].double()[:, None, None]
                both.append(x.reshape(-1, D)[:kv[s]])
            k, v = both
            tok = torch.arange(kv[s], device="cuda")
            for a in range(0, rows[s], 256):
                b = min(rows[s], a + 256)
                p = kv[s] - rows[s] + torch.arange(a, b, device="cuda")[:, None]
                see = tok <= p
                if case.get("window"):
                    see = see & (tok > p - case["window"])
                if case["kind"] == "sparse":
                    ids = picked[at + a:at + b, h]
                    blocks = torch.zeros((b - a, len(pages) + 1), dtype=torch.bool, device="cuda")
                    blocks.scatter_(1, torch.where(ids >= 0, ids, len(pages)), True)
                    see = see & blocks[:, tok // T]
                for j in range(G):
                    logits = st["q"][at + a:at + b, h * G + j].double() @ k.T.contiguous() * scale
                    w = torch.softmax(logits.masked_fill(~see, -math.inf), -1)
                    out[at + a:at + b, h * G + j] = w @ v
        at += rows[s]
    return {"out": out, "selected": None} if case["kind"] == "sparse" else out


def _exact_append(st, rows, kv):
    c, layer = st["c"], st["layer"]
    T, D, fp8 = c["page_tokens"], c["head_dim"], c["fp8"]
    inv = st["rope"].double()
    half = D // 2

    def turn(x, p):
        z = torch.complex(x[..., :half], x[..., half:]) * torch.complex(
            inv[p, :half], inv[p, half:])[:, None]
        return torch.cat([z.real, z.imag], -1)

    cache = st["cache"][layer].double()
    scales = st["scales"][layer].double() if fp8 else None
    q = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    at = 0
    for s in range(c["seqs"]):
        start = kv[s] - rows[s]
        p = torch.arange(start, kv[s], device="cuda")
        own_rows = slice(at, at + rows[s])
        q[own_rows] = turn(st["q"][own_rows].double(), p)
        new = torch.stack([turn(st["k"][own_rows].double(), p), st["v"][own_rows].double()], 1)
        if not fp8:
            cache[st["table"][s, p // T].long(), :, p % T] = new
        else:
            for b in range(start // T, (kv[s] - 1) // T + 1):
                page = int(st["table"][s, b])
                i, j = max(start - b * T, 0), min(kv[s] - b * T, T)
                part = new[b * T + i - start:b * T + j - start]
                need = torch.exp2(torch.ceil(torch.log2(part.abs().amax((0, 3)) / 448)))
                if i:
                    need = torch.maximum(need, scales[page])
                    old = cache[page, :, :i] * (scales[page] / need)[:, None, :, None]
                    cache[page, :, :i] = old.to(torch.float8_e4m3fn).double()
                scales[page] = need
                code = (part / need[..., None]).to(torch.float8_e4m3fn).double()
                cache[page, :, i:j] = code.transpose(0, 1)
        at += rows[s]
    out = {"cache": cache, "q": q}
    if fp8:
        out["scales"] = scales
    if c["bounds"]:
        out["bounds"] = None
        s0 = st["bound_scales"][layer].double()
        for s in range(c["seqs"]):
            for b in range((kv[s] - rows[s]) // T, (kv[s] - 1) // T + 1):
                page = int(st["table"][s, b])
                keys = cache[page, 0, :min(kv[s] - b * T, T)]
                top = keys.abs().amax((0, 2)) * (scales[page, 0] if fp8 else 1.0)
                s0[page] = torch.exp2(torch.ceil(torch.log2(top / 127)))
        out["bound_scales"] = s0
    return out
