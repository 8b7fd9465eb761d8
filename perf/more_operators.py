"""Further cache operators of paper_2609_33762_amd as measurable cases: those of
a cache of latents, and those that rearrange a cache's pages.

Five kinds, each one call of a serving engine:

  latents  new tokens' latents and their shared key parts, rotated, written into
           the pages of a latent cache (16-bit, or fp8 with scales for each
           block), the queries' parts rotated beside them;
  latent   attention of the new tokens' absorbed queries over a latent cache;
  copy     pages copied to other pages of the cache in every layer, with their
           scales and bounds (a fork's copy of the block that it writes on);
  move     kept tokens of edited contexts moved together into other pages, keys
           turned to their new positions, fp8 blocks requantised, bounds made;
  shift    the same for a latent cache.

With `own` false `run` is the plain form, elementary torch operations in 32
bits; with `own` true it is the library's calls.
"""
import math

import torch

own = False

ACT = {"bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    wide = dict(latent=512, turn=64, page_tokens=16, act="bf16")
    moe = dict(heads=4, head_dim=128, page_tokens=16, act="bf16")
    tiny = dict(heads=2, head_dim=64, page_tokens=16, act="bf16")
    return [
        # a decode step of four agents with narrow latents, where launches and
        # latency are all there is
        dict(name="latents_tiny", kind="latents", fp8=False, seqs=4, rows_lo=1, rows_hi=1,
             kv_lo=512, kv_hi=512, q_heads=2, latent=128, turn=32, page_tokens=16, act="bf16"),
        # chunked prefill: ragged pieces of five prompts into fp8 pages
        dict(name="latents_chunks_fp8", kind="latents", fp8=True, seqs=5, rows_lo=301,
             rows_hi=2900, kv_lo=3001, kv_hi=16383, q_heads=16, **wide),
        # decode steps: the four agents'; the agent pool's ragged fp8 contexts
        # with a rank's 16 heads; one agent alone at the longest context with
        # all 128 heads, 16-bit
        dict(name="latent_tiny", kind="latent", fp8=False, seqs=4, rows_lo=1, rows_hi=1,
             kv_lo=512, kv_hi=512, q_heads=2, latent=128, turn=32, page_tokens=16, act="bf16"),
        dict(name="latent_agents_fp8", kind="latent", fp8=True, seqs=64, rows_lo=1, rows_hi=1,
             kv_lo=8192, kv_hi=65536, q_heads=16, **wide),
        dict(name="latent_long", kind="latent", fp8=False, seqs=1, rows_lo=1, rows_hi=1,
             kv_lo=65536, kv_hi=65536, q_heads=128, **wide),
        # drafted tokens checked: up to four rows of each of 24 sequences
        dict(name="latent_drafts", kind="latent", fp8=False, seqs=24, rows_lo=2, rows_hi=4,
             kv_lo=500, kv_hi=16000, q_heads=16, **wide),
        # a prompt's last 2,048 tokens behind a restored 24k-token prefix, on a
        # rank of 16 heads
        dict(name="latent_chunk", kind="latent", fp8=False, seqs=1, rows_lo=2048, rows_hi=2048,
             kv_lo=26624, kv_hi=26624, q_heads=16, **wide),
        # a fork of four agents copies the block that each writes on; a pool of
        # fp8 pages is drawn together after many contexts have ended
        dict(name="copy_fork", kind="copy", fp8=False, bounds=False, pages=4, layers=4, **tiny),
        dict(name="copy_pool_fp8", kind="copy", fp8=True, bounds=True, pages=4096, layers=12,
             **moe),
        # contexts from which old tool outputs were dropped: a short one; the
        # agent pool's in fp8 with bounds; latents, 16-bit
        dict(name="move_tiny", kind="move", fp8=False, bounds=False, seqs=1, kv_lo=200, kv_hi=200,
             kept=0.6, layers=2, **tiny),
        dict(name="move_agents_fp8", kind="move", fp8=True, bounds=True, seqs=16, kv_lo=8192,
             kv_hi=65536, kept=0.6, layers=2, **moe),
        dict(name="shift_agents", kind="shift", fp8=False, seqs=8, kv_lo=8192, kv_hi=65536,
             kept=0.6, layers=2, **wide),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["latents", "latent", "latent", "latent", "copy", "move", "shift"])
    c = dict(kind=kind, fp8=rng.random() < 0.5, act=rng.choice(["bf16", "bf16", "f16"]),
             page_tokens=rng.choice([16, 16, 16, 32, 64, 5]))
    if kind in ("copy", "move"):
        c.update(heads=rng.choice([1, 2, 3, 4, 8]), head_dim=rng.choice([64, 80, 96, 128, 128]),
                 bounds=rng.random() < 0.5)
        token = 2 * c["heads"] * c["head_dim"] * (1 if c["fp8"] else 2)
    else:
        c.update(latent=rng.choice([128, 256, 384, 512, 512, 512]), turn=rng.choice([32, 64, 64]))
        token = (c["latent"] + c["turn"]) * (1 if c["fp8"] else 2)
    if kind == "copy":
        c["layers"] = rng.choice([1, 2, 5, 12])
        c["pages"] = _log(rng, 1, 400_000_000 // (token * c["page_tokens"] * c["layers"]))
        return c
    if kind in ("move", "shift"):
        c["layers"] = rng.choice([1, 2, 4])
        tokens = _log(rng, 16, 500_000_000 // (token * c["layers"]))
        c["seqs"] = _log(rng, 1, min(tokens, 64))
        c["kept"] = rng.choice([0.2, 0.6, 0.9])
        c["kv_hi"] = min(65536, max(1, tokens // c["seqs"]))
        c["kv_lo"] = max(1, c["kv_hi"] // rng.choice([1, 3, 8]))
        return c
    c["q_heads"] = rng.choice([1, 2, 5, 8, 16, 16, 32, 128])
    if kind == "latents":
        rows = _log(rng, 1, 2_000_000 // (512 + 64 * c["q_heads"]))
        c["seqs"] = _log(rng, 1, min(rows, 256))
        c["rows_hi"] = max(1, rows // c["seqs"])
        c["kv_hi"] = max(c["rows_hi"], _log(rng, 1, 60000))
    else:
        tokens = _log(rng, 16, 2_000_000)
        c["seqs"] = _log(rng, 1, min(tokens, 128))
        c["kv_hi"] = min(65536, tokens // c["seqs"])
        c["rows_hi"] = 1
        if rng.random() < 0.6:
            most = 800_000_000 // (c["seqs"] * c["q_heads"] * c["kv_hi"])
            c["rows_hi"] = _log(rng, 1, max(1, min(c["kv_hi"], 2048, most)))
    c["rows_lo"] = max(1, c["rows_hi"] // rng.choice([1, 2, 9]))
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


def _moved(c):
    """(tokens kept, tokens before) of each sequence."""
    kv = _spread(c["kv_lo"], c["kv_hi"], c["seqs"], 0.754878)
    return [max(1, int(c["kept"] * k)) for k in kv], kv


def work(c):
    T, elem = c["page_tokens"], 1 if c["fp8"] else 2
    if c["kind"] == "copy":
        width = 2 * c["heads"] * c["head_dim"]
        piece = width * T * elem
        if c["fp8"]:
            piece += 2 * c["heads"] * 4
        if c["bounds"]:
            piece += width + c["heads"] * 4
        return {"bytes": 2 * c["pages"] * c["layers"] * piece + 8 * c["pages"], "flops": 0}
    if c["kind"] in ("move", "shift"):
        kept, _ = _moved(c)
        n, blocks = sum(kept), sum(-(-k // T) for k in kept)
        if c["kind"] == "move":
            width, turned, scales = 2 * c["heads"] * c["head_dim"], c["heads"] * c["head_dim"], \
                2 * c["heads"] * 4
        else:
            width, turned, scales = c["latent"] + c["turn"], c["turn"], 8
        byts = 2 * n * width * elem + (2 * blocks * scales if c["fp8"] else 0)
        if c.get("bounds"):
            byts += blocks * (width + 4 * c["heads"])
        return {"bytes": c["layers"] * byts + 4 * n, "flops": c["layers"] * n * turned * 3}
    rows, kv = _lengths(c)
    n, H, C, R = sum(rows), c["q_heads"], c["latent"], c["turn"]
    if c["kind"] == "latents":
        byts = n * (C + R) * (2 + elem) + 2 * n * H * R * 2 + n * R * 4
        if c["fp8"]:
            byts += sum(-(-((k - r) % T + r) // T) for r, k in zip(rows, kv)) * 8
        return {"bytes": byts, "flops": 3 * n * R * (H + 1)}
    seen = sum(r * (k - r) + r * (r + 1) // 2 for r, k in zip(rows, kv))
    byts = n * H * (2 * C + R) * 2 + sum(kv) * (C + R) * elem + sum(-(-k // T) for k in kv) * 4
    if c["fp8"]:
        byts += sum(-(-k // T) for k in kv) * 8
    return {"bytes": byts, "flops": 2 * (2 * C + R) * H * seen}


# ---------------------------------------------------------------- inputs

def _normal(shape, g, dtype, spread=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * spread).clamp(-448, 448).to(dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _angles(positions, dim):
    """Cosines and sines of each position, in 32 bits from 64."""
    inv = 10000.0 ** (-torch.arange(0, dim, 2, device="cuda", dtype=torch.float64) / dim)
    ang = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * inv
    return torch.cat([ang.cos(), ang.sin()], 1).float()


def _fill(st, g, shape):
    """A cache of numbers about one, and its scales in fp8."""
    c = st["c"]
    kind = torch.float8_e4m3fn if c["fp8"] else ACT[c["act"]]
    st["cache"] = torch.empty(shape, dtype=kind, device="cuda")
    flat = st["cache"].view(-1)
    step = 1 << 27  # in parts: the numbers are drawn in 32 bits
    for a in range(0, flat.numel(), step):
        b = min(flat.numel(), a + step)
        flat[a:b] = _normal((b - a,), g, kind, 60.0 if c["fp8"] else 1.0)
    st["scales"] = None
    if c["fp8"]:  # powers of two, as the library writes them; attention also reads other ones
        per = (2, c["heads"]) if "heads" in c else (2,)
        e = torch.rand((shape[0], shape[1], *per), generator=g, device="cuda") * 3 - 8
        st["scales"] = torch.exp2(e if c["kind"] == "latent" else e.round()).contiguous()


def _pages_for(counts, perm, at=0):
    """Tables [n][most] of pages perm[at:], zeros past a sequence's own."""
    table = torch.zeros((len(counts), max(max(counts), 1)), dtype=torch.int64)
    for i, n in enumerate(counts):
        table[i, :n] = torch.arange(at, at + n)
        at += n
    return perm[table.cuda()].to(torch.int32), at


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    T = c["page_tokens"]
    st = dict(c=c, layer=0, bounds=None, bound_scales=None)
    if c["kind"] == "copy":
        n, L = c["pages"], c["layers"]
        P = 2 * n + 3
        _fill(st, g, (L, P, 2, T, c["heads"], c["head_dim"]))
        perm = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
        st["src"], st["dst"] = perm[:n].contiguous(), perm[n:2 * n].contiguous()
    elif c["kind"] in ("move", "shift"):
        kept, kv = _moved(c)
        before, after = [-(-k // T) for k in kv], [-(-k // T) for k in kept]
        P, L = sum(before) + sum(after) + 2, c["layers"]
        one = (2, T, c["heads"], c["head_dim"]) if c["kind"] == "move" else (
            T, c["latent"] + c["turn"])
        _fill(st, g, (L, P, *one))
        perm = torch.randperm(P, generator=g, device="cuda")
        st["src_table"], at = _pages_for(before, perm)
        st["dst_table"], _ = _pages_for(after, perm, at)
        # runs of tokens are dropped, as whole tool outputs are
        lists = []
        for n, k in zip(kept, kv):
            run = max(1, k // 16)
            order = torch.rand((-(-k // run),), generator=g, device="cuda").argsort()
            rank = order[torch.arange(k, device="cuda") // run] * run + torch.arange(
                k, device="cuda") % run
            lists.append(rank.argsort()[:n].sort().values)
        st["tokens"] = torch.cat(lists).to(torch.int32)
        st["token_start"] = _ints([sum(kept[:i]) for i in range(len(kept) + 1)])
        st["max_tokens"], st["max_kv"] = max(kept), max(kv)
        st["rope"] = _angles(max(kv), c["head_dim"] if c["kind"] == "move" else c["turn"])
    else:
        rows, kv = _lengths(c)
        C, R = c["latent"], c["turn"]
        counts = [-(-k // T) for k in kv]
        P = sum(counts) + 5
        _fill(st, g, (2, P, T, C + R))
        st["layer"] = 1
        st["table"], _ = _pages_for(counts, torch.randperm(P, generator=g, device="cuda"))
        st["kv_len"], st["max_kv"] = _ints(kv), max(kv)
        st["row_start"] = _ints([sum(rows[:i]) for i in range(len(rows) + 1)])
        st["n_rows"], st["max_rows"] = sum(rows), max(rows)
        act = ACT[c["act"]]
        if c["kind"] == "latent":
            st["q"] = _normal((sum(rows), c["q_heads"], C + R), g, act)
            st["out"] = torch.empty((sum(rows), c["q_heads"], C), dtype=act, device="cuda")
        else:
            # one row of a token holds its latent and the key part side by side;
            # the queries' turning parts lie behind what does not turn
            both = _normal((sum(rows), 1, C + R), g, act)
            st["new"], st["key"] = both[..., :C], both[..., C:]
            st["q"] = _normal((sum(rows), c["q_heads"], 128 + R), g, act)[..., 128:]
            st["q_out"] = torch.empty(st["q"].shape, dtype=act, device="cuda")
            st["rope"] = _angles(max(kv), R)
    if c.get("bounds"):
        L, P = st["cache"].shape[:2]
        st["bounds"] = torch.randint(-127, 128, (L, P, 2, c["heads"], c["head_dim"]), generator=g,
                                     device="cuda", dtype=torch.int8)
        st["bound_scales"] = torch.rand((L, P, c["heads"]), generator=g, device="cuda")
    if own:
        _prepare_own(st)
    return st


def _prepare_own(st):
    from paper_2609_33762_amd import api
    c, (L, P) = st["c"], st["cache"].shape[:2]
    elem = 1 if c["fp8"] else 2
    if "heads" in c:
        st["handle"] = api.Cache(st["cache"], P, L, c["page_tokens"], c["heads"], c["head_dim"],
                                 elem, head_scales=st["scales"], bounds=st["bounds"],
                                 bound_scales=st["bound_scales"])
    else:
        st["handle"] = api.LatentCache(st["cache"], P, L, c["page_tokens"], c["latent"],
                                       c["turn"], elem, scales=st["scales"])
    if "kv_len" in st:
        st["batch"] = api.Batch(st["table"], st["kv_len"], st["max_kv"], st["row_start"],
                                st["n_rows"], st["max_rows"])


# ---------------------------------------------------------------- one pass

def _scale(c):
    return 1.0 / math.sqrt(128 + c["turn"])  # of a head's size before absorption


def run(st):
    c, kind = st["c"], st["c"]["kind"]
    if own:
        h = st["handle"]
        if kind == "latent":
            h.attend_latent(st["layer"], st["batch"], st["q"], st["out"], scale=_scale(c))
            return st["out"]
        if kind == "latents":
            h.append_latent(st["layer"], st["batch"], st["new"], st["key"], rope=st["rope"],
                            q=st["q"], q_out=st["q_out"])
        elif kind == "copy":
            h.copy_pages(st["src"], st["dst"])
        else:
            h.move_tokens(st["src_table"], st["dst_table"], st["tokens"], st["token_start"],
                          max_tokens=st["max_tokens"], max_kv=st["max_kv"], rope=st["rope"],
                          dtype=ACT[c["act"]])
        return _written(st)
    return {"latents": _latents, "latent": _latent, "copy": _copy, "move": _move,
            "shift": _move}[kind](st)


def _written(st):
    out = {k: st[k] for k in ("scales", "bounds", "bound_scales") if st[k] is not None}
    out["cache"] = st["cache"]
    if "q_out" in st:
        out = {k: v[st["layer"]] for k, v in out.items()}
        out["q"] = st["q_out"]
    return out


def _rows_of(st):
    """Sequence and position of each row."""
    start = st["row_start"].long()
    r = torch.arange(st["n_rows"], device="cuda")
    seq = torch.searchsorted(start[1:].contiguous(), r, right=True)
    return seq, st["kv_len"].long()[seq] - (start[seq + 1] - r)


def _power(amax, log2_top, mantissa_top):
    """The smallest power of two s >= 2^-126 with top * s >= amax, where
    top = 2 * mantissa_top * 2^log2_top."""
    m, e = torch.frexp(amax)
    e = torch.where(amax > 0, e - 1 - log2_top + (m > mantissa_top), -126).clamp(-126, 127)
    return ((e + 127).int() << 23).view(torch.float32)


def _turned(x, cos, sin):
    """x with its last dimension, halves as pairs, turned."""
    half = x.shape[-1] // 2
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _latents(st):
    c, layer, T, C, R = st["c"], st["layer"], st["c"]["page_tokens"], st["c"]["latent"], \
        st["c"]["turn"]
    seq, pos = _rows_of(st)
    cos, sin = st["rope"][pos][:, None, :R // 2], st["rope"][pos][:, None, R // 2:]
    st["q_out"].copy_(_turned(st["q"].float(), cos, sin))
    page, slot = st["table"][seq, pos // T].long(), pos % T
    new = torch.cat([st["new"].float(), _turned(st["key"].float(), cos, sin)], -1)[:, 0]
    if st["scales"] is None:
        st["cache"][layer][page, slot] = new.to(st["cache"].dtype)
        return _written(st)
    scales = st["scales"][layer]
    parts = torch.stack([new[:, :C].abs().amax(-1), new[:, C:].abs().amax(-1)], -1)
    need = _power(torch.zeros_like(scales).index_reduce_(0, page, parts, "amax"), 8, 0.875)
    # each sequence's first touched page may hold older tokens
    start = (st["kv_len"] - st["row_start"].diff()).long()
    ids = torch.arange(len(start), device="cuda")
    tail = st["table"][ids, (start // T).clamp(max=st["table"].shape[1] - 1)].long()
    older = torch.arange(T, device="cuda") < (start % T)[:, None]
    keep = older[:, :1]
    s0 = scales[tail]
    s1 = torch.where(keep, torch.maximum(s0, need[tail]), need[tail])
    part = (torch.arange(C + R, device="cuda") >= C).long()
    old = st["cache"][layer, tail]
    again = (old.float() * (s0 / s1)[:, part][:, None]).to(old.dtype)
    again = torch.where(older[..., None], again.view(torch.uint8), old.view(torch.uint8))
    st["cache"][layer].view(torch.uint8)[tail] = again
    touched = torch.zeros(scales.shape[0], dtype=torch.bool, device="cuda").index_fill_(
        0, page, True)
    scales.copy_(torch.where(touched[:, None], need.index_copy(0, tail, s1), scales))
    code = (new / scales[page][:, part]).to(st["cache"].dtype)
    st["cache"][layer].view(torch.uint8)[page, slot] = code.view(torch.uint8)
    return _written(st)


def _latent(st):
    c, C, R, H, T = st["c"], st["c"]["latent"], st["c"]["turn"], st["c"]["q_heads"], \
        st["c"]["page_tokens"]
    seq, pos = _rows_of(st)
    n, M = st["table"].shape[0], st["max_rows"]
    place = torch.arange(st["n_rows"], device="cuda") - st["row_start"].long()[seq]
    q = torch.zeros((n, M, H, C + R), device="cuda")
    q[seq, place] = st["q"].float()
    pages = st["table"].long()
    kv = pages.shape[1] * T
    k = st["cache"][st["layer"], pages].float()  # [n, pages, T, C + R]
    if st["scales"] is not None:
        part = (torch.arange(C + R, device="cuda") >= C).long()
        k = k * st["scales"][st["layer"], pages][:, :, None, part]
    k = k.view(n, kv, C + R)
    token = torch.arange(kv, device="cuda")
    there = token < st["kv_len"][:, None]
    k = torch.where(there[..., None], k, 0.0)
    score = torch.matmul(q.view(n, M * H, C + R), k.transpose(1, 2).contiguous()).mul_(_scale(c))
    at = torch.full((n, M), -1, device="cuda")
    at[seq, place] = pos
    mask = (token <= at[..., None]) & there[:, None]
    mask = mask[:, :, None].expand(n, M, H, kv).reshape(n, M * H, kv)
    score.masked_fill_(~mask, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, k[..., :C].contiguous()) / torch.where(total > 0, total, 1.0)
    return out.view(n, M, H, C)[seq, place].to(st["q"].dtype)


def _copy(st):
    src, dst = st["src"].long(), st["dst"].long()
    for t in (st["cache"], st["scales"], st["bounds"], st["bound_scales"]):
        if t is not None:
            raw = t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t
            raw[:, dst] = raw[:, src]
    return _written(st)


def _move(st):
    c, T = st["c"], st["c"]["page_tokens"]
    start, tokens = st["token_start"].long(), st["tokens"].long()
    i = torch.arange(len(tokens), device="cuda")
    seq = torch.searchsorted(start[1:].contiguous(), i, right=True)
    place = i - start[seq]
    src, dst = st["src_table"][seq, tokens // T].long(), st["dst_table"][seq, place // T].long()
    by = place - tokens  # the turn of a key
    dim = st["rope"].shape[1]
    cos = st["rope"][by.abs(), :dim // 2]
    sin = st["rope"][by.abs(), dim // 2:] * by.sign()[:, None]
    raw = st["cache"].view(torch.uint8) if c["fp8"] else st["cache"]
    places = raw.permute(1, 3, 0, 2, 4, 5) if c["kind"] == "move" else raw.permute(1, 2, 0, 3)
    x = places[src, tokens % T].view(st["cache"].dtype).float().transpose(0, 1)
    if c["kind"] == "move":  # [L, tokens, 2, H, D]
        if st["scales"] is not None:
            x = x * st["scales"][:, src][..., None]
        k = _turned(x[:, :, 0], cos[:, None], sin[:, None])
        x = torch.stack([k, x[:, :, 1]], 2)
        amax = x.abs().amax(-1)
    else:  # [L, tokens, C + R]
        C = c["latent"]
        part = (torch.arange(C + dim, device="cuda") >= C).long()
        if st["scales"] is not None:
            x = x * st["scales"][:, src][..., part]
        x = torch.cat([x[..., :C], _turned(x[..., C:], cos, sin)], -1)
        amax = torch.stack([x[..., :C].abs().amax(-1), x[..., C:].abs().amax(-1)], -1)
    if st["scales"] is not None:
        need = _power(torch.zeros_like(st["scales"]).index_reduce_(1, dst, amax, "amax"), 8, 0.875)
        st["scales"][:, dst] = need[:, dst]
        s = need[:, dst]
        x = x / (s[..., None] if c["kind"] == "move" else s[..., part])
    code = x.to(st["cache"].dtype)
    places[dst, place % T] = (code.view(torch.uint8) if c["fp8"] else code).transpose(0, 1)
    if st["bounds"] is not None:
        k = code[:, :, 0].float()
        if st["scales"] is not None:
            k = k * st["scales"][:, dst, 0][..., None]
        shape = st["bounds"][:, :, 0].shape
        lo = torch.full(shape, math.inf, device="cuda").index_reduce_(1, dst, k, "amin")
        hi = torch.full(shape, -math.inf, device="cuda").index_reduce_(1, dst, k, "amax")
        lo, hi = lo[:, dst], hi[:, dst]
        s = _power(torch.maximum(lo.abs(), hi.abs()).amax(-1), 6, 127 / 128)
        st["bound_scales"][:, dst] = s
        st["bounds"][:, dst] = torch.stack([(lo / s[..., None]).floor(),
                                            (hi / s[..., None]).ceil()], 2).to(torch.int8)
    return _written(st)


# ---------------------------------------------------------------- 64 bits

def exact(case, seed):
    """The outputs from the definitions, in 64 bits, sequence by sequence and
    block by block.  None in the place of whole numbers."""
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    return {"latents": _exact_latents, "latent": _exact_latent, "copy": _exact_copy,
            "move": _exact_move, "shift": _exact_move}[case["kind"]](st, case)


def _exact_latent(st, c):
    rows, kv = _lengths(c)
    H, C = c["q_heads"], c["latent"]
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    at = 0
    for s in range(c["seqs"]):
        pages = st["table"][s, :-(-kv[s] // c["page_tokens"])].long()
        x = st["cache"][st["layer"], pages].double()
        if c["fp8"]:
            x[..., :C] *= st["scales"][st["layer"], pages, 0].double()[:, None, None]
            x[..., C:] *= st["scales"][st["layer"], pages, 1].double()[:, None, None]
        x = x.flatten(0, 1)[:kv[s]].contiguous()
        tok = torch.arange(kv[s], device="cuda")
        step = max(1, 4096 // H)
        for a in range(0, rows[s], step):
            b = min(rows[s], a + step)
            pos = torch.arange(kv[s] - rows[s] + a, kv[s] - rows[s] + b, device="cuda")
            q = st["q"][at + a:at + b].double().flatten(0, 1)
            logits = (q @ x.T.contiguous() * _scale(c)).view(b - a, H, -1)
            w = torch.softmax(logits.masked_fill(tok > pos[:, None, None], -math.inf), -1)
            out[at + a:at + b] = (w.flatten(0, 1) @ x[:, :C].contiguous()).view(b - a, H, C)
        at += rows[s]
    return out


def _complex_turn(x, c, s):
    half = x.shape[-1] // 2
    z = torch.complex(x[..., :half], x[..., half:]) * torch.complex(c, s)
    return torch.cat([z.real, z.imag], -1)


def _top_power(x):
    """The scale of a block part's values."""
    top = float(x.abs().max()) / 448 if x.numel() else 0.0
    return 2.0 ** max(math.ceil(math.log2(top)), -126) if top > 0 else 2.0 ** -126


def _exact_latents(st, c):
    rows, kv = _lengths(c)
    T, C, R, layer = c["page_tokens"], c["latent"], c["turn"], st["layer"]
    cache = st["cache"][layer].double()
    scales = st["scales"][layer].double() if c["fp8"] else None
    rope = st["rope"].double()
    q = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    at = 0
    for s in range(c["seqs"]):
        start, mine = kv[s] - rows[s], slice(at, at + rows[s])
        co, si = rope[start:kv[s], :R // 2], rope[start:kv[s], R // 2:]
        q[mine] = _complex_turn(st["q"][mine].double(), co[:, None], si[:, None])
        new = torch.cat([st["new"][mine, 0].double(),
                         _complex_turn(st["key"][mine, 0].double(), co, si)], -1)
        table = st["table"][s].tolist()
        for b in range(start // T, (kv[s] - 1) // T + 1):
            page, i, j = table[b], max(start - b * T, 0), min(kv[s] - b * T, T)
            part = new[b * T + i - start:b * T + j - start]
            if not c["fp8"]:
                cache[page, i:j] = part
                continue
            for w, cut in ((0, slice(0, C)), (1, slice(C, C + R))):
                need = _top_power(part[:, cut])
                was = float(scales[page, w])
                if i and was >= need:
                    need = was
                elif i:
                    cache[page, :i, cut] = (cache[page, :i, cut] * (was / need)).to(
                        torch.float8_e4m3fn).double()
                scales[page, w] = need
                cache[page, i:j, cut] = (part[:, cut] / need).to(torch.float8_e4m3fn).double()
        at += rows[s]
    out = {"cache": cache, "q": q}
    if c["fp8"]:
        out["scales"] = scales
    return out


def _exact_copy(st, c):
    out = {"cache": st["cache"].double()}
    if c["fp8"]:
        out["scales"] = st["scales"].double()
    if c["bounds"]:
        out["bound_scales"] = st["bound_scales"].double()
    was = {k: v.clone() for k, v in out.items()}
    for a, b in zip(st["src"].tolist(), st["dst"].tolist()):
        for k, v in out.items():
            v[:, b] = was[k][:, a]
    if c["bounds"]:
        out["bounds"] = None
    return out


def _exact_move(st, c):
    kept, kv = _moved(c)
    T, L, latent = c["page_tokens"], c["layers"], c["kind"] == "shift"
    if sum(kept) > 120_000 or sum(kept) / T * L > 20_000:
        return None  # block by block
    cache = st["cache"].double()
    scales = st["scales"].double() if c["fp8"] else None
    rope = st["rope"].double()
    half = rope.shape[1] // 2
    if latent:
        parts = [(slice(0, c["latent"]), False), (slice(c["latent"], None), True)]
    else:
        parts = [(0, True), (1, False)]
    if not latent and c["bounds"]:
        bound_scales = st["bound_scales"].double()
    at = 0
    for s in range(c["seqs"]):
        tokens = st["tokens"][at:at + kept[s]].long()
        pages = st["src_table"][s].long()[tokens // T]
        turn = torch.arange(kept[s], device="cuda") - tokens
        co, si = rope[turn.abs(), :half], rope[turn.abs(), half:] * turn.sign()[:, None]
        dst = st["dst_table"][s].tolist()
        for w, (cut, turns) in enumerate(parts):
            if latent:
                x = cache[:, pages, tokens % T][..., cut]
                f = scales[:, pages, w][..., None] if c["fp8"] else 1.0
                x = _complex_turn(x * f, co, si) if turns else x * f
            else:
                x = cache[:, pages, cut, tokens % T]
                f = scales[:, pages, cut][..., None] if c["fp8"] else 1.0
                x = _complex_turn(x * f, co[:, None], si[:, None]) if turns else x * f
            for b in range(-(-kept[s] // T)):
                y = x[:, b * T:(b + 1) * T]
                n = y.shape[1]
                if c["fp8"]:
                    dims = (1, 2) if latent else (1, 3)
                    need = torch.exp2(torch.ceil(torch.log2(y.abs().amax(dims) / 448)))
                    scales[:, dst[b], w] = need
                    f = need[:, None, None] if latent else need[:, None, :, None]
                    y = (y / f).to(torch.float8_e4m3fn).double()
                if latent:
                    cache[:, dst[b], :n, cut] = y
                else:
                    cache[:, dst[b], cut, :n] = y
                    if c["bounds"] and w == 0:
                        v = y * f if c["fp8"] else y.to(ACT[c["act"]]).double()
                        bound_scales[:, dst[b]] = torch.exp2(torch.ceil(torch.log2(
                            v.abs().amax((1, 3)) / 127)))
        at += kept[s]
    out = {"cache": cache}
    if c["fp8"]:
        out["scales"] = scales
    if not latent and c["bounds"]:
        out["bounds"], out["bound_scales"] = None, bound_scales
    return out
