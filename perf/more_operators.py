"""Decoding of batches that share beginnings, decoding over selected pages, and the norm between a block's parts, as measurable cases with their plain forms.

A case is a dict of plain values; `kind` says which calls one pass makes:
  shared   attention of one new token per sequence over the paged cache, where sequences begin with the same pages (samples of a prompt, prompts behind
           one common text); `plan`: whether the pass also works out which pages are shared ("pass") or the program has that from the fork ("kept")
  pages    a step over selected pages: the bounds of the pages that the new tokens complete, the choice of pages by a score from the
           bounds, attention over the chosen pages
  bounds   the bounds (least and largest key, column by column) of all complete pages of a batch of new prompts
  norm     root-mean-square norm of rows with the residual added before, in the rows' type or in 8 bits with scales
Head counts and widths are those of the repository's LLaMA-7B-shaped layers (32 heads of 128, rows of 4096) and generic ones with shared heads; lengths are its
workloads' (77, 8 x 512, ragged 33 to 701) and generic long ones.

Layout of the cache: K[layer][page][kv head][page/16][d/8][16 tokens][8 of d], V[layer][page][kv head][page/8][d][8 tokens];
table[sequence][max_pages] holds page ids, -1 for none; bounds[layer][page][kv head][least, largest][d].
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
EPS = 1e-6
LEAST_SCALE = 2.0 ** -120


def listed():
    return [
        # interactive use: four samples of one short question, every head with its own keys
        {"name": "shared_4x77", "kind": "shared", "dtype": "bf16", "system": 0, "prompts": 1, "children": 4, "shortest": 77, "longest": 77, "new": 16,
         "heads": 32, "kv": 32, "d": 128, "page": 16, "window": 0, "sinks": 0, "plan": "kept"},
        # a long document asked about or sampled from 32 times at once, shared heads
        {"name": "shared_32x8192", "kind": "shared", "dtype": "bf16", "system": 0, "prompts": 1, "children": 32, "shortest": 8192, "longest": 8192,
         "new": 256, "heads": 32, "kv": 8, "d": 128, "page": 64, "window": 0, "sinks": 0, "plan": "kept"},
        # three samples of each of twelve prompts, all behind one system text; the step right after the fork
        {"name": "shared_12x3_system", "kind": "shared", "dtype": "bf16", "system": 512, "prompts": 12, "children": 3, "shortest": 33, "longest": 701,
         "new": 64, "heads": 32, "kv": 32, "d": 128, "page": 16, "window": 0, "sinks": 0, "plan": "pass"},
        # long conversations sampled twelve times each, cut to a window and four sinks
        {"name": "shared_8x12_window", "kind": "shared", "dtype": "bf16", "system": 100, "prompts": 8, "children": 12, "shortest": 500, "longest": 6000,
         "new": 300, "heads": 32, "kv": 8, "d": 128, "page": 32, "window": 1024, "sinks": 4, "plan": "kept"},
        # the small fp32 configuration: four short caches, every head with its own keys
        {"name": "pages_fp32_4", "kind": "pages", "dtype": "fp32", "seqs": 4, "shortest": 64, "longest": 700, "heads": 16, "kv": 16, "d": 64, "page": 16,
         "top": 8, "first": 1, "last": 2},
        # one very long document: 64 pages of 64 tokens of 1563
        {"name": "pages_1x100003", "kind": "pages", "dtype": "bf16", "seqs": 1, "shortest": 100003, "longest": 100003, "heads": 32, "kv": 8, "d": 128,
         "page": 64, "top": 64, "first": 1, "last": 4},
        # a loaded server with long conversations, a sixteenth to a half of each read
        {"name": "pages_32_ragged", "kind": "pages", "dtype": "bf16", "seqs": 32, "shortest": 2000, "longest": 16000, "heads": 32, "kv": 8, "d": 128,
         "page": 32, "top": 32, "first": 1, "last": 2},
        # the benchmark's prefill batch on its way into the cache
        {"name": "bounds_8x512", "kind": "bounds", "dtype": "bf16", "prompts": 8, "shortest": 512, "longest": 512, "heads": 32, "kv": 32, "d": 128,
         "page": 16},
        # one long document's pages after it was read (or moved by a compaction)
        {"name": "bounds_1x100003", "kind": "bounds", "dtype": "bf16", "prompts": 1, "shortest": 100003, "longest": 100003, "heads": 32, "kv": 8, "d": 128,
         "page": 64},
        # the next token of one sequence
        {"name": "norm_1x4096", "kind": "norm", "dtype": "bf16", "rows": 1, "d": 4096, "residual": True, "block": -1},
        # the benchmark's prefill batch, rows of the residual stream
        {"name": "norm_8x512", "kind": "norm", "dtype": "bf16", "rows": 4096, "d": 4096, "residual": True, "block": -1},
        # the same for products in 8 bits, a scale for every 128 columns
        {"name": "norm_8x512_e4m3", "kind": "norm", "dtype": "bf16", "rows": 4096, "d": 4096, "residual": True, "block": 128},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def _heads(rng):
    """(query heads, key heads): every head its own keys, groups of several sizes, one key head for all."""
    return rng.choice([(32, 32), (32, 8), (32, 8), (16, 16), (28, 4), (40, 8), (16, 1), (8, 2), (14, 14), (48, 1)])


def _span(rng, hi):
    longest = _log_int(rng, 1, hi)
    return {"shortest": longest if rng.random() < 0.3 else rng.randint(max(1, longest // 8), longest), "longest": longest}


def draw(rng):
    kind = rng.choice(["shared"] * 4 + ["pages"] * 4 + ["bounds"] + ["norm"] * 3)
    c = {"kind": kind, "dtype": "fp32" if rng.random() < 0.25 else "bf16"}
    if kind == "norm":
        d = 128 * _log_int(rng, 1, 128) if rng.random() < 0.5 else 8 * _log_int(rng, 1, 2000)
        rows = _log_int(rng, 1, max(1, min(20000, (1 << 24) // (d * _es(c) // 2))))
        blocks = [-1, -1, 0] + [b for b in (32, 64, 128, 256) if d % b == 0]
        return {**c, "rows": rows, "d": d, "residual": rng.random() < 0.7, "block": rng.choice(blocks)}
    heads, kv = _heads(rng)
    d, page = rng.choice([64, 96, 128, 128, 128, 160, 256]), rng.choice([16, 16, 32, 64, 128])
    c |= {"heads": heads, "kv": kv, "d": d, "page": page}
    if kind == "shared":
        prompts, children = _log_int(rng, 1, 24), _log_int(rng, 1, 32)
        # what the batch would read if nothing were shared: no more than the long document's samples
        most = min(20000, (1 << 27) * 2 // _es(c) // (prompts * children * kv * d) * 2)
        system = rng.choice([0, 0, _log_int(rng, 1, max(1, most // 4))])
        window = {"window": 0, "sinks": 0} if rng.random() < 0.6 else {"window": _log_int(rng, 16, 4096), "sinks": rng.choice([0, 4, 4, 21])}
        return {**c, "system": system, "prompts": prompts, "children": children, **_span(rng, max(1, most // 2)), "new": _log_int(rng, 1, max(1, most // 4)), **window,
                "plan": rng.choice(["kept", "pass"])}
    if kind == "pages":
        seqs = _log_int(rng, 1, 64)
        most = min(100000, (1 << 28) // (seqs * kv * d) * 2 // _es(c))
        first, last = rng.choice([0, 1, 1, 4]), rng.choice([1, 2, 2, 5])
        return {**c, "seqs": seqs, **_span(rng, max(16, most)), "top": first + last + _log_int(rng, 1, 120), "first": first, "last": last}
    prompts = _log_int(rng, 1, 32)
    most = (1 << 26) // (kv * d * _es(c) // 2)
    span = _span(rng, max(16, most // prompts))
    return {**c, "prompts": prompts, "shortest": page + span["shortest"], "longest": page + span["longest"]}    # a complete page at least


# ---------------------------------------------------------------------------------------------------- sizes
def _ragged(n, lo, hi, salt=0):
    """Lengths fixed by the case, so that its work is."""
    r = random.Random(n * 1000003 + lo * 1009 + hi + salt * 7919)
    return [r.randint(lo, hi) for _ in range(n)]


def _es(case):
    return 2 if case["dtype"] == "bf16" else 4


def _family(case):
    """Prompt lengths (common text included) and, row by row, (prompt, length of the sequence).  Rows stand sample by sample, not prompt by prompt."""
    n, k = case["prompts"], case["children"]
    prompts = [case["system"] + m for m in _ragged(n, case["shortest"], case["longest"])]
    grown = _ragged(n * k, 1, case["new"], 1)
    return prompts, [(i % n, prompts[i % n] + grown[i]) for i in range(n * k)]


def _seen(i, window, sinks):
    """Number of tokens that the token at position i sees."""
    if not window or i + 1 <= window:
        return i + 1
    return window + min(sinks, i + 1 - window)


def _begins(n, c):
    """First position of the last token's window."""
    return max(0, n - c["window"]) if c["window"] else 0


def _union(spans, a, b):
    """Positions of [a, b) in any of the spans."""
    held, at = 0, a
    for x, y in sorted(spans):
        x, y = max(x, at), min(y, b)
        if y > x:
            held, at = held + y - x, y
    return held


def _distinct(case):
    """Tokens that some row sees, shared ones once: (distinct, seen by all rows together)."""
    page, (prompts, rows) = case["page"], _family(case)
    spans = [(p, [(_begins(n, case), n), (0, min(case["sinks"], _begins(n, case)))]) for p, n in rows]
    common = case["system"] // page * page
    total = _union([x for _, s in spans for x in s], 0, common)
    for p, m in enumerate(prompts):
        total += _union([x for q, s in spans if q == p for x in s], common, m // page * page)
    for (p, n), (_, s) in zip(rows, spans):
        total += _union(s, prompts[p] // page * page, n)
    return total, sum(_seen(n - 1, case["window"], case["sinks"]) for _, n in rows)


def _chosen(case, n):
    """(pages of a sequence of n tokens, scored pages, tokens of the chosen ones about)."""
    cols = -(-n // case["page"])
    if cols <= case["top"]:
        return cols, 0, n
    last = n - (cols - 1) * case["page"]
    return cols, cols - case["first"] - case["last"], (case["top"] - 1) * case["page"] + last


def work(case):
    es = _es(case)
    if case["kind"] == "norm":
        n = case["rows"] * case["d"]
        out = n * es if case["block"] < 0 else n + 4 * case["rows"] * (case["d"] // (case["block"] or case["d"]))
        return {"bytes": n * es * (3 if case["residual"] else 1) + out + 4 * case["d"], "flops": 5 * n}
    row, heads = case["kv"] * case["d"] * es, case["heads"]
    if case["kind"] == "shared":
        distinct, seen = _distinct(case)
        rows = case["prompts"] * case["children"]
        return {"bytes": 2 * distinct * row + rows * heads * (2 * case["d"] * es + 4), "flops": 4 * case["d"] * heads * seen}
    if case["kind"] == "pages":
        sizes = [_chosen(case, n) for n in _ragged(case["seqs"], case["shortest"], case["longest"])]
        scored, tokens = sum(s for _, s, _ in sizes), sum(t for _, _, t in sizes)
        done = sum(n % case["page"] == 0 for n in _ragged(case["seqs"], case["shortest"], case["longest"]))
        return {"bytes": 2 * (scored + tokens + done) * row + done * case["page"] * row + case["seqs"] * (heads * (2 * case["d"] * es + 4) + 4 * case["kv"] * case["top"]),
                "flops": 4 * case["d"] * (heads * tokens + case["kv"] * scored)}
    pages = sum(n // case["page"] for n in _ragged(case["prompts"], case["shortest"], case["longest"]))
    return {"bytes": max(1, pages) * row * (case["page"] + 2), "flops": 2 * pages * case["page"] * case["kv"] * case["d"]}


# ---------------------------------------------------------------------------------------------------- inputs
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _randn(gen, shape, dtype, scale=1.0):
    x = torch.randn(shape, generator=gen, device=DEV, dtype=dtype)
    return x.mul_(scale) if scale != 1.0 else x


def _table(rows):
    t = torch.full((len(rows), max(map(len, rows))), -1, dtype=torch.int32)
    for s, ids in enumerate(rows):
        t[s, :len(ids)] = torch.tensor(ids, dtype=torch.int32)
    return t.to(DEV)


def _shuffled(counts):
    """Page ids of sequences that grew together, by the case alone."""
    total = sum(counts)
    ids = list(range(total))
    random.Random(total * 31 + len(counts)).shuffle(ids)
    got, at = [], 0
    for c in counts:
        got.append(ids[at:at + c])
        at += c
    return got, total


def _cache(case, gen, rows, total, lens):
    kv, d, page, dt = case["kv"], case["d"], case["page"], _dtype(case)
    return {"K": _randn(gen, (1, total, kv, page // 16, d // 8, 16, 8), dt), "V": _randn(gen, (1, total, kv, page // 8, d, 8), dt), "table": _table(rows),
            "len": torch.tensor(lens, dtype=torch.int32, device=DEV)}


def _least_largest(K):
    """Bounds of pages K [..., page/16, d/8, 16, 8] -> [..., 2, d]."""
    return torch.stack([K.amin((-4, -2)), K.amax((-4, -2))], -3).flatten(-2)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    kind, dt = case["kind"], _dtype(case)
    st = {"case": dict(case)}
    if kind == "norm":
        shape = (case["rows"], case["d"])
        st["x"] = _randn(gen, shape, dt)
        st["weight"] = _randn(gen, (case["d"],), dt, 0.1).add_(1.0)
        if case["residual"]:                                       # a stream that has grown over the layers, a few columns far larger
            st["residual"] = _randn(gen, shape, dt, 4.0)
            st["residual"][:, ::max(1, case["d"] // 5)] *= 20
        return st
    page = case["page"]
    if kind == "shared":
        prompts, family = _family(case)
        common = case["system"] // page
        own_cols = [-(-n // page) - prompts[p] // page for p, n in family]
        got, total = _shuffled([common] + [m // page - common for m in prompts] + own_cols)
        rows = []
        for r, (p, n) in enumerate(family):
            row = got[0] + got[1 + p] + got[1 + len(prompts) + r]
            if case["window"]:                                     # what no later token sees was given up
                row = [-1 if c * page >= case["sinks"] and (c + 1) * page <= n - case["window"] + 1 else i for c, i in enumerate(row)]
            rows.append(row)
        st |= _cache(case, gen, rows, total, [n for _, n in family])
        st["q"] = _randn(gen, (len(family), case["heads"], case["d"]), dt, 2.0)
        return st
    n = case["seqs"] if kind == "pages" else case["prompts"]
    lens = _ragged(n, case["shortest"], case["longest"])
    got, total = _shuffled([-(-m // page) for m in lens])
    st |= _cache(case, gen, got, total, lens)
    st["bounds"] = torch.zeros((1, total, case["kv"], 2, case["d"]), dtype=dt, device=DEV)
    if kind == "pages":
        st["q"] = _randn(gen, (n, case["heads"], case["d"]), dt, 2.0)
        # the keys of a page lie near each other, some pages nearer to the query than others
        st["K"] += _randn(gen, (1, total, case["kv"], 1, case["d"] // 8, 1, 8), dt)
        # complete before the new token came
        before = torch.tensor([i for ids, m in zip(got, lens) for i in ids[:(m - 1) // page]], dtype=torch.long, device=DEV)
        st["bounds"][0, before] = _least_largest(st["K"][0, before])
    else:
        st["off"] = torch.tensor([sum(lens[:p]) for p in range(n + 1)], dtype=torch.int32, device=DEV)
    return st


# ---------------------------------------------------------------------------------------------------- the framework's calls
def _run_own(st):
    """The state also holds what a program keeps beside its data: the cache's handle, scratch memory, outputs, the plan."""
    import paper_2605_08568_amd as pa
    c = st["case"]
    if c["kind"] == "norm":
        x = st["x"]
        if "out" not in st:
            st["sum"] = torch.empty_like(x) if c["residual"] else None
            st["out"] = torch.empty_like(x, dtype=x.dtype if c["block"] < 0 else torch.float8_e4m3fn)
            st["scales"] = None if c["block"] < 0 else torch.empty((c["rows"], c["d"] // (c["block"] or c["d"])), device=DEV)
        pa.rmsnorm(x, st["weight"], EPS, residual=st.get("residual"), residual_out=st["sum"], out=st["out"], scales=st["scales"])
        return st["out"], st["scales"], st["sum"]
    if "handle" not in st:
        st["handle"] = pa.KV(st["K"], st["V"], st["table"], st["len"])
    kv = st["handle"]
    if c["kind"] == "shared":
        if "ws" not in st:
            st["ws"] = pa.attend_shared_workspace(kv, c["heads"], st["q"].shape[0])
        if "shares" not in st:
            st["shares"] = pa.shared_plan(kv, c["heads"], st["q"].shape[0], window=c["window"], sinks=c["sinks"])
        elif c["plan"] == "pass":
            pa.shared_plan(kv, c["heads"], st["q"].shape[0], window=c["window"], sinks=c["sinks"], plan=st["shares"])
        return pa.attend_shared(kv, 0, st["q"], st["shares"], window=c["window"], sinks=c["sinks"], with_lse=True, workspace=st["ws"])
    if c["kind"] == "bounds":
        pa.kv_bounds(kv, st["bounds"], 0, st["off"])
        return st["bounds"]
    if "ws" not in st:
        st["ws"] = pa.select_pages_workspace(kv, c["heads"], c["seqs"]), pa.attend_pages_workspace(kv, c["heads"], c["seqs"], c["top"])
    pa.kv_bounds(kv, st["bounds"], 0)
    chosen = pa.select_pages(kv, 0, st["bounds"], st["q"], c["top"], first=c["first"], last=c["last"], workspace=st["ws"][0])
    return (st["bounds"], chosen, *pa.attend_pages(kv, 0, st["q"], chosen, with_lse=True, workspace=st["ws"][1]))


# ---------------------------------------------------------------------------------------------------- the plain forms
def _tokens(K, V):
    """Pages [a][b][pages][page/16][d/8][16][8] and [a][b][pages][page/8][d][8] -> tokens [a][b][token][d] in 32 bits."""
    a, b, n, pb, d8 = K.shape[:5]
    k = K.transpose(4, 5).reshape(a, b, n * pb * 16, d8 * 8).float()
    return k, V.transpose(4, 5).reshape(a, b, n * pb * 16, d8 * 8).float()


def _attend(q, k, v, seen, scale):
    """q [s][kv][rows][d]; seen [s][kv or 1][1][token] -> (o, lse)."""
    s = torch.matmul(q, k.transpose(2, 3)).mul_(scale).masked_fill_(~seen, -math.inf)
    m = s.amax(3, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = s.sub_(m).exp_()
    total = p.sum(3, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)
    return o, (m + total.log()).squeeze(3)


def _grouped(st, c):
    n, h, d = st["q"].shape
    return st["q"].float().view(n, c["kv"], h // c["kv"], d)


def _plain_shared(st, c):
    q = st["q"]
    t = st["table"].clamp(min=0).long()
    k, v = _tokens(st["K"][0][t].transpose(1, 2), st["V"][0][t].transpose(1, 2))
    j = torch.arange(k.shape[2], device=DEV)
    i = st["len"].long()[:, None] - 1
    seen = (j <= i) & (st["table"] >= 0).repeat_interleave(c["page"], 1)
    if c["window"]:
        seen &= (j > i - c["window"]) | (j < c["sinks"])
    o, lse = _attend(_grouped(st, c), k, v, seen[:, None, None], c["d"] ** -0.5)
    return o.reshape(q.shape).to(q.dtype), lse.reshape(q.shape[:2])


def _plain_bounds(st, c):
    """Bounds of all complete pages of the prompts, which are whole sequences here."""
    whole = (torch.arange(st["table"].shape[1], device=DEV) + 1) * c["page"] <= st["len"][:, None]
    ids = st["table"][whole].long()
    st["bounds"][0, ids] = _least_largest(st["K"][0, ids])
    return st["bounds"]


def _plain_pages(st, c):
    q, kv, page, table = st["q"], c["kv"], c["page"], st["table"]
    n, cols, length = q.shape[0], table.shape[1], st["len"].long()
    # pages that the new tokens complete
    newest = table.gather(1, ((length - 1) // page)[:, None])[:, 0].long()
    done = (length % page == 0)[:, None, None, None]
    st["bounds"][0, newest] = torch.where(done, _least_largest(st["K"][0, newest]), st["bounds"][0, newest])
    # scores, in 64 bits: the choice goes by values next to each other
    group = _grouped(st, c).double()
    up, down = group.clamp(min=0).sum(2)[:, None], group.clamp(max=0).sum(2)[:, None]
    bound = st["bounds"][0][table.clamp(min=0).long()].double()
    score = ((up * bound[:, :, :, 1]).sum(3) + (down * bound[:, :, :, 0]).sum(3)).transpose(1, 2)
    # always the first and the last pages, then by score, the lowest column first among equals
    column, held = torch.arange(cols, device=DEV), -(-length // page)[:, None]
    there = (column < held) & (table >= 0)
    rank = torch.where((column < c["first"]) | (column >= held - c["last"]), 0, 1)
    rank = torch.where(there, rank, 2)[:, None].expand(n, kv, cols)
    order = torch.sort(score, dim=2, descending=True, stable=True).indices
    order = order.gather(2, torch.sort(rank.gather(2, order), dim=2, stable=True).indices)[:, :, :c["top"]]
    order = torch.where(rank.gather(2, order) < 2, order, cols).sort(2).values
    chosen = torch.full((n, kv, c["top"]), -1, dtype=torch.int32, device=DEV)
    chosen[:, :, :order.shape[2]] = torch.where(order < cols, order, -1)
    # attention over them
    at = chosen.clamp(min=0).long()
    ids, head = table[:, None].expand(n, kv, cols).gather(2, at).long(), torch.arange(kv, device=DEV)[:, None]
    k, v = _tokens(st["K"][0][ids, head], st["V"][0][ids, head])
    j = (at * page)[..., None] + torch.arange(page, device=DEV)
    seen = ((chosen >= 0)[..., None] & (j < length[:, None, None, None])).flatten(2)
    o, lse = _attend(_grouped(st, c), k, v, seen[:, :, None], c["d"] ** -0.5)
    return st["bounds"], chosen, o.reshape(q.shape).to(q.dtype), lse.reshape(q.shape[:2])


def _plain_norm(st, c):
    x = st["x"].float()
    total = None
    if c["residual"]:
        x = x + st["residual"].float()
        total = x.to(st["x"].dtype)
    y = x * torch.rsqrt(x.square().mean(1, keepdim=True) + EPS) * st["weight"].float()
    if c["block"] < 0:
        return y.to(st["x"].dtype), None, total
    y = y.view(c["rows"], -1, c["block"] or c["d"])
    scales = (y.abs().amax(2) / 448).clamp(min=LEAST_SCALE)
    return (y / scales[..., None]).to(torch.float8_e4m3fn).view(x.shape), scales, total


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    return {"shared": _plain_shared, "pages": _plain_pages, "bounds": _plain_bounds, "norm": _plain_norm}[c["kind"]](state, c)


# ---------------------------------------------------------------------------------------------------- 64 bits
def _softmax64(q, k, v, scale):
    s = (q @ k.t()) * scale
    lse = torch.logsumexp(s, 1)
    return (s - lse[:, None]).exp() @ v, lse


def _page64(st, ids, head):
    """Keys and values of pages `ids` of one head, in order, [token][d]."""
    k, v = st["K"][0][ids, head].double(), st["V"][0][ids, head].double()
    return k.movedim(3, 2).flatten(3).flatten(0, 2), v.movedim(3, 2).flatten(0, 2)


def _exact_over(st, c, columns_of):
    """columns_of(s, head): the columns of the table that sequence s reads for a head, ascending."""
    q, page = st["q"], c["page"]
    g = c["heads"] // c["kv"]
    out, lse = torch.zeros(q.shape, dtype=torch.float64, device=DEV), torch.zeros(q.shape[:2], dtype=torch.float64, device=DEV)
    for s, n in enumerate(st["len"].tolist()):
        for head in range(c["kv"]):
            cols = columns_of(s, head)
            k, v = _page64(st, st["table"][s, cols].long(), head)
            j = (cols[:, None] * page + torch.arange(page, device=DEV)).flatten()
            seen = j < n
            if c.get("window"):
                seen &= (j >= n - c["window"]) | (j < c["sinks"])
            out[s, head * g:(head + 1) * g], lse[s, head * g:(head + 1) * g] = _softmax64(q[s, head * g:(head + 1) * g].double(), k[seen], v[seen], c["d"] ** -0.5)
    return out, lse


def _exact_bounds(st, c, ids):
    b = st["bounds"].double()
    for part in ids.split(4096):
        tokens = st["K"][0, part].double().movedim(4, 3).flatten(2, 3).flatten(3)
        b[0, part, :, 0], b[0, part, :, 1] = tokens.amin(2), tokens.amax(2)
    return b


def _exact_choice(st, c, b, s, head, n):
    """Columns that sequence s reads for a head: one product after another, then a sort of (score, column) pairs."""
    cols, g = -(-n // c["page"]), c["heads"] // c["kv"]
    ids = st["table"][s, :cols].long()
    least, largest = b[0, ids, head, 0], b[0, ids, head, 1]
    score = torch.zeros(cols, dtype=torch.float64, device=DEV)
    for h in range(head * g, (head + 1) * g):
        q = st["q"][s, h].double()
        score += torch.maximum(q * least, q * largest).sum(1)
    score = score.tolist()
    always = set(range(min(cols, c["first"]))) | set(range(max(0, cols - c["last"]), cols))
    others = sorted((i for i in range(cols) if i not in always), key=lambda i: (-score[i], i))
    return sorted(always | set(others[:max(0, c["top"] - len(always))]))


def exact(case, seed):
    c = dict(case)
    st = prepare(case, seed)
    if c["kind"] == "norm":
        s = st["x"].double() + (st["residual"].double() if c["residual"] else 0.0)
        y = s / (s.pow(2).sum(1, keepdim=True) / c["d"] + EPS).sqrt() * st["weight"].double()
        total = s if c["residual"] else None
        if c["block"] < 0:
            return y, None, total
        blocks = y.reshape(c["rows"], -1, c["block"] or c["d"])
        scales = blocks.abs().max(2).values / 448
        return (blocks / scales[..., None]).reshape(y.shape), scales, total
    if c["kind"] == "shared":
        if sum(n for _, n in _family(c)[1]) * c["kv"] * c["d"] > 1 << 31:
            return None
        return _exact_over(st, c, lambda s, head: torch.nonzero(st["table"][s] >= 0)[:, 0])
    lens = st["len"].tolist()
    if c["kind"] == "bounds":
        ids = [st["table"][s, :n // c["page"]] for s, n in enumerate(lens)]
        return _exact_bounds(st, c, torch.cat(ids).long())
    b = _exact_bounds(st, c, st["table"][[s for s, n in enumerate(lens) if n % c["page"] == 0], [n // c["page"] - 1 for n in lens if n % c["page"] == 0]].long())
    chosen = torch.full((len(lens), c["kv"], c["top"]), -1, dtype=torch.int32)
    for s, n in enumerate(lens):
        for head in range(c["kv"]):
            cols = _exact_choice(st, c, b, s, head, n)
            chosen[s, head, :len(cols)] = torch.tensor(cols, dtype=torch.int32)
    chosen = chosen.to(DEV)
    return (b, None, *_exact_over(st, c, lambda s, head: chosen[s, head][chosen[s, head] >= 0].long()))
