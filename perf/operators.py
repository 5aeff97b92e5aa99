"""The paged key-value cache and the attention that reads it, as measurable cases with their plain forms.

A case is a dict of plain values; `kind` says which calls one pass makes:
  decode   attention of one new token per sequence over the paged cache
  prefill  causal attention of the new tokens of a batch of prompts over the paged cache, which holds them and what came before
  append   the new tokens' rows on their way: q and k rotated by position, k and v into their pages
  fork     a step of parallel sampling: last step's children are given up, every parent is forked, every child gets room for a token
  compact  the pages of a thinned-out cache moved together (the bookkeeping is put back first, as after a rollback)
Head counts and widths are those of the repository's LLaMA-7B-shaped layers (32 heads of 128) and generic ones with shared heads;
lengths are its workloads' (77, 8 x 512, ragged 32 to 2048) and generic long ones.

Layout of the cache: K[layer][page][kv head][page/16][d/8][16 tokens][8 of d], V[layer][page][kv head][page/8][d][8 tokens];
table[sequence][max_pages] holds page ids, -1 for none.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"


def listed():
    return [
        # interactive use: the first answer token after one short question, every head with its own keys
        {"name": "decode_1x77", "kind": "decode", "dtype": "bf16", "seqs": 1, "shortest": 77, "longest": 77, "heads": 32, "kv": 32,
         "d": 128, "page": 16, "window": 0, "sinks": 0},
        # one very long document, shared heads: the cache's length has to be spread over the whole card
        {"name": "decode_1x100003", "kind": "decode", "dtype": "bf16", "seqs": 1, "shortest": 100003, "longest": 100003, "heads": 32,
         "kv": 8, "d": 128, "page": 64, "window": 0, "sinks": 0},
        # a server's ordinary batch, lengths of the repository's ragged workload
        {"name": "decode_32_ragged", "kind": "decode", "dtype": "bf16", "seqs": 32, "shortest": 32, "longest": 2048, "heads": 32,
         "kv": 32, "d": 128, "page": 16, "window": 0, "sinks": 0},
        # a loaded server with long conversations cut to a window and four sinks; pages between them were given up
        {"name": "decode_192_window", "kind": "decode", "dtype": "bf16", "seqs": 192, "shortest": 500, "longest": 8000, "heads": 32,
         "kv": 8, "d": 128, "page": 32, "window": 1024, "sinks": 4},
        # the small fp32 configuration: four prompts of 64 tokens, 1024 columns
        {"name": "prefill_fp32_4x64", "kind": "prefill", "dtype": "fp32", "prompts": 4, "shortest": 64, "longest": 64, "past": 0,
         "heads": 16, "kv": 16, "d": 64, "page": 16, "window": 0, "sinks": 0},
        # the benchmark's prefill batch
        {"name": "prefill_8x512", "kind": "prefill", "dtype": "bf16", "prompts": 8, "shortest": 512, "longest": 512, "past": 0,
         "heads": 32, "kv": 32, "d": 128, "page": 16, "window": 0, "sinks": 0},
        # a ragged batch of later turns: new tokens over what the conversations hold already, window and sinks
        {"name": "prefill_20_ragged_window", "kind": "prefill", "dtype": "bf16", "prompts": 20, "shortest": 20, "longest": 701,
         "past": 4000, "heads": 32, "kv": 8, "d": 128, "page": 32, "window": 1024, "sinks": 4},
        # one long document read in one go, the largest product
        {"name": "prefill_1x8192", "kind": "prefill", "dtype": "bf16", "prompts": 1, "shortest": 8192, "longest": 8192, "past": 0,
         "heads": 32, "kv": 8, "d": 128, "page": 64, "window": 0, "sinks": 0},
        # one decode step's rows of the benchmark's batch of 32 sequences
        {"name": "append_32x1", "kind": "append", "dtype": "bf16", "prompts": 32, "shortest": 1, "longest": 1, "past": 2047, "heads": 32,
         "kv": 32, "d": 128, "page": 16},
        # the rows of the benchmark's prefill batch
        {"name": "append_8x512", "kind": "append", "dtype": "bf16", "prompts": 8, "shortest": 512, "longest": 512, "past": 0, "heads": 32,
         "kv": 32, "d": 128, "page": 16},
        # three samples of each of twelve prompts over eight layers: shared pages, one copied page per child and layer
        {"name": "fork_12x3", "kind": "fork", "dtype": "bf16", "layers": 8, "parents": 12, "children": 3, "shortest": 33, "longest": 701,
         "kv": 32, "d": 128, "page": 16},
        # half of 48 sequences ended: what is left moves to the front of the pool
        {"name": "compact_48", "kind": "compact", "dtype": "bf16", "layers": 8, "seqs": 48, "gone": 24, "shortest": 32, "longest": 512,
         "kv": 32, "d": 128, "page": 16},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def _heads(rng):
    """(query heads, key heads): every head its own keys, groups of several sizes, one key head for all."""
    return rng.choice([(32, 32), (32, 8), (32, 8), (16, 16), (28, 4), (40, 8), (16, 1), (8, 2), (14, 14)])


def _span(rng, hi):
    longest = _log_int(rng, 1, hi)
    return {"shortest": longest if rng.random() < 0.3 else rng.randint(max(1, longest // 8), longest), "longest": longest}


def _window(rng):
    return {"window": 0, "sinks": 0} if rng.random() < 0.5 else {"window": _log_int(rng, 16, 4096), "sinks": rng.choice([0, 4, 4, 21])}


def draw(rng):
    kind = rng.choice(["decode"] * 4 + ["prefill"] * 4 + ["append"] * 2 + ["fork", "compact"])
    heads, kv = _heads(rng)
    d = rng.choice([64, 128, 128, 128, 160, 256]) if kind != "append" else rng.choice([128, 128, 160])
    c = {"kind": kind, "dtype": "fp32" if rng.random() < 0.2 else "bf16"}
    page = rng.choice([16, 16, 32, 64, 128])
    if kind == "decode":
        seqs = _log_int(rng, 1, 256)
        most = min(100000, (1 << 27) // (seqs * kv * d))                  # half of the ragged batch's bytes at most
        return {**c, "seqs": seqs, **_span(rng, max(16, most)), "heads": heads, "kv": kv, "d": d, "page": page, **_window(rng)}
    if kind == "prefill":
        prompts = _log_int(rng, 1, 32)
        past = rng.choice([0, 0, _log_int(rng, 1, 8192 // prompts)])
        most, flops = 4096 // prompts, 5e11 if c["dtype"] == "bf16" else 5e10
        while 4 * heads * d * prompts * most * (past + most / 2) > flops:    # no more than the long document's work
            most = most * 3 // 4
        return {**c, "prompts": prompts, **_span(rng, max(1, most)), "past": past, "heads": heads, "kv": kv, "d": d, "page": page,
                **_window(rng)}
    if kind == "append":
        prompts = _log_int(rng, 1, 64)
        return {**c, "prompts": prompts, **_span(rng, 1600 // prompts), "past": _log_int(rng, 1, 2000), "heads": heads, "kv": kv, "d": d,
                "page": page}
    # the bytes of a page and their number no more than in the listed cases
    c |= {"layers": rng.choice([1, 2, 4, 8])}
    page = min(page, 64)
    while kv > 1 and kv * page * d * _es(c) > 32 * 16 * 128 * 2:
        kv //= 2
    if kind == "fork":
        parents = _log_int(rng, 1, 12)
        return {**c, "parents": parents, "children": rng.randint(1, 36 // parents if parents > 4 else 8), **_span(rng, 700), "kv": kv, "d": d,
                "page": page}
    seqs = _log_int(rng, 2, 48)
    return {**c, "seqs": seqs, "gone": rng.randint(1, seqs), **_span(rng, 500), "kv": kv, "d": d, "page": page}


# ---------------------------------------------------------------------------------------------------- sizes
def _ragged(case, n, lo, hi, salt=0):
    """Lengths fixed by the case, so that its work is."""
    r = random.Random(n * 1000003 + lo * 1009 + hi + salt * 7919)
    return [r.randint(lo, hi) for _ in range(n)]


def _new_and_past(case):
    n = case["prompts"]
    new = _ragged(case, n, case["shortest"], case["longest"])
    past = _ragged(case, n, case["past"] // 2, case["past"], 1) if case["past"] else [0] * n
    return new, past


def _es(case):
    return 2 if case["dtype"] == "bf16" else 4


def _seen(i, window, sinks):
    """Number of tokens that the token at position i sees."""
    if not window or i + 1 <= window:
        return i + 1
    return window + min(sinks, i + 1 - window)


def _moves(case):
    """What compaction moves: (live pages, pages moved), from the layout that _page_ids gives."""
    lens = _ragged(case, case["seqs"], case["shortest"], case["longest"])
    ids, total = _page_ids(case, lens)
    keep = _kept(case)
    live = [p for s in keep for p in ids[s]]
    return len(live), sum(p >= len(live) for p in live), total


def _page_ids(case, lens):
    """Page ids of sequences that grew together: shuffled, by the case alone."""
    counts = [-(-n // case["page"]) for n in lens]
    total = sum(counts)
    ids = list(range(total))
    random.Random(total * 31 + len(lens)).shuffle(ids)
    got, at = [], 0
    for c in counts:
        got.append(ids[at:at + c])
        at += c
    return got, total


def _kept(case):
    return sorted(random.Random(case["seqs"] * 17 + case["gone"]).sample(range(case["seqs"]), case["seqs"] - case["gone"]))


def work(case):
    es, kind = _es(case), case["kind"]
    if kind == "decode":
        seen = sum(_seen(n - 1, case["window"], case["sinks"]) for n in _ragged(case, case["seqs"], case["shortest"], case["longest"]))
        rows = case["seqs"] * case["heads"]
        return {"bytes": 2 * seen * case["kv"] * case["d"] * es + rows * (2 * case["d"] * es + 4),
                "flops": 4 * case["d"] * case["heads"] * seen}
    if kind == "prefill":
        new, past = _new_and_past(case)
        w, s = case["window"], case["sinks"]
        pairs = sum(_seen(i, w, s) for n, p in zip(new, past) for i in range(p, p + n))
        kept = 0
        for n, p in zip(new, past):
            first = max(0, p + 1 - w) if w else 0                            # what the first new token's window begins with
            kept += p + n - first + min(first, s)
        rows = sum(new) * case["heads"]
        return {"bytes": 2 * kept * case["kv"] * case["d"] * es + rows * (2 * case["d"] * es + 4), "flops": 4 * case["d"] * case["heads"] * pairs}
    if kind == "append":
        new, _ = _new_and_past(case)
        return {"bytes": 2 * sum(new) * (case["heads"] + 2 * case["kv"]) * case["d"] * es + sum(new) * case["d"] * 4,
                "flops": 3 * sum(new) * (case["heads"] + case["kv"]) * case["d"]}
    per_page = 2 * case["kv"] * case["page"] * case["d"] * es * case["layers"]
    if kind == "fork":
        lens = _ragged(case, case["parents"], case["shortest"], case["longest"])
        copied = case["children"] * sum(n % case["page"] != 0 for n in lens)
        entries = case["children"] * sum(-(-n // case["page"]) for n in lens)
        return {"bytes": 2 * copied * per_page + 4 * 4 * entries, "flops": 0}
    live, moved, total = _moves(case)
    return {"bytes": 2 * moved * per_page + 4 * (live + 2 * total), "flops": 0}


# ---------------------------------------------------------------------------------------------------- inputs
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _randn(gen, shape, dtype, scale=1.0):
    x = torch.randn(shape, generator=gen, device=DEV, dtype=dtype)
    return x.mul_(scale) if scale != 1.0 else x


def _pool(case, gen, n_pages, layers=1):
    kv, d, page = case["kv"], case["d"], case["page"]
    K = _randn(gen, (layers, n_pages, kv, page // 16, d // 8, 16, 8), _dtype(case))
    V = _randn(gen, (layers, n_pages, kv, page // 8, d, 8), _dtype(case))
    return K, V


def _free_words(refs):
    """Bit p of the words is set where page p has no user."""
    n = refs.numel()
    bits = torch.zeros(-(-n // 32) * 32, dtype=torch.int64, device=refs.device)
    bits[:n] = (refs == 0).long()
    w = (bits.view(-1, 32) << torch.arange(32, device=refs.device)).sum(1)
    return torch.where(w >= 2 ** 31, w - 2 ** 32, w).int()


def _uses(table, n_pages):
    """How many table entries hold each page."""
    refs = torch.zeros(n_pages, dtype=torch.int32, device=table.device)
    return refs.index_add_(0, table.clamp(min=0).flatten(), (table >= 0).int().flatten())


def _table(rows, max_pages):
    t = torch.full((len(rows), max_pages), -1, dtype=torch.int32)
    for s, ids in enumerate(rows):
        if len(ids):
            t[s, :len(ids)] = torch.tensor(ids, dtype=torch.int32)
    return t


def _cache_of(case, gen, lens, firsts):
    """Cache of one layer whose sequences hold lens tokens; pages wholly between the sinks and firsts[s] were given up."""
    page, w, s0 = case["page"], case.get("window", 0), case.get("sinks", 0)
    wanted = [[not w or c * page < s0 or (c + 1) * page > f for c in range(-(-n // page))] for n, f in zip(lens, firsts)]
    total = max(1, sum(map(sum, wanted)))
    ids = list(range(total))
    random.Random(total * 31 + len(lens)).shuffle(ids)
    rows, at = [], 0
    for keep in wanted:
        row = []
        for k in keep:
            row.append(ids[at] if k else -1)
            at += k
        rows.append(row)
    K, V = _pool(case, gen, total)
    return {"K": K, "V": V, "table": _table(rows, max(map(len, rows))).to(DEV), "len": torch.tensor(lens, dtype=torch.int32, device=DEV)}


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    kind, dt = case["kind"], _dtype(case)
    st = {"case": dict(case)}
    if kind == "decode":
        lens = _ragged(case, case["seqs"], case["shortest"], case["longest"])
        st |= _cache_of(case, gen, lens, [n - case["window"] for n in lens])
        st["q"] = _randn(gen, (case["seqs"], case["heads"], case["d"]), dt, 2.0)
        return st
    if kind in ("prefill", "append"):
        new, past = _new_and_past(case)
        st |= _cache_of(case, gen, [n + p for n, p in zip(new, past)], [p + 1 - case.get("window", 0) for p in past])
        off = [0]
        for n in new:
            off.append(off[-1] + n)
        rows = off[-1]
        st["off"] = torch.tensor(off, dtype=torch.int32, device=DEV)
        if kind == "prefill":
            st["q"] = _randn(gen, (rows, case["heads"], case["d"]), dt, 2.0)
            return st
        # one row of the fused q/k/v projection per token
        st["qkv"] = _randn(gen, (rows, case["heads"] + 2 * case["kv"], case["d"]), dt)
        n_pos, half = max(n + p for n, p in zip(new, past)), case["d"] // 2
        angle = torch.arange(n_pos, device=DEV, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)
        st["rope"] = torch.cat([angle.cos(), angle.sin()], 1).float()
        st["q_out"] = torch.empty((rows, case["heads"], case["d"]), dtype=dt, device=DEV)
        return st
    if kind == "fork":
        lens = _ragged(case, case["parents"], case["shortest"], case["longest"])
        ids, total = _page_ids(case, lens)
        children = case["parents"] * case["children"]
        n_pages, max_pages = total + children + 5, max(map(len, ids)) + 2
        st["K"], st["V"] = _pool(case, gen, n_pages, case["layers"])
        st["table"] = _table([[p + 1 for p in row] for row in ids] + [[]] * children, max_pages).to(DEV)
        st["len"] = torch.tensor(lens + [0] * children, dtype=torch.int32, device=DEV)
        st["refs"] = _uses(st["table"], n_pages)
        st["free"] = _free_words(st["refs"])
        dst = list(range(case["parents"], case["parents"] + children))
        st["src"] = torch.tensor([i % case["parents"] for i in range(children)], dtype=torch.int32, device=DEV)
        st["dst"] = torch.tensor(dst, dtype=torch.int32, device=DEV)
        st["keep"] = torch.tensor(lens + [0] * children, dtype=torch.int32, device=DEV)
        st["n_new"] = torch.tensor([0] * case["parents"] + [1] * children, dtype=torch.int32, device=DEV)
        return st
    lens = _ragged(case, case["seqs"], case["shortest"], case["longest"])
    ids, total = _page_ids(case, lens)
    keep = set(_kept(case))
    rows = [row if s in keep else [] for s, row in enumerate(ids)]
    max_pages = max(map(len, ids))
    st["K"], st["V"] = _pool(case, gen, total, case["layers"])
    table = _table(rows, max_pages).to(DEV)
    refs = _uses(table, total)
    free = _free_words(refs)
    # the bookkeeping in one buffer, and its copy to go back to
    ints = torch.cat([table.flatten(), refs, free])
    st["before"], st["ints"] = ints, ints.clone()
    a, b = table.numel(), table.numel() + total
    st["table"], st["refs"], st["free"] = st["ints"][:a].view(table.shape), st["ints"][a:b], st["ints"][b:]
    st["len"] = torch.tensor([n if s in keep else 0 for s, n in enumerate(lens)], dtype=torch.int32, device=DEV)
    return st


# ---------------------------------------------------------------------------------------------------- the framework's calls
def _handle(st):
    """What a program keeps beside its data: the cache's handle and the calls' scratch memory."""
    import paper_2605_08568_amd as pa
    if "kv" not in st:
        st["kv"] = pa.KV(st["K"], st["V"], st["table"], st["len"], st.get("refs"), st.get("free"))
    return pa, st["kv"]


def _run_own(st):
    c = st["case"]
    pa, kv = _handle(st)
    if c["kind"] == "decode":
        if "ws" not in st:
            st["ws"] = pa.attend_decode_workspace(kv, c["heads"], c["seqs"])
        return pa.attend_decode(kv, 0, st["q"], window=c["window"], sinks=c["sinks"], with_lse=True, workspace=st["ws"])
    if c["kind"] == "prefill":
        if "ws" not in st:
            st["ws"] = pa.attend_prefill_workspace(kv, c["heads"], st["q"].shape[0], c["prompts"])
        return pa.attend_prefill(kv, 0, st["q"], st["off"], window=c["window"], sinks=c["sinks"], with_lse=True, workspace=st["ws"])
    if c["kind"] == "append":
        h, n = c["heads"], c["heads"] + c["kv"]
        qkv = st["qkv"]
        pa.kv_append(kv, 0, qkv[:, h:n], qkv[:, n:], st["off"], q=qkv[:, :h], q_out=st["q_out"], rope=st["rope"])
        return st["q_out"], st["K"], st["V"]
    if "ws" not in st:
        st["ws"] = pa.kv_workspace(kv)
    if c["kind"] == "fork":
        pa.kv_trim(kv, st["keep"])
        pa.kv_fork(kv, st["src"], st["dst"])
        served = pa.kv_reserve(kv, st["n_new"], workspace=st["ws"])
        return st["table"], st["len"], st["refs"], st["free"], served, st["K"], st["V"]
    st["ints"].copy_(st["before"])
    n_live = pa.kv_compact(kv, workspace=st["ws"])
    return st["table"], st["refs"], st["free"], n_live, st["K"], st["V"]


# ---------------------------------------------------------------------------------------------------- the plain forms
def _tokens(st, table):
    """K and V of the tables' sequences in 32 bits, [sequence][kv head][token][d]."""
    t = table.clamp(min=0).long()
    k, v = st["K"][0][t], st["V"][0][t]
    n, mp, kv, pb, d8 = k.shape[:5]
    k = k.permute(0, 2, 1, 3, 5, 4, 6).reshape(n, kv, mp * pb * 16, d8 * 8).float()
    return k, v.permute(0, 2, 1, 3, 5, 4).reshape(n, kv, mp * pb * 16, d8 * 8).float()


def _visible(st, c, pos):
    """[sequence][row][token]: whether the row at position pos sees the token."""
    j = torch.arange(st["table"].shape[1] * c["page"], device=DEV)
    i = pos[:, :, None]
    seen = (j <= i) & (st["table"] >= 0).repeat_interleave(c["page"], 1)[:, None, :]
    if c["window"]:
        seen &= (j > i - c["window"]) | (j < c["sinks"])
    return seen


def _attend(q, k, v, seen, scale):
    """q [s][kv][rows][d]; seen [s][1][rows][token] -> (o, lse)."""
    s = torch.matmul(q, k.transpose(2, 3)).mul_(scale).masked_fill_(~seen, -math.inf)
    m = s.amax(3, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = s.sub_(m).exp_()
    total = p.sum(3, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)
    return o, (m + total.log()).squeeze(3)


def _plain_decode(st, c):
    q, kv = st["q"], c["kv"]
    n, h, d = q.shape
    k, v = _tokens(st, st["table"])
    seen = _visible(st, c, (st["len"] - 1)[:, None].long())
    o, lse = _attend(q.float().view(n, kv, h // kv, d), k, v, seen[:, None], 1 / math.sqrt(d))
    return o.reshape(n, h, d).to(q.dtype), lse.reshape(n, h)


def _rows(st, longest):
    """(prompt of each row, its place in the prompt, position of each padded row [prompt][longest])."""
    off = st["off"].long()
    row = torch.arange(st["q"].shape[0] if "q" in st else st["qkv"].shape[0], device=DEV)
    p = torch.searchsorted(off, row, right=True) - 1
    new = off[1:] - off[:-1]
    return p, row - off[p], (st["len"].long() - new)[:, None] + torch.arange(longest, device=DEV)


def _plain_prefill(st, c):
    q, kv = st["q"], c["kv"]
    rows, h, d = q.shape
    n, longest, g = c["prompts"], max(_new_and_past(c)[0]), h // kv
    p, t, pos = _rows(st, longest)
    k, v = _tokens(st, st["table"])
    qs = torch.zeros((n, longest, h, d), device=DEV)
    qs[p, t] = q.float()
    qs = qs.view(n, longest, kv, g, d).permute(0, 2, 3, 1, 4).reshape(n, kv, g * longest, d)
    seen = _visible(st, c, pos)
    o, lse = _attend(qs, k, v, seen.repeat(1, g, 1)[:, None], 1 / math.sqrt(d))
    o = o.view(n, kv, g, longest, d).permute(0, 3, 1, 2, 4).reshape(n, longest, h, d)[p, t]
    lse = lse.view(n, kv, g, longest).permute(0, 3, 1, 2).reshape(n, longest, h)[p, t]
    return o.to(q.dtype), lse


def _rotated(x, rope):
    half = x.shape[2] // 2
    a, b = x[..., :half].float(), x[..., half:].float()
    cos, sin = rope[:, None, :half], rope[:, None, half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], 2).to(x.dtype)


def _plain_append(st, c):
    h, n, page = c["heads"], c["heads"] + c["kv"], c["page"]
    p, t, pos = _rows(st, max(_new_and_past(c)[0]))
    at = pos[p, t]
    rope = st["rope"][at]
    st["q_out"].copy_(_rotated(st["qkv"][:, :h], rope))
    k, v = _rotated(st["qkv"][:, h:n], rope), st["qkv"][:, n:]
    ids, w = st["table"][p, at // page].long(), at % page
    st["K"][0][ids, :, w // 16, :, w % 16, :] = k.reshape(k.shape[0], c["kv"], c["d"] // 8, 8)
    st["V"][0][ids, :, w // 8, :, w % 8] = v
    return st["q_out"], st["K"], st["V"]


def _plain_fork(st, c):
    table, length, refs, free, page = st["table"], st["len"], st["refs"], st["free"], c["page"]
    src, dst = st["src"].long(), st["dst"].long()
    # the children of the last step are given up, the parents forked
    column = torch.arange(table.shape[1], device=DEV)
    length.copy_(torch.minimum(length, st["keep"]))
    table.copy_(torch.where(column * page < length[:, None], table, torch.full_like(table, -1)))
    table[dst] = table[src]
    length[dst] = length[src]
    refs.copy_(_uses(table, refs.numel()))
    # room for a token: the lowest free pages in order, a shared page that is begun is replaced by its copy
    old = length[dst].long()
    new = old + st["n_new"][dst]
    begun = (old % page != 0) & (new > old)
    part = table[dst].gather(1, (old // page).clamp(max=table.shape[1] - 1)[:, None])[:, 0].long().clamp(min=0)
    earlier = ((part[:, None] == part) & begun & torch.ones(len(dst), len(dst), device=DEV, dtype=torch.bool).tril(-1)).sum(1)
    copied = begun & (refs[part] - earlier > 1)
    need = (new + page - 1) // page - (old + page - 1) // page + copied
    last = need.cumsum(0)
    order = torch.argsort((refs > 0).int(), stable=True)                       # free pages first, lowest id first
    served = last <= (refs == 0).sum()
    first = torch.where(copied, old // page, (old + page - 1) // page)
    fresh = (column >= first[:, None]) & (column < first[:, None] + need[:, None]) & served[:, None]
    ids = order[(last - need)[:, None].add(column).sub(first[:, None]).clamp(0, refs.numel() - 1)]
    rows = torch.where(fresh, ids.int(), table[dst])
    to = torch.where(copied & served, rows.gather(1, (old // page)[:, None])[:, 0].long(), part)
    st["K"][:, to] = st["K"][:, part]
    st["V"][:, to] = st["V"][:, part]
    table[dst] = rows
    length[dst] = torch.where(served, new, old).int()
    refs.copy_(_uses(table, refs.numel()))
    free.copy_(_free_words(refs))
    told = torch.zeros_like(length)
    told[dst] = served.int()
    return table, length, refs, free, told, st["K"], st["V"]


def _plain_compact(st, c):
    st["ints"].copy_(st["before"])
    table, refs = st["table"], st["refs"]
    live = refs > 0
    page = torch.arange(refs.numel(), device=DEV)
    n_live = live.sum()
    src, dst = torch.nonzero(live & (page >= n_live))[:, 0], torch.nonzero(~live & (page < n_live))[:, 0]
    st["K"][:, dst] = st["K"][:, src]
    st["V"][:, dst] = st["V"][:, src]
    moved = page.clone()
    moved[src] = dst
    table.copy_(torch.where(table >= 0, moved[table.clamp(min=0).long()].int(), table))
    refs.copy_(_uses(table, refs.numel()))
    st["free"].copy_(_free_words(refs))
    return table, refs, st["free"], n_live.int().view(1), st["K"], st["V"]


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    plain = {"decode": _plain_decode, "prefill": _plain_prefill, "append": _plain_append, "fork": _plain_fork, "compact": _plain_compact}
    return plain[c["kind"]](state, c)


# ---------------------------------------------------------------------------------------------------- 64 bits
def _sequence(st, s, n, head, c):
    """Keys and values of one sequence's first n tokens and one head, and which of them have a page."""
    ids = st["table"][s, :-(-n // c["page"])].long()
    k, v = st["K"][0].select(1, head)[ids.clamp(min=0)].double(), st["V"][0].select(1, head)[ids.clamp(min=0)].double()
    k = k.movedim(3, 2).flatten(3).flatten(0, 2)
    v = v.movedim(3, 2).flatten(0, 2)
    return k[:n], v[:n], (ids >= 0)[torch.arange(n, device=DEV) // c["page"]]


def _softmax64(q, k, v, seen, scale):
    s = (q @ k.t()) * scale
    s[~seen] = -math.inf
    lse = torch.logsumexp(s, 1)
    return (s - lse[:, None]).exp().nan_to_num(0.0) @ v, lse


def _exact_attend(st, c, rows_of):
    """rows_of(s): (rows of q, positions) of sequence s."""
    q = st["q"]
    g = c["heads"] // c["kv"]
    out, lse = torch.zeros(q.shape, dtype=torch.float64, device=DEV), torch.zeros(q.shape[:2], dtype=torch.float64, device=DEV)
    for s, n in enumerate(st["len"].tolist()):
        a, b, first = rows_of(s, n)
        i = torch.arange(first, first + b - a, device=DEV)[:, None]
        j = torch.arange(n, device=DEV)
        for head in range(c["kv"]):
            k, v, there = _sequence(st, s, n, head, c)
            seen = (j <= i) & there
            if c["window"]:
                seen = seen & ((i - j < c["window"]) | (j < c["sinks"]))
            for h in range(head * g, (head + 1) * g):
                out[a:b, h], lse[a:b, h] = _softmax64(q[a:b, h].double(), k, v, seen, c["d"] ** -0.5)
    return out, lse


def _exact_fork(st, c):
    """One sequence after another, on lists."""
    page = c["page"]
    length = st["len"].tolist()
    rows = [[p for p in row if p >= 0] for row in st["table"].tolist()]
    refs = [0] * st["refs"].numel()
    src, dst = st["src"].tolist(), st["dst"].tolist()
    for a, b in zip(src, dst):
        rows[b], length[b] = list(rows[a]), length[a]
    for row in rows:
        for p in row:
            refs[p] += 1
    K, V = st["K"].double(), st["V"].double()
    for b in dst:
        if length[b] % page == 0 or refs[rows[b][-1]] > 1:
            fresh = refs.index(0)
            refs[fresh] = 1
            if length[b] % page:
                old = rows[b].pop()
                refs[old] -= 1
                K[:, fresh], V[:, fresh] = K[:, old], V[:, old]
            rows[b].append(fresh)
        length[b] += 1
    return None, None, None, None, None, K, V


def _exact_compact(st, c):
    refs = st["refs"].tolist()
    n_live = sum(r > 0 for r in refs)
    K, V = st["K"].double(), st["V"].double()
    holes = iter([p for p in range(n_live) if not refs[p]])
    for p in range(n_live, len(refs)):
        if refs[p]:
            hole = next(holes)
            K[:, hole], V[:, hole] = K[:, p], V[:, p]
    return None, None, None, None, K, V


def exact(case, seed):
    c = dict(case)
    st = prepare(case, seed)
    if c["kind"] == "fork":
        return _exact_fork(st, c)
    if c["kind"] == "compact":
        return _exact_compact(st, c)
    if c["kind"] == "decode":
        return _exact_attend(st, c, lambda s, n: (s, s + 1, n - 1))
    new, past = _new_and_past(c)
    if c["kind"] == "prefill":
        off = st["off"].tolist()
        return _exact_attend(st, c, lambda s, n: (off[s], off[s + 1], past[s]))
    h, n, half = c["heads"], c["heads"] + c["kv"], c["d"] // 2
    K, V, x = st["K"].double(), st["V"].double(), st["qkv"].double()
    pos = torch.cat([torch.arange(p, p + m, device=DEV) for m, p in zip(new, past)])
    seq = torch.cat([torch.full((m,), s, device=DEV) for s, m in enumerate(new)])
    turn = torch.complex(st["rope"][pos, :half].double(), st["rope"][pos, half:].double())[:, None]
    z = torch.complex(x[:, :n, :half], x[:, :n, half:]) * turn
    qk = torch.cat([z.real, z.imag], 2)
    ids, w = st["table"][seq, pos // c["page"]].long(), pos % c["page"]
    for t8 in range(c["d"] // 8):
        K[0][ids, :, w // 16, t8, w % 16] = qk[:, h:, 8 * t8:8 * t8 + 8]
    V[0].permute(0, 1, 2, 4, 3)[ids, :, w // 8, w % 8] = x[:, n:]
    return qk[:, :h], K, V
