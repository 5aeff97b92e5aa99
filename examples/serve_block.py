"""One decoder block's attention served from end to end: routed low-rank q/k/v and o projections around the paged key-value cache.

Prompts are prefilled (pool and route, one plan for the batch, q/k/v fused, room in the cache, rotation and append, causal attention, o projection), every
prompt is forked into samples that share its pages, and the samples are decoded step by step, one HIP graph replayed: q/k/v over a
decode plan, room for a token (a page that is shared and begun is copied), append, attention over window and sinks (pages that samples share are read once for
all of them), o projection, its output added to the residual stream and the stream's norm, pages that no later token sees given up.  At the end half of the samples
stop and the rest of the cache moves together.

    python examples/serve_block.py [--hidden 4096 --heads 32 --kv 32 --prompts 4 --length 512 --samples 4 --steps 64 --check]

Weights are random and there is no MLP or vocabulary: a step's input is the norm of the stream after the step before.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2605_08568_amd as pa  # noqa: E402

DEV = "cuda"


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def make_layer(gen, n, m, G, gs):
    """A random low-rank layer in the kernels' operand order, singular values folded in."""
    R = G * gs
    Vt = torch.randn((R, n), generator=gen, device=DEV).mul_(n ** -0.5).bfloat16()
    Ut = torch.randn((R, m), generator=gen, device=DEV).mul_(R ** -0.5).bfloat16()
    return pa.layer_to_mfma16(pa.Layer(Vt, Ut, n, m, R, G))


def rope_table(n_pos, d):
    angle = torch.arange(n_pos, device=DEV, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(d // 2, device=DEV, dtype=torch.float64) / (d // 2))
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def attention_of(q, k, v, window, sinks):
    """Plain attention of the last row: q [heads][d], k, v [tokens][n_kv][d], 32 bits."""
    n = k.shape[0]
    j = torch.arange(n, device=DEV)
    seen = (j > n - 1 - window) | (j < sinks) if window else j >= 0
    g = q.shape[0] // k.shape[1]
    k, v = k[seen].repeat_interleave(g, 1), v[seen].repeat_interleave(g, 1)
    s = (q[None] * k).sum(2) * q.shape[1] ** -0.5
    return (torch.softmax(s, 0)[..., None] * v).sum(0)


def run(hidden=4096, heads=32, kv_heads=32, prompts=4, length=512, samples=4, steps=64, groups=16, gs=128, k=8, window=256, sinks=4, page=16, check=False,
        seed=0):
    d = hidden // heads
    gen = torch.Generator(device=DEV); gen.manual_seed(seed)
    qkv = [make_layer(gen, hidden, m, groups, gs) for m in (hidden, kv_heads * d, kv_heads * d)]
    o = make_layer(gen, hidden, hidden, groups, gs)
    Wr = torch.randn((groups, hidden), generator=gen, device=DEV) * hidden ** -0.5
    lengths = [max(1, length - 37 * p) for p in range(prompts)]
    off = i32([sum(lengths[:p]) for p in range(prompts + 1)])
    rows, seqs = sum(lengths), prompts * (1 + samples)
    columns = -(-(length + steps + 1) // page)
    pages = sum(-(-n // page) for n in lengths) + prompts * samples * (2 + (min(steps, window + 2 * page) if window else steps) // page) + 2
    cache = pa.KV.empty(1, pages, page, kv_heads, d, seqs, columns)
    rope = rope_table(length + steps + 1, d)
    room = pa.kv_workspace(cache)

    # ---- prefill: one subset of rank groups per prompt, one plan for the batch
    X = torch.randn((rows, hidden), generator=gen, device=DEV).bfloat16()
    subsets = pa.route(X, off, Wr, k)
    pid, _, _, n_patterns, rep = pa.bucket_patterns(subsets, k)
    packed = [pa.Patterns(k, prompts, *pa.pack_patterns(l, subsets, k, k, rep, n_patterns, prompts)) for l in qkv + [o]]
    q, key, value = pa.lowrank_prefill_multi(qkv, packed[:3], X, off, pid)
    placed = torch.empty(prompts, dtype=torch.int32, device=DEV)
    pa.kv_reserve(cache, i32(lengths + [0] * (seqs - prompts)), workspace=room, seqs_served=placed)
    q, key, value = q.view(rows, heads, d), key.view(rows, kv_heads, d), value.view(rows, kv_heads, d)
    pa.kv_append(cache, 0, key, value, off, placed, q=q, q_out=q, rope=rope)
    attn = pa.attend_prefill(cache, 0, q, off, placed)
    y = pa.lowrank_forward(pa.PARSE_PREFILL, o, packed[3], attn.view(rows, hidden), off, pid)

    # ---- every prompt's samples share its pages; each starts from the prompt's last row and a little noise
    parents = [p for p in range(prompts) for _ in range(samples)]
    children = list(range(prompts, seqs))
    pa.kv_fork(cache, i32(parents), i32(children))
    pa.kv_trim(cache, i32([0] * prompts + [length + steps + 1] * len(children)))
    n = len(children)
    last = y[(off[1:] - 1).long()][parents].float()
    stream = (last / last.square().mean(1, keepdim=True).sqrt() + 0.1 * torch.randn((n, hidden), generator=gen, device=DEV)).bfloat16()
    gain = torch.ones(hidden, dtype=torch.bfloat16, device=DEV)
    x = pa.rmsnorm(stream, gain, 1e-6)
    log = {s: [] for s in range(n)}
    if check:                                                      # the prompts' rows as the cache has them
        turned = torch.empty_like(key)
        for p in range(prompts):
            a, b = sum(lengths[:p]), sum(lengths[:p + 1])
            turned[a:b] = rotate(key[a:b], rope[:b - a])
        for s, p in enumerate(parents):
            a, b = sum(lengths[:p]), sum(lengths[:p + 1])
            log[s] = [turned[a:b].float(), value[a:b].float()]

    # ---- decode: the whole step as one graph
    chosen = pa.Patterns(k, prompts, subsets=subsets)
    which = i32(parents)
    plan_qkv, plan_o = pa.decode_plan(qkv, [chosen] * 3, which), pa.decode_plan([o], [chosen], which)
    scratch = torch.empty(max(pa.lowrank_decode_planned_workspace_bytes(qkv), pa.lowrank_decode_planned_workspace_bytes([o])), dtype=torch.uint8, device=DEV)
    ws = pa.attend_shared_workspace(cache, heads, n)
    out = [torch.empty((n, m), dtype=torch.bfloat16, device=DEV) for m in (hidden, kv_heads * d, kv_heads * d, hidden)]
    turned_q, attn = torch.empty((n, heads, d), dtype=torch.bfloat16, device=DEV), torch.empty((n, heads, d), dtype=torch.bfloat16, device=DEV)
    one, served, seq = i32([0] * prompts + [1] * n), torch.empty(seqs, dtype=torch.int32, device=DEV), i32(children)
    room_for = torch.empty_like(seq)                               # the samples that got room for their token, -1 for the others: those are passed over
    common = pa.shared_plan(cache, heads, n, seq, window, sinks)   # holds as long as the samples only grow and their windows move

    def step():
        pa.lowrank_decode_planned(qkv, x, plan_qkv, out[:3], scratch)
        pa.kv_reserve(cache, one, served, room, seq, room_for)
        pa.kv_append(cache, 0, out[1].view(n, kv_heads, d), out[2].view(n, kv_heads, d), seqs=room_for, q=out[0].view(n, heads, d), q_out=turned_q, rope=rope)
        pa.attend_shared(cache, 0, turned_q, common, room_for, window=window, sinks=sinks, out=attn, workspace=ws)
        pa.lowrank_decode_planned([o], attn.view(n, hidden), plan_o, out[3:], scratch)
        if window:
            pa.kv_trim(cache, None, window, sinks)
        pa.rmsnorm(out[3], gain, 1e-6, residual=stream, residual_out=stream, out=x)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph, worst, done = None, 0.0, 0

    def compare():
        torch.cuda.synchronize()
        far = 0.0
        for s in range(n):
            log[s][0] = torch.cat([log[s][0], rotate(out[1].view(n, kv_heads, d)[s:s + 1], rope[log[s][0].shape[0]:][:1]).float()])
            log[s][1] = torch.cat([log[s][1], out[2].view(n, kv_heads, d)[s:s + 1].float()])
            want = attention_of(turned_q[s].float(), *log[s], window, sinks)
            far = max(far, float((attn[s].float() - want).norm() / want.norm()))
        return far
    with torch.cuda.stream(side):
        step()                                                     # the first step eagerly, then the recorded one
    torch.cuda.current_stream().wait_stream(side)
    done = 1
    if check:
        worst = compare()
    if steps > 1:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(steps - 1):
        graph.replay()
        done += 1
        if check:
            worst = max(worst, compare())
    torch.cuda.synchronize()
    took = time.perf_counter() - began

    # ---- half of the samples stop, the rest moves together
    lens = cache.len.tolist()
    pa.kv_trim(cache, i32([0 if s >= prompts and (s - prompts) % 2 else lens[s] for s in range(seqs)]))
    before = int((cache.refs > 0).sum())
    live = int(pa.kv_compact(cache, workspace=room))
    held = sorted(set(cache.table[cache.table >= 0].tolist()))
    assert held == list(range(live)) and live == before, "pages in use stand at the front"
    assert bool(served[prompts:].all()), "the cache was large enough"
    return {"sequences": n, "steps": done, "ms_per_step": took / max(1, steps - 1) * 1e3, "pages_in_use": live, "worst": worst, "lengths": lens, "x": x}


def rotate(x, rope):
    h = x.shape[2] // 2
    a, b, c, s = x[..., :h].float(), x[..., h:].float(), rope[:, None, :h], rope[:, None, h:]
    return torch.cat([a * c - b * s, b * c + a * s], 2).to(x.dtype)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("hidden", 4096), ("heads", 32), ("kv", 32), ("prompts", 4), ("length", 512), ("samples", 4), ("steps", 64), ("window", 256), ("sinks", 4)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--check", action="store_true", help="every step's attention against a plain one")
    a = ap.parse_args()
    r = run(a.hidden, a.heads, a.kv, a.prompts, a.length, a.samples, a.steps, window=a.window, sinks=a.sinks, check=a.check)
    print(f"{r['sequences']} sequences, {r['steps']} steps, {r['ms_per_step']:.3f} ms a step, {r['pages_in_use']} pages in use after half of them stopped"
          + (f"; attention at most {r['worst']:.2e} off the plain one" if a.check else ""))
