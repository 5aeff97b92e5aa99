"""Attention of batches that begin alike against the float64 oracle: every position that a row does not see holds NaN, pages stand in any order, rows
share pages as forks leave them or in any other way, outputs, plans and workspaces between canaries."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import kv_oracle as ko

pytestmark = pytest.mark.gpu

pa = pytest.importorskip("paper_2605_08568_amd")
from helpers import check_guards, guarded_bytes, i32  # noqa: E402
from test_gpu_kv import compare, guarded, rounded, upload  # noqa: E402

DEV = "cuda"


class Family:
    """A cache of one layer (behind another that holds NaN).  rows: per sequence a list of (name, columns) whose pages all sequences with that name have, and the
    number of tokens behind them that are its own.  gone(s, c): column c of sequence s was given up."""

    def __init__(self, dtype, n_kv, d, page, rows, gone=None, seed=0, table=None, lens=None, room=0):
        rng = np.random.default_rng(seed)
        self.dtype, self.n_kv, self.d, self.page = dtype, n_kv, d, page
        if table is None:
            names = {}
            for shared, _ in rows:
                for name, cols in shared:
                    names.setdefault(name, cols)
            lens = [sum(cols for _, cols in shared) * page + more for shared, more in rows]
            cols = max(-(-(n + room) // page) for n in lens) + 1
            own = [-(-(more + room) // page) for _, more in rows]
            total = sum(names.values()) + sum(own)
            ids = iter(rng.permutation(total + 3)[:total])
            held = {name: [next(ids) for _ in range(c)] for name, c in names.items()}
            table = np.full((len(rows), cols), -1, np.int64)
            for s, (shared, _) in enumerate(rows):
                row = [p for name, c in shared for p in held[name][:c]] + [next(ids) for _ in range(own[s])]
                table[s, :len(row)] = row
            n_pages = total + 3
        else:
            n_pages = int(table.max()) + 3
        self.table, self.lens = table, list(lens)
        most = [0] * n_pages                                       # tokens of a page that some row has
        for s in range(len(self.lens)):
            for c in range(table.shape[1]):
                if table[s, c] >= 0:
                    most[table[s, c]] = max(most[table[s, c]], min(max(self.lens[s] + room - c * page, 0), page))
        self.pages = [rounded(rng.standard_normal((n_pages, page, n_kv, d)), dtype) for _ in range(2)]
        for x in self.pages:
            for p in range(n_pages):
                x[p, most[p]:] = np.nan
        if gone:
            for s in range(len(self.lens)):
                for c in range(table.shape[1]):
                    if gone(s, c):
                        table[s, c] = -1
        K = upload(np.stack([ko.k_to_pages(x) for x in self.pages[0]]), dtype)
        V = upload(np.stack([ko.v_to_pages(x) for x in self.pages[1]]), dtype)
        self.kv = pa.KV(torch.stack([torch.full_like(K, torch.nan), K]), torch.stack([torch.full_like(V, torch.nan), V]), i32(table), i32(np.array(self.lens)))

    def write_v(self, p, w, value):
        """Token w of page p, every head."""
        self.pages[1][p, w] = value
        self.kv.V[1, p] = upload(ko.v_to_pages(self.pages[1][p]), self.dtype)

    def tokens(self, s):
        """(k, v, there) of a sequence."""
        n = self.lens[s]
        cols = self.table[s, :-(-n // self.page)]
        k, v = (x[np.maximum(cols, 0)].reshape(-1, self.n_kv, self.d)[:n] for x in self.pages)
        return k, v, np.repeat(cols >= 0, self.page)[:n]


def tiles_of(plan):
    return int(plan[:64].view(torch.int32)[8])


def run(f, n_q, window=0, sinks=0, seqs=None, plan_seqs=None, plan=None, scale=None, seed=1, pad=0, shares=None, check=True):
    """plan: a ready one (else made here, between canaries); shares: whether tiles are expected."""
    rng = np.random.default_rng(seed)
    rows = len(f.lens) if seqs is None else len(seqs)
    q = rounded(2 * rng.standard_normal((rows, n_q, f.d)), f.dtype)
    wide = torch.full((rows, n_q * f.d + pad), torch.nan, device=DEV, dtype=f.kv.K.dtype)
    wide[:, :n_q * f.d] = upload(q, f.dtype).flatten(1)
    qd = wide[:, :n_q * f.d].unflatten(1, (n_q, f.d))
    listed = None if seqs is None else i32(np.array(seqs))
    if plan is None:
        pbuf, plan = guarded_bytes(pa.shared_plan_bytes(f.kv, n_q, rows))
        pa.shared_plan(f.kv, n_q, rows, listed if plan_seqs is None else i32(np.array(plan_seqs)), window, sinks, plan)
        check_guards(pbuf, "plan")
        if shares is not None:
            assert (tiles_of(plan) > 0) == shares, tiles_of(plan)
    buf, whole, out = guarded(rows, n_q, f.d, qd, pad)
    lbuf, lmid = guarded_bytes(rows * n_q * 4)
    wbuf, ws = guarded_bytes(int(pa.lib().parse_attend_shared_workspace_bytes(f.kv.c(), n_q, rows)))
    ws[:] = 0xff                                                   # NaN, and counts of -1
    before, kept = whole[:, n_q * f.d:].clone(), plan.clone()
    lse = lmid[:rows * n_q * 4].view(torch.float32).view(rows, n_q)
    pa.attend_shared(f.kv, 1, qd, plan, listed, scale, window, sinks, out, lse, workspace=ws)
    for b, what in ((buf, "out"), (lbuf, "lse"), (wbuf, "workspace")):
        check_guards(b, what)
    assert torch.equal(whole[:, n_q * f.d:].view(torch.uint8), before.view(torch.uint8)), "stores between the rows"
    assert torch.equal(plan, kept), "the plan is read only"
    if check:
        scale = f.d ** -0.5 if scale is None else scale
        want = []
        for r in range(rows):
            s = r if seqs is None else seqs[r]
            if not 0 <= s < len(f.lens):
                want.append((np.zeros((n_q, f.d)), np.full(n_q, -np.inf), np.zeros((n_q, f.d)), np.zeros(n_q), 1))
                continue
            k, v, there = f.tokens(s)
            want.append((*ko.attend_row(q[r], k, v, ko.visible(f.lens[s] - 1, there, window, sinks), scale), f.lens[s]))
        compare(f, out, lse, want, f.d)
    return out, lse, plan, qd


def tree(page, prompts=2, children=3, system=256, prompt=320, own=(1, 40, 77)):
    """Children of prompts behind a system text."""
    return [([("system", system // page), (f"p{p}", prompt // page + p)], own[(p + c) % len(own)]) for c in range(children) for p in range(prompts)]


WIDTHS = [(t, d) for t in ("bf16", "fp32") for d in (32, 64, 96, 128, 160, 192, 224, 256)]


@pytest.mark.parametrize("dtype,d", WIDTHS)
def test_widths(dtype, d):
    run(Family(dtype, 2, d, 16, tree(16), seed=d), 6, pad=8, shares=True)


@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 4), (8, 1), (17, 1), (40, 2), (28, 4), (80, 1), (130, 2), (300, 1)])
def test_head_groups(heads, kv):
    run(Family("bf16", kv, 64, 32, tree(32), seed=heads), heads, shares=True)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (200, 0), (300, 4), (400, 300), (5000, 4), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_windows(page, window, sinks):
    run(Family("bf16", 2, 64, page, tree(page, 3, 4, 512, 768, (1, 16, 33, 150)), seed=page), 4, window, sinks)


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("window,sinks", [(300, 5), (260, 0), (700, 130)])
def test_pages_outside_the_windows_are_gone(page, window, sinks):
    """Every row has given up its own pages: the shortest row holds some that the others do not."""
    rows = tree(page, 2, 6, 512, 512, (1, 30, 99, 170, 200))
    lens = [sum(c for _, c in sh) * page + n for sh, n in rows]
    f = Family("bf16", 2, 128, page, rows, lambda s, c: c * page >= sinks and (c + 1) * page <= lens[s] - window + 1, seed=3)
    run(f, 8, window, sinks, shares=True)


@pytest.mark.parametrize("rows", [1, 2, 64, 65, 200])
def test_numbers_of_rows(rows):
    """One prompt for all, every head with its own keys: up to 128 columns a tile."""
    family = [([("p", 10)], 1 + s % 19) for s in range(rows)]
    run(Family("bf16", 2, 32, 16, family, seed=rows), 2, shares=rows > 1)


@pytest.mark.parametrize("dtype,d,rows", [("bf16", 32, 300), ("bf16", 32, 1500), ("fp32", 256, 300)])
def test_more_rows_than_a_workgroup_has_threads(dtype, d, rows):
    """Many groups of two to five rows, their order shuffled: plans of more rows than the threads that make them, sums over entries in several rounds."""
    rng = np.random.default_rng(rows)
    family = [([(f"p{g}", 8 + g % 2)], int(rng.integers(1, 40))) for g in range(rows // 3) for _ in range(2 + g % 3)][:rows]
    family = [family[i] for i in rng.permutation(len(family))]
    _, _, plan, _ = run(Family(dtype, 1, d, 16, family, seed=rows), 2, shares=True)
    assert tiles_of(plan) == len({sh[0][0] for sh, _ in family if sum(x[0][0][0] == sh[0][0] for x in family) > 1})


@pytest.mark.parametrize("rows,cols", [(3, 375), (64, 30), (70, 30), (70, 300)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 40), (4000, 4)])
def test_windows_of_few_and_many_rows(rows, cols, window, sinks):
    """Plans of a wavefront and of a workgroup a row, of more columns than that has threads."""
    f = Family("bf16", 1, 32, 16, [([("s", 9), (f"p{r % 3}", cols + r % 3)], 1 + 7 * r % 50) for r in range(rows)], seed=rows)
    # three rows have a prompt each; of the text before them, 144 tokens, the windows leave the sinks' pages: ceil(40 / 16) * 16 = 48 tokens, ceil(4 / 16) * 16 = 16, both below 128
    run(f, 1, window, sinks, seqs=list(range(rows)), shares=rows > 3 or window == 0)


def test_many_groups_in_any_order():
    rng = np.random.default_rng(5)
    family = [([("s", 9), (f"g{g}", 8 + g % 3), (f"g{g}.{c}", 12)], int(rng.integers(1, 60))) for g in range(11) for c in range(2) for _ in range(3)]
    rng.shuffle(family)
    _, _, plan, _ = run(Family("bf16", 1, 64, 16, family, seed=6), 4, shares=True)
    assert tiles_of(plan) == 3 + 11 + 22                           # the text: 66 rows of four heads in tiles of 128 columns, the prompts: 24 columns each, their forks: 12


def test_a_short_text_before_the_prompts_goes_with_them():
    """Two pages that all share are too few for a tile of their own: the prompts' tiles begin with them."""
    family = [([("s", 2), (f"p{p}", 20)], 5 + p) for p in range(4) for _ in range(3)]
    _, _, plan, _ = run(Family("bf16", 2, 64, 16, family, seed=7), 4, shares=True)
    assert tiles_of(plan) == 4


def test_nothing_shared_and_short_runs():
    run(Family("bf16", 2, 64, 16, [([(f"p{s}", 10)], 7) for s in range(5)], seed=8), 4, shares=False)
    run(Family("bf16", 2, 64, 16, [([("p", 7)], 7 + s) for s in range(5)], seed=9), 4, shares=False)
    run(Family("fp32", 2, 64, 16, [([], 1 + 37 * s) for s in range(9)], seed=9), 4, shares=False)


def test_equal_rows_and_the_same_sequence_twice():
    f = Family("bf16", 2, 64, 16, [([("p", 20)], 1), ([("p", 20)], 1), ([("p", 20)], 30)], seed=10)
    run(f, 4, shares=True)
    run(f, 4, seqs=[2, 0, 2, 2, 1, 0], shares=True)
    f = Family("bf16", 2, 64, 16, None, table=np.tile(np.arange(12), (4, 1)), lens=[190, 190, 190, 190], seed=11)    # forked, nothing appended yet
    run(f, 4, shares=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_without_tokens(dtype):
    """Sequences that the table does not have, lengths of zero, and sequences that were not served where the plan had their number."""
    f = Family(dtype, 2, 64, 16, tree(16), seed=12)
    run(f, 4, seqs=[0, -1, 3, 99, 1, 2], shares=True)
    run(f, 4, seqs=[0, -1, 2, -1, 4, 5], plan_seqs=[0, 1, 2, 3, 4, 5], shares=True)
    run(f, 4, seqs=[-1] * 6, plan_seqs=[0, 1, 2, 3, 4, 5], shares=True)
    run(f, 4, 300, 4, seqs=[-1, 1, -1, 3, 4, 5], plan_seqs=[0, 1, 2, 3, 4, 5])
    f.lens[2] = 0
    f.kv.len.copy_(i32(np.array(f.lens)))
    run(f, 4, shares=True)


@pytest.mark.parametrize("seed", range(8))
def test_tables_that_no_fork_made(seed):
    """Every column of a row is one of two or three pages, or none; runs of equal columns of all lengths."""
    rng = np.random.default_rng(100 + seed)
    rows, cols, page = 7, 60, 16
    pick = np.zeros((rows, cols), np.int64)
    for c in range(cols):
        pick[:, c] = pick[:, c - 1] if c and rng.random() < 0.9 else rng.integers(0, 3, rows)
    holes = rng.random((rows, cols)) < (0.0 if seed % 2 else 0.03)
    table = np.where(holes, -1, np.arange(cols) * 3 + pick)
    lens = [int(n) for n in rng.integers(cols * page // 2, cols * page + 1, rows)]
    window, sinks = [(0, 0), (400, 4), (150, 40), (0, 0)][seed % 4]
    run(Family("bf16", 2, 64, page, None, table=table, lens=lens, seed=seed), 4, window, sinks)


def test_a_plan_holds_while_sequences_grow():
    rows = tree(16, 2, 3, 256, 320, (1, 20, 37))
    f = Family("bf16", 2, 64, 16, rows, seed=13, room=90)
    for window, sinks in ((0, 0), (330, 4), (60, 0)):
        _, _, plan, _ = run(f, 4, window, sinks)
        begun = list(f.lens)
        for step in (1, 17, 88):
            f.lens = [n + step - (s == 1) for s, n in enumerate(begun)]    # one of them was not served once
            f.kv.len.copy_(i32(np.array(f.lens)))
            run(f, 4, window, sinks, plan=plan, seed=step)
        f.lens = begun
        f.kv.len.copy_(i32(np.array(f.lens)))


def test_a_plan_for_another_call_shares_nothing():
    f = Family("bf16", 2, 64, 16, tree(16), seed=14)
    _, _, plan, _ = run(f, 4, shares=True)
    big = torch.zeros(4 * plan.numel(), dtype=torch.uint8, device=DEV)
    big[:plan.numel()] = plan
    run(f, 4, 300, 4, plan=big)
    run(f, 8, plan=big)
    run(f, 4, seqs=[0, 1, 2], plan=big)
    run(f, 4, plan=torch.zeros_like(big))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_values_that_some_rows_see_and_others_do_not(dtype, bad):
    """Windows that begin in a shared run: an infinity or NaN of V reaches the rows that see it, and no other."""
    rows = [([("p", 30)], n) for n in (1, 40, 100)]
    f = Family(dtype, 1, 64, 16, rows, seed=15)
    at = 480 + 1 - 200 + 10                                        # the first row's window has it, the others' do not
    f.write_v(f.table[0, at // 16], at % 16, bad)
    out, _, _, _ = run(f, 3, 200, 0, shares=True, check=False)
    clean = Family(dtype, 1, 64, 16, rows, seed=15)
    ref, _, _, _ = run(clean, 3, 200, 0, shares=True)
    assert torch.equal(out[1:], ref[1:])
    if np.isnan(bad):
        assert bool(out[0].isnan().all())
    else:
        assert bool((out[0] == bad).all())


@pytest.mark.parametrize("scale", [0.0, -0.2, 1.7])
def test_scales(scale):
    run(Family("bf16", 2, 64, 16, tree(16), seed=16), 4, scale=scale, shares=True)


@pytest.mark.parametrize("n_q", [128, 640])
def test_shares_of_more_steps_than_lanes(n_q):
    """Heads of so many caches that a share has over 64 steps: narrow (four columns) and wide tiles (twenty), and the first row's own tokens."""
    run(Family("bf16", 128, 32, 64, [([("p", 150)], 30), ([("p", 150)], 1), ([("p", 150)], 64), ([("p", 150)], 5)], seed=18), n_q, shares=True)
    run(Family("bf16", 128, 32, 64, [([], 9700), ([], 3)], seed=19), n_q, shares=False)


def test_a_pool_that_does_not_stay_in_the_caches():
    """Over 192 MB: loads of narrow entries past the caches; of tokens that only one row has, and of a prompt's."""
    run(Family("bf16", 8, 128, 64, [([("p", 330)], 70), ([("p", 330)], 1), ([], 4000)], seed=20), 16, shares=True)


def test_a_plan_for_a_larger_table_shares_nothing():
    f = Family("bf16", 1, 64, 16, tree(16), seed=21)
    n = len(f.lens)
    first = list(range(3))
    _, _, plan, _ = run(f, 2, seqs=[n - 1, n - 2, n - 3], shares=True)
    f.table, f.lens = f.table[:3], f.lens[:3]
    f.kv = pa.KV(f.kv.K, f.kv.V, i32(f.table), i32(np.array(f.lens)))
    run(f, 2, seqs=first, plan=plan)


def test_long_prompts_are_cut_over_the_card():
    run(Family("bf16", 1, 64, 64, [([("p", 160)], 50 + 100 * s) for s in range(6)], seed=17), 4, shares=True)


def test_same_bits_graph_and_streams():
    """Captured and replayed with other inputs, on another stream, and twice at once with a workspace each."""
    f = Family("bf16", 2, 128, 16, tree(16, 3, 5), seed=18)
    n_q = 8
    out, lse, plan, q = run(f, n_q, shares=True)
    wants = [out.clone()]
    q2 = torch.randn_like(q)
    wants.append(pa.attend_shared(f.kv, 1, q2, plan))
    ws, ws2 = pa.attend_shared_workspace(f.kv, n_q, q.shape[0]), pa.attend_shared_workspace(f.kv, n_q, q.shape[0])
    static, got, made = q.clone(), torch.empty_like(out), torch.empty_like(plan)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pa.attend_shared(f.kv, 1, static, plan, out=got, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, wants[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pa.shared_plan(f.kv, n_q, q.shape[0], plan=made)
        pa.attend_shared(f.kv, 1, static, made, out=got, workspace=ws)
    for i in (0, 1, 0, 1, 1, 0):
        static.copy_(q2 if i else q)
        ws.fill_(0xee)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, wants[i]), i
    a, b = torch.empty_like(out), torch.empty_like(out)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        with torch.cuda.stream(side):
            pa.attend_shared(f.kv, 1, q, plan, out=a, workspace=ws)
        with torch.cuda.stream(other):
            pa.attend_shared(f.kv, 1, q2, plan, out=b, workspace=ws2)
    torch.cuda.synchronize()
    assert torch.equal(a, wants[0]) and torch.equal(b, wants[1])


def test_after_real_forks():
    """Sequences made with fork, reserve and trim, shared pages copied where they are begun: the same as the decode attention, whatever the plan finds."""
    torch.manual_seed(3)
    kv = pa.KV.empty(2, 300, 16, 2, 64, 12, 60)
    kv.K.normal_(), kv.V.normal_()
    pa.kv_reserve(kv, i32([700, 333] + [0] * 10))
    pa.kv_fork(kv, i32([0, 0, 0, 1, 1, 0]), i32([2, 3, 4, 5, 6, 7]))
    pa.kv_reserve(kv, i32([0, 0, 5, 20, 50, 1, 17, 0, 0, 0, 0, 0]))
    pa.kv_fork(kv, i32([4, 4]), i32([8, 9]))
    pa.kv_reserve(kv, i32([0] * 8 + [30, 2, 0, 0]))
    q = torch.randn(12, 8, 64, device=DEV).bfloat16()
    for window, sinks in ((0, 0), (500, 4)):
        plan = pa.shared_plan(kv, 8, 12, window=window, sinks=sinks)
        assert tiles_of(plan) > 0
        for step in range(3):
            got, gl = pa.attend_shared(kv, 1, q, plan, window=window, sinks=sinks, with_lse=True)
            want, wl = pa.attend_decode(kv, 1, q, window=window, sinks=sinks, with_lse=True)
            # two joins of the same sums: each result rounded once more than the exact one
            assert torch.equal(gl.isinf(), wl.isinf())
            seen = ~wl.isinf()
            assert float((gl - wl)[seen].abs().max()) < 2e-5
            assert bool(((got.float() - want.float()).abs() <= 2.0 ** -7 * want.float().abs() + 1e-4).all())
            pa.kv_reserve(kv, i32([0, 0, 9, 9, 9, 9, 9, 9, 9, 9, 0, 0]))
            if window:
                pa.kv_trim(kv, None, window, sinks)


@pytest.mark.parametrize("window,sinks", [(0, 0), (200, 4)])
def test_the_example_serves_samples_that_share_their_prompts(window, sinks):
    """Norm, projections, cache and attention together, prompts long enough to be shared, one recorded step; every step's attention against a plain one."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_block.py")
    spec = importlib.util.spec_from_file_location("serve_block", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    r = m.run(hidden=512, heads=8, kv_heads=4, prompts=2, length=300, samples=5, steps=30, groups=8, gs=32, k=4, window=window, sinks=sinks, check=True)
    # weights rounded as two halves, the result once (2^-8); the plain form in 32 bits
    assert r["worst"] <= 2.0 ** -7 and r["steps"] == 30 and bool(torch.isfinite(r["x"].float()).all())
    assert r["lengths"] == [0, 0] + [330] * 5 + [293] * 5


# ---- pages that a row has given up and others of its tile have not --------------------------------------------------------
def give_up(f, window, sinks, which=None):
    """What parse_kv_trim gives up at the present lengths."""
    for s in range(len(f.lens)) if which is None else which:
        for c in range(f.table.shape[1]):
            if c * f.page >= sinks and (c + 1) * f.page <= f.lens[s] - window + 1:
                f.table[s, c] = -1
    f.kv.table.copy_(i32(f.table))


def grow(f, n):
    f.lens = [m + n for m in f.lens]
    f.kv.len.copy_(i32(np.array(f.lens)))


def marked(dtype, page, own, seed, n_kv=1, room=0):
    """A prompt of 512 tokens and what the rows have behind it.  V of every page's last token is large: who counts one that the row has given up is far off."""
    f = Family(dtype, n_kv, 64, page, [([("p", 512 // page)], n) for n in own], seed=seed, room=room)
    for c in range(512 // page):
        f.write_v(f.table[0, c], page - 1, 1000.0)
    return f


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("page", [16, 32])
@pytest.mark.parametrize("n_q", [2, 12, 40])
def test_rows_of_a_tile_that_gave_up_the_first_token_that_they_see(dtype, page, n_q):
    """parse_kv_trim gives up what the NEXT token does not see: a page that ends with the first token of the last one's window too.  The shortest row still has it."""
    f = marked(dtype, page, (28, 43, 59, 44), seed=30, room=40)             # windows of 300 begin at 240, 255, 271, 256
    _, _, plan, _ = run(f, n_q, 300, 4, shares=True)
    for step in (0, 1, 15, 1, 0):
        grow(f, step)
        give_up(f, 300, 4)
        run(f, n_q, 300, 4, plan=plan, seed=step)


@pytest.mark.parametrize("rows,n_q", [(3, 4), (70, 1)])
@pytest.mark.parametrize("keeps", ["first", "last", "none", "all"])
def test_rows_of_one_length_of_which_some_gave_up_a_page(rows, n_q, keeps):
    """Of rows of the least length one may hold a page that the others have given up: it is the one that is read."""
    f = marked("bf16", 16, [43] * rows, seed=31)
    _, _, plan, _ = run(f, n_q, 300, 4, shares=True)
    give_up(f, 300, 4, {"first": range(1, rows), "last": range(rows - 1), "none": range(rows), "all": ()}[keeps])
    run(f, n_q, 300, 4, plan=plan)


def levels_of(plan, rows):
    return plan[64:64 + 32 * rows].view(torch.int32).view(rows, 8)[:, 1].tolist()


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("rows", [4, 70])
def test_a_plan_made_after_pages_were_given_up_has_every_row(rows, page):
    """Rows whose window begins with the last token of a page that they have given up share as the others do; the plan then holds as one made before."""
    f = marked("bf16", page, [28, 43, 59, 44, *(28 + r % 60 for r in range(rows - 4))], seed=32, room=40)
    give_up(f, 300, 4)
    _, _, plan, _ = run(f, 2, 300, 4, shares=True)
    assert levels_of(plan, rows) == [1] * rows
    for step in (0, 1, 15):
        grow(f, step)
        give_up(f, 300, 4)
        run(f, 2, 300, 4, plan=plan, seed=step)


# ---- tiles of many columns ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,d", [("bf16", 32), ("bf16", 64), ("bf16", 96), ("bf16", 128), ("fp32", 32), ("fp32", 64)])
@pytest.mark.parametrize("rows,n_q", [(5, 26), (9, 24), (33, 8), (20, 12)])
def test_tiles_of_two_blocks_a_wavefront(dtype, d, rows, n_q):
    """65 to 128 columns: 65, 108, 128 and a rest of 4, 120."""
    run(Family(dtype, 2, d, 16, [([("p", 21)], 1 + 7 * s % 60) for s in range(rows)], seed=d + rows), n_q, shares=True)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("bf16", 160), ("fp32", 64), ("fp32", 128)])
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("n_q", [12, 40])
def test_values_that_some_rows_of_a_wide_tile_see(dtype, d, bad, n_q):
    """24 and 80 columns, one block and two a wavefront where the heads are narrow: the sums are made once more, from the pages."""
    rows = [([("p", 30)], n) for n in (1, 40, 100)]
    f, clean = (Family(dtype, 1, d, 16, rows, seed=33) for _ in range(2))
    at = 480 + 1 - 200 + 10                                        # the first row's window has it, the others' do not
    f.write_v(f.table[0, at // 16], at % 16, bad)
    out, _, plan, _ = run(f, n_q, 200, 0, shares=True, check=False)
    assert levels_of(plan, 3) == [1, 1, 0]                         # the third row's window has 100 tokens of the prompt, from 380 on, fewer than 128
    ref, _, _, _ = run(clean, n_q, 200, 0, shares=True)
    assert bool(out[0].isnan().all() if np.isnan(bad) else (out[0] == bad).all())
    # sums of 200 weighted values added in another order, 200 * 2^-24 of at most 4 in size; the result rounded once in either, half a step each
    off = 200 * 2.0 ** -24 * 2 * 4 + (2.0 ** -7 * ref[1:].float().abs() if dtype == "bf16" else 0.0)
    assert bool(((out[1:].float() - ref[1:].float()).abs() <= off).all())


def test_as_many_entries_as_are_allowed():
    """3 * (3200 / 64 + 3200 / 2 + 1) + 3200 = 8153 entries of fp32 heads of 256 columns, 8176 at most: their sums stand beside a ring of 128 KiB in a unit's 160."""
    rows = 3200
    f = Family("fp32", 1, 256, 16, None, table=np.arange(rows)[:, None] % 8, lens=[1 + 7 * r % 16 for r in range(rows)], seed=41)
    run(f, 1, shares=False)


class FuncAttributes(C.Structure):
    """hipFuncAttributes, as far as it is read."""
    _fields_ = [("binary_version", C.c_int), ("cache_mode", C.c_int), ("const_bytes", C.c_size_t), ("local_bytes", C.c_size_t), ("most_dynamic", C.c_int), ("most_threads", C.c_int),
                ("registers", C.c_int), ("carveout", C.c_int), ("ptx_version", C.c_int), ("shared_bytes", C.c_size_t), ("room", C.c_char * 256)]


def test_no_call_lowers_what_another_may_launch_with():
    """The plan's and the attention's LDS go with their rows: 24 bytes a row; a ring of 64 KiB and 4 bytes an entry.  The limit that a call raises before its launch holds for all calls
    of the kernel, of other threads too: behind a small call it still covers a large one."""
    from paper_2605_08568_amd import build
    most = 4000
    kv = pa.KV(torch.zeros(1, 8, 1, 1, 16, 16, 8, device=DEV).bfloat16(), torch.zeros(1, 8, 1, 2, 128, 8, device=DEV).bfloat16(), i32(np.zeros((most, 1))), i32(np.ones(most)))
    lib, hip = C.CDLL(build.LIB), C.CDLL("libamdhip64.so.7")
    for rows in (most, 2800):
        plan = pa.shared_plan(kv, 1, rows)
        pa.attend_shared(kv, 0, torch.zeros(rows, 1, 128, device=DEV).bfloat16(), plan)
    torch.cuda.synchronize()
    for kernel, need in (("_ZN5parse12shared_tilesILi1024EEEv8parse_kvPKiiiiiiNS_6PtPlanE", 24 * most), ("_ZN5parse12attend_partsItLi4ELb0ELb0EEEvNS_6PtArgsE", 65536 + 4 * most)):
        a = FuncAttributes()
        assert hip.hipFuncGetAttributes(C.byref(a), C.c_void_p(C.addressof(C.c_char.in_dll(lib, kernel)))) == 0, kernel
        assert a.most_dynamic >= need, (kernel, a.most_dynamic)


def test_two_threads_with_batches_of_different_sizes():
    """A plan and a call of either need LDS by their rows: what one asks for is not taken from the other between its asking and its launch."""
    import threading
    rng = np.random.default_rng(40)
    most = 4000
    kv = pa.KV(torch.randn(1, 8, 1, 1, 16, 16, 8, device=DEV).bfloat16(), torch.randn(1, 8, 1, 2, 128, 8, device=DEV).bfloat16(), i32(rng.integers(0, 8, (most, 1))),
               i32(rng.integers(1, 17, most)))
    jobs = []
    for rows in (2800, most):
        q, plan, ws = torch.randn(rows, 1, 128, device=DEV).bfloat16(), pa.shared_plan(kv, 1, rows), pa.attend_shared_workspace(kv, 1, rows)
        jobs.append((rows, q, plan, ws, pa.attend_shared(kv, 0, q, plan, workspace=ws).clone(), torch.cuda.Stream()))
    torch.cuda.synchronize()
    wrong = []

    def work(rows, q, plan, ws, want, stream):
        try:
            with torch.cuda.stream(stream):
                out = torch.empty_like(want)
                for _ in range(300):
                    pa.shared_plan(kv, 1, rows, plan=plan)
                    pa.attend_shared(kv, 0, q, plan, out=out, workspace=ws)
                stream.synchronize()
                if not torch.equal(out, want):
                    wrong.append(f"{rows} rows: another result")
        except Exception as e:
            wrong.append(f"{rows} rows: {e}")
    threads = [threading.Thread(target=work, args=job) for job in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not wrong, wrong
