"""Bounds of pages, the choice by them and the attention over chosen pages against the float64 oracle."""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as ko
from oracle import step_oracle as so

pytestmark = pytest.mark.gpu

pa = pytest.importorskip("paper_2605_08568_amd")
from helpers import check_guards, guarded_bytes, i32  # noqa: E402
from test_gpu_kv import Case, compare, guarded, rounded, upload  # noqa: E402

DEV = "cuda"
TORCH = {"bf16": torch.bfloat16, "fp32": torch.float32}
WIDTHS = [(t, d) for t in ("bf16", "fp32") for d in (32, 64, 96, 128, 160, 192, 224, 256)]


# ---- bounds ------------------------------------------------------------------------------------------------------------
def run_bounds(case, new, seqs=None, layer=1, mark=7.0):
    """new: tokens of each prompt, None: one each."""
    kv = case.kv
    n = kv.n_layers * kv.n_pages * kv.n_kv * 2 * kv.d
    assert n * case.kv.K.element_size() == pa.lib().parse_kv_bounds_bytes(kv.c())
    buf, mid = guarded_bytes(n * kv.K.element_size())
    bounds = mid[:n * kv.K.element_size()].view(kv.K.dtype).view(kv.n_layers, kv.n_pages, kv.n_kv, 2, kv.d)
    bounds.fill_(mark)
    off = None if new is None else i32(np.concatenate([[0], np.cumsum(new)]))
    pa.kv_bounds(kv, bounds, layer, off, None if seqs is None else i32(np.array(seqs)))
    check_guards(buf, "bounds")
    got, want = bounds.double().cpu().numpy(), np.full(tuple(bounds.shape), mark)
    for p, s in enumerate(range(len(case.lens)) if seqs is None else seqs):
        if not 0 <= s < len(case.lens):
            continue
        n, m = case.lens[s], 1 if new is None else new[p]
        for c in range(max(n - m, 0) // case.page, n // case.page):
            if case.table[s, c] >= 0:
                k = case.k[s][c * case.page:(c + 1) * case.page]
                for l in range(kv.n_layers) if layer < 0 else [layer]:
                    want[l, case.table[s, c]] = so.page_bounds(k) if l == 1 else np.nan      # layer 0 holds NaN
    np.testing.assert_array_equal(got, want)
    return bounds


@pytest.mark.parametrize("dtype,d", WIDTHS)
def test_bounds_widths(dtype, d):
    run_bounds(Case(dtype, 3, d, 32, [31, 32, 33, 300], seed=d), [31, 32, 33, 300])


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_bounds_of_new_tokens(page):
    lens = [1, page - 1, page, page + 1, 2 * page, 5 * page + 3, 6 * page]
    case = Case("bf16", 2, 64, page, lens, seed=page)
    run_bounds(case, None)                                         # one token each
    run_bounds(case, lens, layer=-1)                               # whole sequences, every layer
    run_bounds(case, [n + 1000 for n in lens])                     # more than there are
    run_bounds(case, [0, 1, 0, 1, page, 2 * page + 3, page + 1])
    run_bounds(case, [3 * page, 1, page], seqs=[6, -1, 5])
    run_bounds(case, [1, 1], seqs=[99, 2])


def test_bounds_of_many_sequences_and_missing_pages():
    lens = [16 * (1 + s % 5) + (s % 3) for s in range(150)]
    run_bounds(Case("bf16", 1, 32, 16, lens, lambda s, c: (s + c) % 4 == 0, seed=1), lens)
    run_bounds(Case("bf16", 1, 32, 16, lens, lambda s, c: (s + c) % 4 == 0, seed=1), None)


def test_bounds_in_a_pool_that_does_not_stay_in_the_caches():
    run_bounds(Case("bf16", 8, 128, 64, [64 * 250 + 63, 64 * 140, 5], seed=7), [64 * 3, 64 * 139 + 1, 5])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_bounds_of_many_heads(dtype):
    """Heads one after another in a wavefront, their number not a multiple of it."""
    run_bounds(Case(dtype, 127, 32, 16, [16 * 100, 16 * 100 + 7, 16 * 99], seed=6), [1600] * 3)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_bounds_of_infinities_and_nan(dtype):
    case = Case(dtype, 1, 32, 16, [48], seed=2)
    case.write(0, 3, k=np.inf), case.write(0, 5, k=-np.inf), case.write(0, 20, k=np.nan)
    b = run_bounds(case, [48])[1, case.table[0, :3]].double().cpu().numpy()
    assert np.all(b[0, 0, 0] == -np.inf) and np.all(b[0, 0, 1] == np.inf) and np.all(np.isnan(b[1])) and np.all(np.isfinite(b[2]))


# ---- choice ------------------------------------------------------------------------------------------------------------
def table_cache(rng, dtype, n_kv, d, page, lens, holes=0.0):
    """A cache whose K and V nobody reads, and its bounds."""
    cols = max(max(-(-n // page) for n in lens), 1) + 1
    total = len(lens) * cols
    table = rng.permutation(total).reshape(len(lens), cols)
    table[rng.random(table.shape) < holes] = -1
    for s, n in enumerate(lens):
        table[s, -(-n // page):] = -1
    kv = pa.KV(torch.empty((2, total, n_kv, page // 16, d // 8, 16, 8), dtype=TORCH[dtype], device=DEV),
               torch.empty((2, total, n_kv, page // 8, d, 8), dtype=TORCH[dtype], device=DEV), i32(table), i32(np.array(lens)))
    mid, wide = rng.standard_normal((total, n_kv, 1, d)), np.abs(rng.standard_normal((total, n_kv, 1, d)))
    return kv, table, rounded(np.concatenate([mid - wide, mid + wide], 2), dtype)


def run_select(kv, table, b, lens, n_q, top, first=1, last=1, seqs=None, seed=1, dtype="bf16", q=None):
    rng = np.random.default_rng(seed)
    rows = len(lens) if seqs is None else len(seqs)
    if q is None:
        q = rounded(rng.standard_normal((rows, n_q, kv.d)), dtype)
    wide = torch.full((rows, n_q * kv.d + 8), torch.nan, device=DEV, dtype=kv.K.dtype)
    wide[:, :n_q * kv.d] = upload(q, dtype).flatten(1)
    bounds = torch.full((2, kv.n_pages, kv.n_kv, 2, kv.d), torch.nan, dtype=kv.K.dtype, device=DEV)
    bounds[1] = upload(b, dtype)
    buf, mid = guarded_bytes(rows * kv.n_kv * top * 4)
    pages = mid[:rows * kv.n_kv * top * 4].view(torch.int32).view(rows, kv.n_kv, top)
    wbuf, ws = guarded_bytes(int(pa.lib().parse_select_pages_workspace_bytes(kv.c(), n_q, rows)))
    pa.select_pages(kv, 1, bounds, wide[:, :n_q * kv.d].unflatten(1, (n_q, kv.d)), top, first, last, None if seqs is None else i32(np.array(seqs)), pages, ws)
    check_guards(buf, "pages"), check_guards(wbuf, "workspace")
    got, g = pages.cpu().numpy(), n_q // kv.n_kv
    for r in range(rows):
        s = r if seqs is None else seqs[r]
        n = -(-lens[s] // kv.page) if 0 <= s < len(lens) else 0
        for h in range(kv.n_kv):
            row = table[s, :n] if n else np.zeros(0, np.int64)
            want, gap = so.choose(q[r, h * g:(h + 1) * g], b[np.maximum(row, 0), h], row >= 0, top, first, last)
            # sums in 64 bits in another order: d products a head, half a step of the largest each
            assert gap == 0 or abs(gap) > 2.0 ** -52 * kv.d * g, "the inputs leave the order open"
            np.testing.assert_array_equal(got[r, h], np.concatenate([want, np.full(top - len(want), -1)]), err_msg=f"row {r}, head {h}")
    return pages


@pytest.mark.parametrize("dtype,d", WIDTHS)
def test_select_widths(dtype, d):
    rng = np.random.default_rng(d)
    lens = [700, 16 * 9, 16 * 9 + 1, 1000]
    run_select(*table_cache(rng, dtype, 2, d, 16, lens), lens, 6, 9, dtype=dtype)


@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 4), (17, 1), (40, 2), (28, 4)])
def test_select_head_groups(heads, kv):
    lens = [3000, 500]
    run_select(*table_cache(np.random.default_rng(heads), "bf16", kv, 64, 16, lens), lens, heads, 20, 1, 2)


@pytest.mark.parametrize("top,first,last", [(1, 0, 1), (2, 0, 1), (2, 1, 1), (7, 0, 5), (64, 4, 2), (64, 30, 34), (300, 1, 1), (5000, 1, 1)])
def test_select_numbers(top, first, last):
    lens = [1, 16, 17, 16 * top, 16 * top + 1, 4500, 0]
    lens = [min(n, 9000) for n in lens]
    run_select(*table_cache(np.random.default_rng(top), "bf16", 2, 32, 16, lens), lens, 2, top, first, last)


@pytest.mark.parametrize("rows,kv,cols", [(70, 2, 700), (3, 2, 700), (2, 520, 40), (40, 4, 2300)])
def test_select_launches(rows, kv, cols):
    """One launch for many heads with tables of middle length; two for few of them, for very many, and for longer tables."""
    lens = [16 * cols - 5 - 3 * r for r in range(rows)]
    run_select(*table_cache(np.random.default_rng(cols), "bf16", kv, 32, 16, lens), lens, kv, 9, 1, 1)


def test_select_from_long_tables():
    lens = [16 * 20011 - 3, 16 * 4096, 100]
    run_select(*table_cache(np.random.default_rng(7), "bf16", 1, 32, 16, lens), lens, 4, 1000, 2, 3)
    run_select(*table_cache(np.random.default_rng(8), "fp32", 1, 32, 16, lens), lens, 4, 9, 2, 3, dtype="fp32")


@pytest.mark.parametrize("dtype,d", WIDTHS)
def test_select_widths_in_two_launches(dtype, d):
    """Tables of more than 256 columns and few heads: scores by as many lanes a page as it is wide, several rounds of a wavefront's pages, the last one begun."""
    lens = [16 * 2300 - 3, 16 * 261, 16 * 40]
    run_select(*table_cache(np.random.default_rng(50 + d), dtype, 2, d, 16, lens), lens, 6, 33, 1, 2, dtype=dtype)


def chosen(kv, b, q, top, dtype):
    bounds = torch.zeros((2, kv.n_pages, kv.n_kv, 2, kv.d), dtype=kv.K.dtype, device=DEV)
    bounds[1] = upload(b, dtype)
    return pa.select_pages(kv, 1, bounds, upload(q, dtype), top)[0, 0].tolist()


@pytest.mark.parametrize("cols", [30, 2600])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_select_looks_at_no_column_without_queries(dtype, cols):
    """A column where all queries of the group are zero is not looked at, whatever its bounds hold, NaN too; where one is not zero NaN comes first."""
    rng = np.random.default_rng(60 + cols)
    lens = [16 * cols]
    kv, table, b = table_cache(rng, dtype, 1, 64, 16, lens)
    q = rounded(rng.standard_normal((1, 2, 64)), dtype)
    q[:, :, 7] = 0.0
    want = run_select(kv, table, b, lens, 2, 9, dtype=dtype, q=q)[0, 0].tolist()
    b[table[0, 3:cols:5], 0, :, 7] = np.nan
    b[table[0, 4:cols:5], 0, :, 7] = [-np.inf, np.inf]
    assert chosen(kv, b, q, 9, dtype) == want
    b[table[0, 20], 0, :, 8] = np.nan
    assert 20 in chosen(kv, b, q, 3, dtype)


def test_select_missing_pages_and_sequences():
    rng = np.random.default_rng(9)
    lens = [2000, 900, 300, 40]
    kv, table, b = table_cache(rng, "bf16", 2, 64, 16, lens, holes=0.3)
    run_select(kv, table, b, lens, 4, 12, 2, 2)
    run_select(kv, table, b, lens, 4, 100, 2, 2)
    run_select(kv, table, b, lens, 4, 12, 2, 2, seqs=[3, -1, 0, 99, 0])
    table[0, :] = -1
    kv.table.copy_(i32(table))
    run_select(kv, table, b, lens, 4, 12, 2, 2)


@pytest.mark.parametrize("kinds", [1, 2, 3])
def test_select_ties_go_to_the_lower_column(kinds):
    """Pages of only so many kinds, zeros of both signs among them: nearly every choice is one between equals."""
    rng = np.random.default_rng(kinds)
    lens = [16 * 300, 16 * 77 + 5]
    kv, table, b = table_cache(rng, "bf16", 2, 32, 16, lens)
    b[:] = b[rng.integers(0, kinds, len(b))]
    if kinds == 1:
        b[:] = 0.0 * np.sign(rng.standard_normal(b.shape))
    run_select(kv, table, b, lens, 4, 40, 1, 1)


def test_select_nan_and_infinities():
    rng = np.random.default_rng(11)
    lens = [16 * 200]
    kv, table, b = table_cache(rng, "bf16", 1, 32, 16, lens)
    q = rounded(np.abs(rng.standard_normal((1, 2, 32))) + 0.1, "bf16")
    b[table[0, 150], 0, :, 3] = np.nan
    b[table[0, 120], 0, 1, 5] = np.inf
    b[table[0, 10], 0, 0, 5] = -np.inf                             # no q is negative there: not looked at
    got = run_select_only(kv, b, q, 4)
    assert 150 in got and 120 in got and 10 not in got
    b[table[0, 50], 0, :, 5] = -np.inf
    got = run_select_only(kv, b, q, 199)
    assert 50 not in got and 10 in got and len(set(got)) == 199


def run_select_only(kv, b, q, top):
    bounds = torch.zeros((2, kv.n_pages, kv.n_kv, 2, kv.d), dtype=kv.K.dtype, device=DEV)
    bounds[1] = upload(b, "bf16")
    return pa.select_pages(kv, 1, bounds, upload(q, "bf16"), top)[0, 0].tolist()


# ---- attention over chosen pages -----------------------------------------------------------------------------------------
def run_attend(case, n_q, pages, seqs=None, scale=None, seed=1, pad=0):
    """pages: [rows][n_kv][top]."""
    rng = np.random.default_rng(seed)
    pages = np.asarray(pages)
    rows, _, top = pages.shape
    q = rounded(2 * rng.standard_normal((rows, n_q, case.d)), case.dtype)
    wide = torch.full((rows, n_q * case.d + pad), torch.nan, device=DEV, dtype=case.kv.K.dtype)
    wide[:, :n_q * case.d] = upload(q, case.dtype).flatten(1)
    qd = wide[:, :n_q * case.d].unflatten(1, (n_q, case.d))
    buf, whole, out = guarded(rows, n_q, case.d, qd, pad)
    lbuf, lmid = guarded_bytes(rows * n_q * 4)
    wbuf, ws = guarded_bytes(int(pa.lib().parse_attend_pages_workspace_bytes(case.kv.c(), n_q, rows, top)))
    ws[:] = 0xff
    before = whole[:, n_q * case.d:].clone()
    lse = lmid[:rows * n_q * 4].view(torch.float32).view(rows, n_q)
    pa.attend_pages(case.kv, 1, qd, i32(pages), None if seqs is None else i32(np.array(seqs)), scale, out, lse, workspace=ws)
    for b, what in ((buf, "out"), (lbuf, "lse"), (wbuf, "workspace")):
        check_guards(b, what)
    assert torch.equal(whole[:, n_q * case.d:].view(torch.uint8), before.view(torch.uint8)), "stores between the rows"
    scale = case.d ** -0.5 if scale is None else scale
    want, g = [], n_q // case.n_kv
    for r in range(rows):
        s = r if seqs is None else seqs[r]
        o, l, mag, big = np.zeros((n_q, case.d)), np.full(n_q, -np.inf), np.zeros((n_q, case.d)), np.zeros(n_q)
        most = 1
        for h in range(case.n_kv):
            if not 0 <= s < len(case.lens):
                continue
            n = case.lens[s]
            at = [c * case.page + w for c in pages[r, h] if 0 <= c < case.table.shape[1] and case.table[s, c] >= 0 for w in range(case.page) if c * case.page + w < n]
            at, hs = np.array(at, np.int64), slice(h * g, (h + 1) * g)
            k, v = case.k[s][at][:, h:h + 1], case.v[s][at][:, h:h + 1]
            o[hs], l[hs], mag[hs], big[hs] = ko.attend_row(q[r, hs], k, v, np.ones(len(at), bool), scale)
            most = max(most, len(at))
        want.append((o, l, mag, big, most))
    compare(case, out, lse, want, case.d)
    return out, lse, qd


def some_pages(rng, case, rows, top, holes=0.2):
    """Different columns of each row in any order, -1 between them."""
    p = np.full((rows, case.n_kv, top), -1)
    for r in range(rows):
        n = -(-case.lens[r] // case.page)
        for h in range(case.n_kv):
            c = rng.permutation(max(n, 1))[:top]
            p[r, h, :len(c)] = c
            p[r, h][rng.random(top) < holes] = -1
            rng.shuffle(p[r, h])
    return p


@pytest.mark.parametrize("dtype,d", WIDTHS)
def test_attend_widths(dtype, d):
    case = Case(dtype, 2, d, 16, [1, 16, 17, 77, 300], seed=d)
    run_attend(case, 6, some_pages(np.random.default_rng(d), case, 5, 7), pad=8)


@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 4), (16, 1), (17, 1), (40, 2), (28, 4), (80, 1), (130, 2), (300, 1)])
def test_attend_head_groups(heads, kv):
    case = Case("bf16", kv, 64, 32, [31, 32, 33, 130, 400], seed=heads)
    run_attend(case, heads, some_pages(np.random.default_rng(heads), case, 5, 5))


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("top", [1, 2, 3, 33])
def test_attend_pages_and_numbers(page, top):
    case = Case("bf16", 2, 64, page, [1, page - 1, page, page + 1, 9 * page + 5, 40 * page], seed=page)
    run_attend(case, 4, some_pages(np.random.default_rng(top), case, 6, top, 0.1))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attend_odd_lists(dtype):
    """A column twice, columns outside the table and past the sequence, lists of nothing, sequences that the table does not have, missing pages."""
    case = Case(dtype, 1, 64, 16, [100, 100, 5, 64], lambda s, c: s == 0 and c == 2, seed=3, extra_columns=3)
    run_attend(case, 4, [[[3, 3, 0, -1]], [[6, 5, 100, 8]], [[-1, -1, -1, -7]], [[2 ** 31 - 1, 1, 2, -2 ** 31]]])
    run_attend(case, 4, [[[2, 1, 0]], [[2, 2, 2]], [[0, 1, 2]]], seqs=[0, -1, 99])
    run_attend(case, 4, [[[2, 1, 0]], [[2, 2, 2]], [[0, 1, 2]]], seqs=[3, 3, 1])


@pytest.mark.parametrize("heads", [128, 2560])
def test_attend_shares_of_more_steps_than_lanes(heads):
    """Lists of mostly nothing, 400 steps for four shares a head: narrow and wide entries, pages behind a share's 64th step."""
    case = Case("bf16", 128, 32, 256, [700, 600], seed=4)
    pages = np.full((1, 128, 50), -1)
    for i, c in ((0, 2), (9, 0), (10, 1), (37, 0), (49, 2)):
        pages[0, :, i] = c
    run_attend(case, heads, pages)


def test_attend_lists_that_do_not_stay_in_the_caches():
    """Over 96 MB as the list's length has it: loads past the caches."""
    case = Case("bf16", 1, 256, 256, [2000, 513], seed=5)
    pages = np.full((2, 1, 256), -1)
    pages[0, 0, ::37], pages[1, 0, 250:253] = np.arange(7), (2, 0, 1)
    run_attend(case, 3, pages)


@pytest.mark.parametrize("rows", [1, 63, 65, 300])
def test_attend_numbers_of_rows(rows):
    case = Case("bf16", 1, 32, 16, [1 + (37 * s) % 200 for s in range(rows)], seed=rows)
    run_attend(case, 2, some_pages(np.random.default_rng(rows), case, rows, 6))


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_attend_infinities(bad):
    """One of V that is listed comes out, one that is not listed has no influence."""
    case = Case("bf16", 1, 64, 16, [160], seed=5)
    pages = np.array([[[0, 4, 9]]])
    ref, _, _ = run_attend(case, 3, pages)
    case.kv.V[1, case.table[0, 2]] = bad
    out, _, _ = run_attend(case, 3, pages)
    assert torch.equal(out, ref)
    case.kv.V[1, case.table[0, 4], :, 0, :, 3] = bad
    out = pa.attend_pages(case.kv, 1, upload(np.ones((1, 3, 64)), "bf16"), i32(pages))
    assert bool(out.isnan().all() if np.isnan(bad) else (out == bad).all())


@pytest.mark.parametrize("scale", [0.0, -0.2, 1.7])
def test_attend_scales(scale):
    case = Case("bf16", 2, 64, 16, [300, 77], seed=6)
    run_attend(case, 4, some_pages(np.random.default_rng(1), case, 2, 9), scale=scale)


def test_all_pages_are_the_whole_attention():
    case = Case("bf16", 2, 128, 16, [333, 1000, 16], seed=7)
    q = torch.randn(3, 8, 128, device=DEV).bfloat16()
    bounds = pa.kv_bounds_empty(case.kv)
    pages = pa.select_pages(case.kv, 1, pa.kv_bounds(case.kv, bounds, 1, i32([0, 1000, 2000, 3000])), q, 80)
    got, gl = pa.attend_pages(case.kv, 1, q, pages, with_lse=True)
    want, wl = pa.attend_decode(case.kv, 1, q, with_lse=True)
    assert float((gl - wl).abs().max()) < 2e-5
    assert bool(((got.float() - want.float()).abs() <= 2.0 ** -7 * want.float().abs() + 1e-4).all())


def test_a_step_as_it_is_used():
    """Prompts in, bounds of all of them; then tokens one by one: append, bounds of the pages that they complete, choice, attention, all in one replayed graph, checked
    against the oracle; a compaction in between, after which the bounds are made anew."""
    torch.manual_seed(5)
    rng = np.random.default_rng(5)
    n_kv, n_q, d, page, top, lens = 2, 4, 64, 16, 6, [150, 333, 47, 16]
    kv = pa.KV.empty(1, 90, page, n_kv, d, 5, 40)
    kv.K.fill_(torch.nan), kv.V.fill_(torch.nan)
    pa.kv_reserve(kv, i32([0] + lens))                              # sequence 0 is given up below, so that the others' pages move
    pa.kv_reserve(kv, i32([100, 0, 0, 0, 0]))
    off = np.concatenate([[0], np.cumsum(lens)])
    k, v = (torch.randn(int(off[-1]), n_kv, d, device=DEV).bfloat16() for _ in range(2))
    seqs = i32([1, 2, 3, 4])
    pa.kv_append(kv, 0, k, v, i32(off), seqs)
    pa.kv_append(kv, 0, torch.zeros(100, n_kv, d, device=DEV).bfloat16(), torch.zeros(100, n_kv, d, device=DEV).bfloat16(), i32([0, 100]), i32([0]))
    bounds = pa.kv_bounds_empty(kv).fill_(torch.nan)
    pa.kv_bounds(kv, bounds, 0, i32(off), seqs)
    ks, vs = ([x[off[p]:off[p + 1]].double().cpu().numpy() for p in range(4)] for x in (k, v))
    q, k1, v1 = (torch.empty(4, n, d, device=DEV).bfloat16() for n in (n_q, n_kv, n_kv))
    placed, one = torch.empty_like(seqs), i32([0, 1, 1, 1, 1])
    pages, out = torch.empty((4, n_kv, top), dtype=torch.int32, device=DEV), torch.empty_like(q)
    room, w1, w2 = pa.kv_workspace(kv), pa.select_pages_workspace(kv, n_q, 4), pa.attend_pages_workspace(kv, n_q, 4, top)
    served = torch.empty(5, dtype=torch.int32, device=DEV)

    def step():
        pa.kv_reserve(kv, one, served, room, seqs, placed)
        pa.kv_append(kv, 0, k1, v1, seqs=placed)
        pa.kv_bounds(kv, bounds, 0, seqs=placed)
        pa.select_pages(kv, 0, bounds, q, top, 1, 2, placed, pages, w1)
        pa.attend_pages(kv, 0, q, pages, placed, out=out, workspace=w2)

    graph = None
    for t in range(40):
        q.normal_(), k1.normal_(), v1.normal_()
        if t == 0:
            step()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        else:
            graph.replay()
        torch.cuda.synchronize()
        table, qn = kv.table.cpu().numpy(), q.double().cpu().numpy()
        got, chosen = out.double().cpu().numpy(), pages.cpu().numpy()
        for p in range(4):
            ks[p] = np.concatenate([ks[p], k1[p:p + 1].double().cpu().numpy()])
            vs[p] = np.concatenate([vs[p], v1[p:p + 1].double().cpu().numpy()])
            n = len(ks[p])
            cols = -(-n // page)
            b = np.stack([so.page_bounds(ks[p][c * page:(c + 1) * page]) for c in range(cols)])
            for h in range(n_kv):
                want, _ = so.choose(qn[p, 2 * h:2 * h + 2], b[:, h], np.ones(cols, bool), top, 1, 2)
                np.testing.assert_array_equal(chosen[p, h][chosen[p, h] >= 0], want)
                at = (want[:, None] * page + np.arange(page)).ravel()
                at = at[at < n]
                o, _, mag, _ = ko.attend_row(qn[p, 2 * h:2 * h + 2], ks[p][at][:, h:h + 1], vs[p][at][:, h:h + 1], np.ones(len(at), bool), d ** -0.5)
                # a weight and the result are rounded, 2^-8 each at most
                assert np.all(np.abs(got[p, 2 * h:2 * h + 2] - o) <= 1.05 * 2.0 ** -8 * (mag + np.abs(o)) + 1e-4 * mag)
        if t == 20:
            pa.kv_trim(kv, i32([0, 1000, 1000, 1000, 1000]))
            pa.kv_compact(kv, workspace=room)
            bounds.fill_(torch.nan)
            pa.kv_bounds(kv, bounds, 0, i32(1000 * np.arange(5)), seqs)
            assert bool((kv.table[1:] != i32(table)[1:]).any()), "pages moved"
