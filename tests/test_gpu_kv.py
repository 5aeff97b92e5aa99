"""The paged key-value cache and the attention over it against the float64 oracle: every position that a row does not see holds
NaN or infinities, pages stand in any order, outputs and workspaces between canaries."""
import numpy as np
import pytest
import torch

import synth_inputs as si
from oracle import kv_oracle as ko

pytestmark = pytest.mark.gpu

pa = pytest.importorskip("paper_2605_08568_amd")
from helpers import CANARY, check_guards, guarded_bytes, i32  # noqa: E402

DEV = "cuda"


def rounded(x, dtype):
    """Values that the dtype has, as float64."""
    if dtype == "fp32":
        return x.astype(np.float32).astype(np.float64)
    return torch.from_numpy(x.astype(np.float32)).bfloat16().double().numpy()


def upload(x, dtype):
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32))
    return (t.bfloat16() if dtype == "bf16" else t).to(DEV)


class Case:
    """A cache of one layer (behind another that holds NaN) with sequences of given lengths, pages shuffled, unseen places poisoned."""

    def __init__(self, dtype, n_kv, d, page, lens, gone=None, seed=0, extra_columns=1, poison=np.nan):
        rng = np.random.default_rng(seed)
        self.dtype, self.n_kv, self.d, self.page, self.lens = dtype, n_kv, d, page, lens
        counts = [-(-n // page) for n in lens]
        total, cols = sum(counts), max(counts) + extra_columns
        n_pages = total + 3
        ids = rng.permutation(n_pages)[:total]
        self.table = np.full((len(lens), cols), -1, np.int64)
        K = np.full((n_pages, n_kv, page // 16, d // 8, 16, 8), poison)
        V = np.full((n_pages, n_kv, page // 8, d, 8), poison)
        self.k = [rounded(rng.standard_normal((n, n_kv, d)), dtype) for n in lens]
        self.v = [rounded(rng.standard_normal((n, n_kv, d)), dtype) for n in lens]
        self.there, at = [], 0
        for s, n in enumerate(lens):
            there = np.ones(n, bool)
            for c in range(counts[s]):
                if gone and gone(s, c):
                    there[c * page:(c + 1) * page] = False
                    continue
                p = ids[at]; at += 1
                self.table[s, c] = p
                a, b = c * page, min((c + 1) * page, n)
                full = np.full((2, page, n_kv, d), poison)
                full[0, :b - a], full[1, :b - a] = self.k[s][a:b], self.v[s][a:b]
                K[p], V[p] = ko.k_to_pages(full[0]), ko.v_to_pages(full[1])
            self.there.append(there)
        K, V = upload(K, dtype), upload(V, dtype)
        self.kv = pa.KV(torch.stack([torch.full_like(K, torch.nan), K]), torch.stack([torch.full_like(V, torch.nan), V]),
                        i32(self.table), i32(np.array(lens)))

    def write(self, s, j, k=None, v=None):
        """Puts single rows in place, in the cache and in the oracle's arrays."""
        p, w = self.table[s, j // self.page], j % self.page
        if k is not None:
            self.k[s][j] = k
            self.kv.K[1, p, :, w // 16, :, w % 16, :] = upload(np.broadcast_to(k, (self.n_kv, self.d)), self.dtype).view(self.n_kv, self.d // 8, 8)
        if v is not None:
            self.v[s][j] = v
            self.kv.V[1, p, :, w // 8, :, w % 8] = upload(np.broadcast_to(v, (self.n_kv, self.d)), self.dtype)


def bounds(dtype, d, n, o, lse, mag, big):
    """What the roundings can make, element by element.  Scores: d products and sums in 32 bits, 2^-24 of |q|.|k| each, and the
    scale's and the 2^x's rounding (2^-22 of the score, 2^-22); a weight is off by as much, the mean by twice that; n sums of weights
    and products.  bf16 (8 significand bits): a weight and the result are rounded, 2^-8 each."""
    w = (d + 4) * 2.0 ** -24 * big + 2.0 ** -22 * big + 2.0 ** -21 + n * 2.0 ** -24
    tol = 2 * w[:, None] * mag + 1e-30
    if dtype == "bf16":
        tol = tol + 1.01 * 2.0 ** -8 * (mag + np.abs(o) + 2 * w[:, None] * mag)
    return tol, w + 2.0 ** -22 * (1 + np.abs(lse))


def compare(case, out, lse, want, d):
    """want: per row (o, lse, mag, big, tokens)."""
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for r, (o, l, mag, big, n) in enumerate(want):
        empty = np.isneginf(l)
        assert np.array_equal(np.isneginf(lse[r]), empty), f"row {r}: lse"
        tol, ltol = bounds(case.dtype, d, n, o, np.where(empty, 0, l), mag, big)
        off = np.abs(out[r] - o) - tol
        assert np.all(off <= 0), f"row {r}: {off.max():.3e} over the bound, at {np.unravel_index(off.argmax(), off.shape)}"
        assert np.all(np.abs(lse[r] - l)[~empty] <= ltol[~empty]), f"row {r}: lse {np.abs(lse[r] - l).max()}"


def guarded(rows, heads, d, like, pad=0):
    """Output rows `pad` elements further apart than they are long."""
    es = like.element_size()
    buf, mid = guarded_bytes(rows * (heads * d + pad) * es)
    t = mid[:rows * (heads * d + pad) * es].view(like.dtype).view(rows, heads * d + pad)
    return buf, t, t[:, :heads * d].unflatten(1, (heads, d))


def run_decode(case, n_q, window=0, sinks=0, seqs=None, scale=None, seed=1, pad=0, q=None):
    rng = np.random.default_rng(seed)
    rows = len(case.lens) if seqs is None else len(seqs)
    if q is None:
        q = rounded(2 * rng.standard_normal((rows, n_q, case.d)), case.dtype)
    wide = torch.full((rows, n_q * case.d + pad), torch.nan, device=DEV, dtype=case.kv.K.dtype)
    wide[:, :n_q * case.d] = upload(q, case.dtype).flatten(1)
    qd = wide[:, :n_q * case.d].unflatten(1, (n_q, case.d))
    buf, whole, out = guarded(rows, n_q, case.d, qd, pad)
    lbuf, lmid = guarded_bytes(rows * n_q * 4)
    wbuf, ws = guarded_bytes(int(pa.lib().parse_attend_decode_workspace_bytes(case.kv.c(), n_q, rows)))
    ws[:2048] = 0                                                  # the tickets; the rest holds anything
    before = whole[:, n_q * case.d:].clone()
    lse = lmid[:rows * n_q * 4].view(torch.float32).view(rows, n_q)
    pa.attend_decode(case.kv, 1, qd, seqs=None if seqs is None else i32(np.array(seqs)), scale=scale, window=window, sinks=sinks, out=out, lse=lse,
                     workspace=ws)
    for b, what in ((buf, "out"), (lbuf, "lse"), (wbuf, "workspace")):
        check_guards(b, what)
    assert not bool(ws[:2048].any()), "tickets left"
    assert torch.equal(whole[:, n_q * case.d:].view(torch.uint8), before.view(torch.uint8)), "stores between the rows"
    scale = case.d ** -0.5 if scale is None else scale
    want = []
    for r in range(rows):
        s = r if seqs is None else seqs[r]
        if not 0 <= s < len(case.lens):
            want.append((np.zeros((n_q, case.d)), np.full(n_q, -np.inf), np.zeros((n_q, case.d)), np.zeros(n_q), 1))
            continue
        n = case.lens[s]
        want.append((*ko.attend_row(q[r], case.k[s], case.v[s], ko.visible(n - 1, case.there[s], window, sinks), scale), n))
    compare(case, out, lse, want, case.d)
    return out, lse


def run_prefill(case, n_q, new, window=0, sinks=0, seqs=None, seed=1, pad=0, one_row=False):
    rng = np.random.default_rng(seed)
    rows = sum(new)
    off = np.concatenate([[0], np.cumsum(new)])
    q = rounded(2 * rng.standard_normal((rows, n_q, case.d)), case.dtype)
    wide = torch.full((rows, n_q * case.d + pad), torch.nan, device=DEV, dtype=case.kv.K.dtype)
    wide[:, :n_q * case.d] = upload(q, case.dtype).flatten(1)
    qd = wide[:, :n_q * case.d].unflatten(1, (n_q, case.d))
    buf, whole, out = guarded(rows, n_q, case.d, qd, pad)
    lbuf, lmid = guarded_bytes(rows * n_q * 4)
    wbuf, ws = guarded_bytes(int(pa.lib().parse_attend_prefill_workspace_bytes(case.kv.c(), n_q, rows, len(new))))
    before = whole[:, n_q * case.d:].clone()
    lse = lmid[:rows * n_q * 4].view(torch.float32).view(rows, n_q)
    pa.attend_prefill(case.kv, 1, qd, None if one_row else i32(off), seqs=None if seqs is None else i32(np.array(seqs)), window=window, sinks=sinks,
                      out=out, lse=lse, workspace=ws)
    for b, what in ((buf, "out"), (lbuf, "lse"), (wbuf, "workspace")):
        check_guards(b, what)
    assert torch.equal(whole[:, n_q * case.d:].view(torch.uint8), before.view(torch.uint8)), "stores between the rows"
    want = []
    for p, n in enumerate(new):
        s = p if seqs is None else seqs[p]
        for t in range(n):
            ok = 0 <= s < len(case.lens)
            i = case.lens[s] - n + t if ok else -1
            seen = ko.visible(i, case.there[s], window, sinks) if ok else np.zeros(1, bool)
            k, v = (case.k[s], case.v[s]) if ok else (np.zeros((1, case.n_kv, case.d)),) * 2
            want.append((*ko.attend_row(q[off[p] + t], k, v, seen, case.d ** -0.5), max(i + 1, 1)))
    compare(case, out, lse, want, case.d)
    return out, lse


WIDTHS = [(t, d) for t in ("bf16", "fp32") for d in (32, 64, 96, 128, 160, 192, 224, 256)]


@pytest.mark.parametrize("dtype,d", WIDTHS)
def test_decode_widths(dtype, d):
    run_decode(Case(dtype, 2, d, 16, [1, 16, 17, 77, 300], seed=d), 6, pad=8)


@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 4), (8, 1), (16, 1), (17, 1), (40, 2), (28, 4)])
def test_decode_head_groups(heads, kv):
    run_decode(Case("bf16", kv, 64, 32, [31, 32, 33, 130], seed=heads), heads)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (40, 0), (40, 4), (64, 21), (1000, 4), (33, 200), (1 << 31 - 1 - 1, 2 ** 31 - 1)])
def test_decode_windows(page, window, sinks):
    lens = [1, 5, 39, 40, 41, 127, 128, 129, 255, 500, 1025]
    window = min(window, 2 ** 31 - 1)
    run_decode(Case("bf16", 2, 64, page, lens, seed=page), 4, window, sinks)


def test_decode_pages_outside_the_window_are_gone():
    lens, page, window, sinks = [700, 90, 400], 16, 100, 5

    def gone(s, c):
        return c * page >= sinks and (c + 1) * page <= lens[s] - window
    run_decode(Case("bf16", 2, 128, page, lens, gone, seed=3), 8, window, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_decode_rows_without_tokens(dtype):
    """Lengths of zero, a missing page, sequences that the table does not have; every row sees nothing."""
    run_decode(Case(dtype, 2, 64, 16, [0, 40, 0, 0, 3, 0], seed=5), 4)
    run_decode(Case(dtype, 2, 64, 16, [40, 33], lambda s, c: s == 0, seed=6), 4)
    run_decode(Case(dtype, 2, 64, 16, [40, 33, 20], seed=7), 4, seqs=[2, -1, 0, 3, 1, 1])
    case = Case(dtype, 2, 64, 16, [17, 30], seed=8)
    case.kv.len.zero_()
    case.lens = [0, 0]
    run_decode(case, 4)


def test_decode_unseen_places_hold_infinities():
    for poison in (np.inf, -np.inf):
        run_decode(Case("bf16", 2, 64, 16, [5, 100, 250], seed=9, poison=poison), 4, 60, 3)
        run_decode(Case("fp32", 2, 64, 64, [5, 100, 250], seed=9, poison=poison), 4, 60, 3)
    case = Case("bf16", 2, 64, 16, [200], seed=10)
    for j in (3, 4, 100, 139):                 # between the sinks and the window, in pages that are read
        case.write(0, j, np.nan, np.inf)
    run_decode(case, 4, 60, 3)


@pytest.mark.parametrize("lens", [[20000], [5000, 1, 9000, 3], [128 * 9] * 7, [1] * 300, list(range(1, 400, 7))])
def test_decode_splits(lens):
    """Long caches cut over many workgroups, many short ones in one, shares that end inside a cache."""
    run_decode(Case("bf16", 1, 32, 64, lens, seed=len(lens)), 2)


@pytest.mark.parametrize("dtype,kv,d", [("bf16", 32, 32), ("fp32", 16, 64), ("bf16", 64, 128)])
@pytest.mark.parametrize("rows", [5, 23, 64, 65, 130])
def test_decode_many_short_rows(dtype, kv, d, rows):
    """Rows of a step or a few, several to a share: whole ones, ones that a share's end cuts, empty ones between them."""
    rng = np.random.default_rng(rows)
    lens = [int(n) for n in rng.choice([0, 1, 17, 31, 32, 33, 64, 90, 150], rows)]
    lens[0], lens[-1] = max(lens[0], 1), 40
    run_decode(Case(dtype, kv, d, 32, lens, seed=rows), kv, *((0, 0) if rows % 2 else (50, 4)))


@pytest.mark.parametrize("dtype,kv,n_q,d,lens", [
    ("bf16", 2, 8, 64, [512, 0, 40, 1, 300]), ("bf16", 2, 8, 64, [513, 0, 40, 1, 300]), ("fp32", 2, 8, 64, [384, 1, 5]), ("fp32", 2, 8, 64, [385, 1, 5]),
    ("bf16", 1, 16, 128, [512, 0, 33, 1, 512]), ("bf16", 1, 16, 128, [0, 513, 33, 1, 512]), ("bf16", 1, 16, 64, [1, 33, 65, 0, 512] * 14),
    ("bf16", 1, 16, 64, [1, 33, 65, 0, 512] * 13 + [2000]), ("fp32", 1, 32, 32, [1, 2, 33, 0, 64] * 103 + [3000]),
    ("bf16", 32, 32, 32, [640, 300, 310, 0, 320, 64, 290, 333, 1, 30]), ("bf16", 32, 32, 32, [300, 673, 310, 0, 320, 64, 290, 333, 1, 30])])
def test_decode_rows_whole_and_cut(dtype, kv, n_q, d, lens):
    """Batches whose rows are a workgroup's each, and such that have one row too long for it; joins by rows and by shares."""
    run_decode(Case(dtype, kv, d, 32, lens, seed=len(lens)), n_q)


def test_decode_large_scores_and_scale():
    """Scores of +-300 in order and against it: the running maximum lags and grows."""
    for order in (1, -1):
        case = Case("fp32", 1, 32, 16, [600], seed=11)
        direction = np.sign(np.random.default_rng(1).standard_normal(32))
        for j in range(600):
            case.k[0][j] = direction * (j if order == 1 else 600 - j) / 64
        full = np.zeros((608, 1, 32)); full[:600] = case.k[0]
        for c in range(38):
            case.kv.K[1, case.table[0, c]] = upload(ko.k_to_pages(full[16 * c:16 * c + 16]), "fp32")
        run_decode(case, 2, scale=1.0, q=np.stack([[direction, -direction]]))
        run_decode(case, 2, scale=0.0)
        run_decode(case, 2, scale=-0.3)


def test_decode_is_the_same_every_time_and_row_by_row():
    case = Case("bf16", 2, 128, 16, [300, 1000, 77], seed=12)
    a, la = run_decode(case, 8)
    b, lb = run_decode(case, 8)
    assert torch.equal(a.view(torch.int16), b.view(torch.int16)) and torch.equal(la, lb)


@pytest.mark.parametrize("dtype,d", WIDTHS)
def test_prefill_widths(dtype, d):
    run_prefill(Case(dtype, 2, d, 16, [1, 16, 17, 77], seed=d), 4, [1, 16, 5, 77], pad=8)


@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 4), (8, 1), (17, 1), (40, 2), (28, 4)])
def test_prefill_head_groups(heads, kv):
    run_prefill(Case("bf16", kv, 64, 32, [33, 70, 150], seed=heads), heads, [33, 1, 40])


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (40, 4), (64, 21), (33, 200), (1000, 4), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_prefill_windows(page, window, sinks):
    run_prefill(Case("bf16", 1, 64, page, [1, 40, 129, 300], seed=page), 2, [1, 40, 129, 70], window, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_prefill_lengths(dtype):
    for n in (1, 15, 16, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200):
        run_prefill(Case(dtype, 1, 64, 16, [n, n + 50], seed=n), 1, [n, n])
    run_prefill(Case(dtype, 1, 64, 16, [30, 1, 2], seed=5), 2, [1, 1, 1], one_row=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_prefill_rows_without_tokens(dtype):
    run_prefill(Case(dtype, 2, 64, 16, [40, 33], lambda s, c: s == 0, seed=6), 4, [40, 10])
    run_prefill(Case(dtype, 2, 64, 16, [40, 33, 20], seed=7), 4, [7, 3, 11, 0, 2], seqs=[2, -1, 0, 1, 9])
    run_prefill(Case(dtype, 2, 64, 16, [10, 33], seed=7), 4, [25, 3])         # more rows than tokens: the first ones have no position
    run_prefill(Case(dtype, 2, 64, 16, [100], lambda s, c: c == 2, seed=8), 2, [100])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 256])
def test_prefill_infinities_and_nan_reach_only_rows_that_see_them(dtype, d):
    """Token 70's values are infinite, 75's NaN, 90's -infinite: rows before them stay finite, rows after them follow the formula."""
    case = Case(dtype, 1, d, 16, [128], seed=13)
    val = case.v[0][70].copy(); val[0, 3] = np.inf; val[0, d - 1] = np.inf
    case.write(0, 70, v=val)
    val = case.v[0][90].copy(); val[0, 7] = -np.inf
    case.write(0, 90, v=val)
    val = case.v[0][75].copy(); val[0, 5] = np.nan
    case.write(0, 75, v=val)
    for window, sinks in ((0, 0), (20, 4)):
        q = rounded(np.random.default_rng(2).standard_normal((128, 2, d)), dtype)
        out = pa.attend_prefill(case.kv, 1, upload(q, dtype), i32(np.array([0, 128])), window=window, sinks=sinks).double().cpu().numpy()
        for i in range(128):
            o, _, mag, big = ko.attend_row(q[i], case.k[0], case.v[0], ko.visible(i, case.there[0], window, sinks), d ** -0.5)
            assert np.array_equal(np.isnan(out[i]), np.isnan(o)), i
            assert np.array_equal(np.isinf(out[i]), np.isinf(o)) and np.array_equal(out[i][np.isinf(o)], o[np.isinf(o)]), i
            fine = np.isfinite(o)
            tol, _ = bounds(dtype, d, 128, np.where(fine, o, 0), np.zeros(2), np.where(np.isfinite(mag), mag, 0), big)
            assert np.all(np.abs(out[i][fine] - o[fine]) <= tol[fine]), i


def test_prefill_long_and_shared():
    """Several tiles of rows and many of tokens, heads that share, a window in the middle of it."""
    run_prefill(Case("bf16", 2, 128, 16, [700, 333], seed=14), 8, [700, 130])
    run_prefill(Case("bf16", 1, 128, 64, [900], seed=15), 4, [500], 256, 4)


def test_prefill_few_rows_over_a_long_cache():
    run_prefill(Case("bf16", 1, 64, 64, [6000, 200], seed=16), 4, [5, 3])
    run_prefill(Case("fp32", 1, 32, 16, [3000], seed=17), 2, [9], 2500, 4)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (700, 40), (256, 4)])
def test_prefill_splits_of_long_caches(dtype, window, sinks):
    """Tokens cut over several workgroups: caches of which one, some and all cuts are used, rows that see nothing, many prompts."""
    assert int(pa.lib().parse_attend_prefill_workspace_bytes(Case(dtype, 2, 64, 16, [2100], seed=1).kv.c(), 4, 40, 1)) > 0
    run_prefill(Case(dtype, 2, 64, 16, [2100, 250, 20, 700], lambda s, c: s == 3, seed=19), 4, [40, 64, 30, 3], window, sinks)
    run_prefill(Case(dtype, 1, 160, 64, [1500], seed=20), 1, [130], window, sinks)
    lens = [1 + 37 * i % 600 for i in range(70)]
    run_prefill(Case(dtype, 1, 32, 32, lens, seed=21), 2, [1 + i % 2 if n > 1 else 1 for i, n in enumerate(lens)], window, sinks)


def test_prefill_split_rows_meet_infinities():
    """A row tile whose cut is worked on twice (values that are infinite for some of its rows only) beside cuts that are not."""
    case = Case("bf16", 1, 64, 16, [1000], seed=22)
    val = case.v[0][990].copy(); val[0, 3] = np.inf
    case.write(0, 990, v=val)
    q = rounded(np.random.default_rng(2).standard_normal((20, 2, 64)), "bf16")
    out = pa.attend_prefill(case.kv, 1, upload(q, "bf16"), i32(np.array([0, 20]))).double().cpu().numpy()
    for t in range(20):
        o, _, mag, big = ko.attend_row(q[t], case.k[0], case.v[0], ko.visible(980 + t, case.there[0], 0, 0), 0.125)
        assert np.array_equal(np.isinf(out[t]), np.isinf(o)) and not np.isnan(out[t]).any(), t
        fine = np.isfinite(o)
        tol, _ = bounds("bf16", 64, 1000, np.where(fine, o, 0), np.zeros(2), np.where(np.isfinite(mag), mag, 0), big)
        assert np.all(np.abs(out[t][fine] - o[fine]) <= tol[fine]), t


def test_prefill_of_single_tokens_equals_decode():
    case = Case("bf16", 2, 64, 16, [100, 5, 333], seed=18)
    q = upload(rounded(np.random.default_rng(3).standard_normal((3, 4, 64)), "bf16"), "bf16")
    a = pa.attend_decode(case.kv, 1, q).float()
    b = pa.attend_prefill(case.kv, 1, q).float()
    assert (a - b).abs().max() <= 2.0 ** -6 * a.abs().max()


# ---- the rows' way in -------------------------------------------------------------------------------------------------
def rope_table(n, d):
    angle = np.arange(n)[:, None] * 10000.0 ** (-np.arange(d // 2) / (d // 2))
    return np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,page,rope,in_place", [(64, 16, True, False), (32, 32, True, True), (128, 64, False, False), (160, 16, True, True), (256, 256, True, False)])
def test_append(dtype, d, page, rope, in_place):
    rng = np.random.default_rng(d + page)
    n_kv, n_q, lens, new, seqs = 2, 6, [40, 17, 300, 16, 9], [5, 17, 100, 0, 1], [3, 0, 2, 1, 4]
    table = np.full((5, 300 // page + 2), -1, np.int32)
    ids = iter(rng.permutation(60))
    seq_len = [0] * 5
    for p, s in enumerate(seqs):
        seq_len[s] = lens[p]
        for c in range(-(-lens[p] // page)):
            table[s, c] = next(ids)
    table[2, 250 // page] = -1                                     # a page that is not there
    off = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    rows = int(off[-1])
    kv = pa.KV(torch.full((2, 60, n_kv, page // 16, d // 8, 16, 8), 7.0, device=DEV, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32),
               torch.full((2, 60, n_kv, page // 8, d, 8), 7.0, device=DEV, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32),
               i32(table), i32(np.array(seq_len)))
    x = rounded(rng.standard_normal((rows, n_q + 2 * n_kv, d)), dtype)
    fused = upload(x, dtype)
    table_rope = rope_table(290, d)                                # shorter than the longest sequence: the last row serves
    q = fused[:, :n_q]
    q_out = q if in_place else torch.empty((rows, n_q, d), dtype=fused.dtype, device=DEV)
    pa.kv_append(kv, 1, fused[:, n_q:n_q + n_kv], fused[:, n_q + n_kv:], i32(off), i32(np.array(seqs)), q=q, q_out=q_out,
                 rope=torch.from_numpy(table_rope).to(DEV) if rope else None)
    pos = np.concatenate([lens[p] - n + np.arange(n) for p, n in enumerate(new)])
    turn = table_rope[np.clip(pos, 0, 289)].astype(np.float64)
    qk = ko.rotate(x[:, :n_q + n_kv], turn) if rope else x[:, :n_q + n_kv]
    size = ko.rotate(np.abs(x[:, :n_q + n_kv]), np.abs(turn) * np.repeat([[1.0, -1.0]], d // 2, 1).reshape(1, -1)) if rope else np.abs(qk)
    size = np.abs(np.concatenate([np.abs(x[:, :n_q + n_kv, :d // 2]) + np.abs(x[:, :n_q + n_kv, d // 2:])] * 2, 2)) if rope else size
    tol = 2.0 ** -23 * size + (1.01 * 2.0 ** -8 * np.abs(qk) if dtype == "bf16" else 0)
    assert np.all(np.abs(q_out.double().cpu().numpy() - qk[:, :n_q]) <= tol[:, :n_q])
    if not in_place:
        assert np.array_equal(fused.double().cpu().numpy(), x)
    assert bool((kv.K[0] == 7).all()) and bool((kv.V[0] == 7).all()), "another layer was written"
    K = ko.k_from_pages(kv.K[1].double().cpu().numpy())
    V = ko.v_from_pages(kv.V[1].double().cpu().numpy())
    touched = np.zeros((60, page), bool)
    for p, n in enumerate(new):
        for t in range(n):
            j, r = lens[p] - n + t, off[p] + t
            id_ = table[seqs[p], j // page]
            if id_ < 0:
                continue
            touched[id_, j % page] = True
            assert np.all(np.abs(K[id_, j % page] - qk[r, n_q:]) <= tol[r, n_q:]), (p, t)
            assert np.array_equal(V[id_, j % page], x[r, n_q + n_kv:]), (p, t)
    assert np.all(K[~touched] == 7) and np.all(V[~touched] == 7), "a place of no new token was written"


def test_append_of_single_rows_without_offsets_or_q():
    kv = pa.KV.empty(1, 8, 16, 3, 64, 4, 2)
    pa.kv_reserve(kv, i32(np.array([1, 0, 17, 2])))
    k = torch.randn((4, 3, 64), device=DEV).bfloat16(); v = torch.randn((4, 3, 64), device=DEV).bfloat16()
    assert pa.kv_append(kv, 0, k, v) is None                       # sequence 1 is empty: its row has no position
    table = kv.table.cpu().numpy()
    K = ko.k_from_pages(kv.K[0].float().cpu().numpy()); V = ko.v_from_pages(kv.V[0].float().cpu().numpy())
    for s, j in ((0, 0), (2, 16), (3, 1)):
        assert np.array_equal(K[table[s, j // 16], j % 16], k[s].float().cpu().numpy())
        assert np.array_equal(V[table[s, j // 16], j % 16], v[s].float().cpu().numpy())


# ---- bookkeeping --------------------------------------------------------------------------------------------------------
class Both:
    """The same calls on the device and on the oracle, everything compared after each."""

    def __init__(self, n_seqs, max_pages, n_pages, page, layers=2, dtype=torch.bfloat16, n_kv=2, d=32, seed=0):
        self.kv = pa.KV.empty(layers, n_pages, page, n_kv, d, n_seqs, max_pages, dtype)
        gen = torch.Generator(device=DEV); gen.manual_seed(seed)
        self.kv.K.copy_(torch.randn(self.kv.K.shape, generator=gen, device=DEV)); self.kv.V.copy_(torch.randn(self.kv.V.shape, generator=gen, device=DEV))
        self.K, self.V = self.kv.K.cpu().clone(), self.kv.V.cpu().clone()
        self.o = ko.Pages(n_seqs, max_pages, n_pages, page)
        self.wbuf, self.ws = guarded_bytes(int(pa.lib().parse_kv_workspace_bytes(self.kv.c())))
        self.check()

    def check(self):
        torch.cuda.synchronize()
        assert np.array_equal(self.kv.table.cpu().numpy(), self.o.table)
        assert np.array_equal(self.kv.len.cpu().numpy(), self.o.len)
        assert np.array_equal(self.kv.refs.cpu().numpy(), self.o.refs)
        assert np.array_equal(self.kv.free_bits.cpu().numpy().view(np.uint32), self.o.free_words())
        assert torch.equal(self.kv.K.cpu(), self.K) and torch.equal(self.kv.V.cpu(), self.V)
        check_guards(self.wbuf, "workspace")

    def copied(self, copies):
        for a, b in copies:
            self.K[:, b], self.V[:, b] = self.K[:, a].clone(), self.V[:, a].clone()

    def reserve(self, n_new):
        served = pa.kv_reserve(self.kv, i32(np.array(n_new)), workspace=self.ws)
        copies, want = self.o.reserve(n_new)
        self.copied(copies)
        assert np.array_equal(served.cpu().numpy(), want)
        self.check()
        return len(copies), int(want.sum())

    def fork(self, src, dst):
        pa.kv_fork(self.kv, i32(np.array(src)), i32(np.array(dst)))
        self.o.fork(src, dst)
        self.check()

    def trim(self, keep=None, window=0, sinks=0):
        pa.kv_trim(self.kv, None if keep is None else i32(np.array(keep)), window, sinks)
        self.o.trim(keep, window, sinks)
        self.check()

    def compact(self):
        n = pa.kv_compact(self.kv, workspace=self.ws)
        moves, live = self.o.compact()
        self.copied(moves)
        assert int(n.item()) == live
        self.check()
        return len(moves)


def test_pages_of_forks_and_copies():
    b = Both(8, 10, 40, 16)
    b.reserve([20, 16, 0, 0, 0, 0, 0, 0])
    b.fork([0, 0, 1], [2, 3, 4])
    assert b.reserve([1, 1, 1, 1, 1, 0, 0, 0]) == (2, 5)           # three users of a begun page: two copies, the last one keeps it
    b.fork([2, 3, 0], [0, 2, 3])                                    # a cycle
    b.fork([0, 1], [0, 5])                                          # onto itself: nothing
    b.trim([5, 0, 100, -3, 16, 17, 0, 0])
    b.reserve([100, 100, 1, 0, 16, 1, 161, 160])                    # the last but one outgrows the table and takes nothing
    b.compact()
    b.trim(window=20, sinks=3)
    b.reserve([3] * 8)
    b.compact()
    b.compact()


def test_pages_run_out():
    b = Both(6, 8, 5, 16)
    assert b.reserve([16, 33, 16, 0, 1, 0]) == (0, 3)               # 1 + 3 + 1 pages; nothing is left for the fifth
    b.trim([0, 33, 16, 0, 0, 0])
    b.reserve([0, 0, 40, 5, 0, 1])                                  # the first does not fit: the ones behind it get nothing either
    b.reserve([0, 15, 0, 5, 0, 1])                                  # room in a begun page needs no page


@pytest.mark.parametrize("seed", range(6))
def test_pages_random_histories(seed):
    rng = np.random.default_rng(seed)
    n_seqs = int(rng.choice([3, 30, 70])); max_pages = int(rng.choice([5, 9, 17])); n_pages = int(rng.choice([31, 64, 200]))
    b = Both(n_seqs, max_pages, n_pages, 16, layers=1, n_kv=1, seed=seed)
    for _ in range(25):
        what = rng.integers(5)
        if what <= 1:
            b.reserve(np.where(rng.random(n_seqs) < 0.4, rng.integers(-1, 40, n_seqs), 0))
        elif what == 2:
            n = int(rng.integers(1, n_seqs + 1))
            b.fork(rng.integers(0, n_seqs, n), rng.permutation(n_seqs)[:n])
        elif what == 3:
            b.trim(np.where(rng.random(n_seqs) < 0.3, rng.integers(0, 60, n_seqs), 1000), int(rng.choice([0, 1, 30])), int(rng.choice([0, 4, 20])))
        else:
            b.compact()


def test_pages_many():
    """More sequences than threads, more words of free pages than threads."""
    b = Both(2500, 3, 70000, 16, layers=1, n_kv=1, d=32)
    rng = np.random.default_rng(4)
    b.reserve(rng.integers(0, 40, 2500))
    b.fork(np.arange(1000), 1500 + np.arange(1000))
    b.reserve(np.where(np.arange(2500) % 3, 1, 0))
    b.trim(np.where(np.arange(2500) % 2, 1000, 0))
    b.compact()
    b.reserve(np.full(2500, 2))


def test_fork_skips_sequences_that_are_not_there():
    b = Both(4, 4, 20, 16)
    b.reserve([20, 30, 0, 0])
    pa.kv_fork(b.kv, i32(np.array([0, 9, 1, -1])), i32(np.array([2, 3, 4, 0])))
    b.o.fork([0], [2])
    b.check()


def test_copies_of_wide_pages_and_fp32():
    for dtype, n_kv, d, page in ((torch.bfloat16, 3, 160, 32), (torch.float32, 2, 32, 16), (torch.bfloat16, 1, 32, 16)):
        b = Both(4, 4, 20, page, layers=3, dtype=dtype, n_kv=n_kv, d=d)
        b.reserve([page + 1, 5, 0, 0])
        b.fork([0, 1], [2, 3])
        b.reserve([1, 1, 1, 1])
        b.trim([0, 100, 100, 0])
        assert b.compact() > 0


def test_a_step_is_recorded_and_replayed():
    """reserve, append, decode and trim as one HIP graph: every replay equals the eager step on a copy of the state."""
    torch.manual_seed(0)
    n_seqs, n_kv, n_q, d = 3, 2, 4, 64

    def fresh():
        kv = pa.KV.empty(1, 40, 16, n_kv, d, n_seqs, 12)
        kv.K.zero_(); kv.V.zero_()
        return kv
    qkv = torch.randn((n_seqs, n_q + 2 * n_kv, d), device=DEV).bfloat16()
    one = i32(np.ones(n_seqs))
    rope = torch.from_numpy(rope_table(200, d)).to(DEV)

    def make(kv):
        ws, wa = pa.kv_workspace(kv), pa.attend_decode_workspace(kv, n_q, n_seqs)
        served, q, out = torch.empty(n_seqs, dtype=torch.int32, device=DEV), torch.empty((n_seqs, n_q, d), dtype=torch.bfloat16, device=DEV), torch.empty((n_seqs, n_q, d), dtype=torch.bfloat16, device=DEV)

        def step():
            pa.kv_reserve(kv, one, served, ws)
            pa.kv_append(kv, 0, qkv[:, n_q:n_q + n_kv], qkv[:, n_q + n_kv:], q=qkv[:, :n_q], q_out=q, rope=rope)
            pa.attend_decode(kv, 0, q, window=30, sinks=2, out=out, workspace=wa)
            pa.kv_trim(kv, None, 30, 2)
        return step, out
    a, b = fresh(), fresh()
    step_a, out_a = make(a)
    step_b, out_b = make(b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step_a()                                                   # warm-up, on another stream
    torch.cuda.current_stream().wait_stream(side)
    step_b()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step_a()
    for i in range(60):
        qkv.normal_()
        graph.replay()
        step_b()
        torch.cuda.synchronize()
        assert torch.equal(out_a.view(torch.int16), out_b.view(torch.int16)), i
        assert torch.equal(a.table, b.table) and torch.equal(a.len, b.len) and torch.equal(a.refs, b.refs) and torch.equal(a.free_bits, b.free_bits)
    assert int(a.len[0]) == 61 and int((a.refs > 0).sum()) < 3 * 4 + 1


def test_long_cache_past_32_bits():
    """Elements past 2^31 in a layer, and a second layer behind it: the same tokens at low and at high page ids give the same bits."""
    n_kv, d, page, n_pages = 16, 128, 256, 4608                    # 2.4e9 elements a layer
    kv = pa.KV(torch.zeros((2, n_pages, n_kv, page // 16, d // 8, 16, 8), dtype=torch.bfloat16, device=DEV),
               torch.zeros((2, n_pages, n_kv, page // 8, d, 8), dtype=torch.bfloat16, device=DEV), i32(np.array([[0, 1], [n_pages - 1, n_pages - 2]])),
               i32(np.array([0, 0])))
    rows = 300
    x = torch.randn((rows, 3 * n_kv, d), device=DEV).bfloat16()
    kv.len.fill_(rows)
    off = i32(np.array([0, rows]))
    outs = []
    for s in (0, 1):
        seqs = i32(np.array([s]))
        pa.kv_append(kv, 1, x[:, n_kv:2 * n_kv], x[:, 2 * n_kv:], off, seqs)
        outs.append((pa.attend_prefill(kv, 1, x[:, :n_kv], off, seqs), pa.attend_decode(kv, 1, x[-1:, :n_kv], seqs)))
    for a, b in zip(*outs):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16)) and bool(a.float().abs().sum() > 0)
    assert not bool(kv.K[0].any()) and int((kv.K[1].flatten(1).any(1)).sum()) == 4
    # a copy between the ends
    kv.refs, kv.free_bits = torch.zeros(n_pages, dtype=torch.int32, device=DEV), torch.zeros(n_pages // 32, dtype=torch.int32, device=DEV)
    kv.table.fill_(-1); kv.table[1, 0] = n_pages - 1; kv.refs[n_pages - 1] = 1
    kv.free_bits.fill_(-1); kv.free_bits[-1] = 2 ** 31 - 1
    assert int(pa.kv_compact(kv)) == 1
    assert torch.equal(kv.K[1, 0], kv.K[1, n_pages - 1]) and int(kv.table[1, 0]) == 0


def test_the_example_serves_a_block():
    """Projections, cache and attention together: prompts, samples that share pages, a recorded step; every step's attention against a plain one."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_block.py")
    spec = importlib.util.spec_from_file_location("serve_block", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    r = m.run(hidden=512, heads=8, kv_heads=4, prompts=2, length=70, samples=3, steps=40, groups=8, gs=32, k=4, window=48, sinks=4, check=True)
    # weights rounded as two halves, the result once (2^-8); the plain form in 32 bits
    assert r["worst"] <= 2.0 ** -7 and r["steps"] == 40 and bool(torch.isfinite(r["x"].float()).all())
    assert r["lengths"] == [0, 0] + [110] * 3 + [73] * 3


SEEN = [("bf16", 2, 8, 64, [1, 3, 40, 77, 200]), ("fp32", 2, 8, 64, [1, 3, 40, 77, 200]),          # a workgroup a row
        ("bf16", 32, 32, 32, [33, 1, 64, 90, 17, 150, 40, 31] * 9), ("fp32", 16, 16, 64, [33, 1, 64, 90, 17, 150, 40, 31] * 9),      # a wavefront a row
        ("bf16", 2, 8, 64, [5000, 7]), ("fp32", 2, 8, 64, [5000, 7]),                              # joined by the workgroup that comes last
        ("bf16", 1, 16, 128, [5000, 900]), ("bf16", 2, 8, 256, [600, 40])]                         # joined by a second launch; wide heads


@pytest.mark.parametrize("dtype,kv,n_q,d,lens", SEEN)
@pytest.mark.parametrize("window,sinks", [(0, 0), (30, 4)])
def test_decode_infinities_and_nan_that_are_seen(dtype, kv, n_q, d, lens, window, sinks):
    """An infinity of V that a row sees comes out as it is, whatever its weight's rounding left; both signs in a column, and NaN, give NaN; the other
    columns stay finite.  Some of the tokens lie outside the window: those reach nothing."""
    case = Case(dtype, kv, d, 16, lens, seed=len(lens) + d)
    for s, n in enumerate(lens):
        for j, columns in ((n // 3, {3: np.inf, 9: np.inf}), (2 * n // 3, {7: -np.inf, 9: -np.inf}), (n // 2, {5: np.nan}), (n - 1, {11: np.inf, d - 1: -np.inf})):
            v = case.v[s][j].copy()
            for c, x in columns.items():
                v[:, c] = x
            case.write(s, j, v=v)
    q = rounded(np.random.default_rng(2).standard_normal((len(lens), n_q, d)), dtype)
    out, lse = pa.attend_decode(case.kv, 1, upload(q, dtype), window=window, sinks=sinks, with_lse=True)
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for s, n in enumerate(lens):
        with np.errstate(invalid="ignore"):
            o, l, mag, big = ko.attend_row(q[s], case.k[s], case.v[s], ko.visible(n - 1, case.there[s], window, sinks), d ** -0.5)
        assert np.array_equal(np.isnan(out[s]), np.isnan(o)), s
        assert np.array_equal(np.isinf(out[s]), np.isinf(o)) and np.array_equal(out[s][np.isinf(o)], o[np.isinf(o)]), s
        fine = np.isfinite(o)
        tol, ltol = bounds(dtype, d, n, np.where(fine, o, 0), l, np.where(np.isfinite(mag), mag, 0), big)
        assert np.all(np.abs(out[s][fine] - o[fine]) <= tol[fine]) and np.all(np.abs(lse[s] - l) <= ltol), s


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("window,sinks", [(2 ** 31 - 1, 0), (2 ** 31 - 1, 4), (2 ** 31 - 12, 0)])
def test_prefill_rows_before_the_first_token_with_a_window_without_end(dtype, window, sinks):
    """More rows than tokens: the first rows' positions lie below 0, and their window's begin below what 32 bits hold."""
    run_prefill(Case(dtype, 2, 64, 16, [10, 33], seed=7), 4, [25, 3], window, sinks)
    run_prefill(Case(dtype, 1, 64, 16, [700, 5], seed=8), 1, [760, 5], window, sinks)


@pytest.mark.parametrize("n_seqs", [4, 1500])
def test_a_sequence_without_room_leaves_its_pages_as_they_are(n_seqs):
    """Forks of a begun page in a pool that runs out: the list that reserve gives keeps append and attention away from the sequences that got nothing."""
    n_kv, d, page = 2, 32, 16
    kv = pa.KV.empty(1, 3, page, n_kv, d, n_seqs, 4)
    kv.K.zero_(); kv.V.zero_()
    want = np.zeros(n_seqs, np.int32); want[[0, 1]] = [5, 16]
    placed = i32(np.array([7, 7]))
    pa.kv_reserve(kv, i32(want), seqs_served=placed)
    assert placed.tolist() == [0, 1]
    rows = torch.randn((21, n_kv, d), device=DEV).bfloat16()
    pa.kv_append(kv, 0, rows, rows, i32(np.array([0, 5, 21])), placed)
    pa.kv_fork(kv, i32(np.array([0, 0])), i32(np.array([2, n_seqs - 1])))      # one free page: the first of the three gets a copy, the second nothing
    one = np.zeros(n_seqs, np.int32); one[[0, 2, n_seqs - 1]] = 1
    K, V = kv.K.clone(), kv.V.clone()
    served = torch.empty(n_seqs, dtype=torch.int32, device=DEV)
    seqs = i32(np.array([n_seqs - 1, 2, 0, 1, -5, n_seqs, 2]))
    room = torch.full_like(seqs, 9)
    pa.kv_reserve(kv, i32(one), served, seqs=seqs, seqs_served=room)
    assert np.flatnonzero(served.cpu().numpy()).tolist() == [0] and room.tolist() == [-1, -1, 0, -1, -1, -1, -1] and seqs.tolist()[0] == n_seqs - 1
    q = torch.randn((7, 4, d), device=DEV).bfloat16()
    new = torch.randn((7, n_kv, d), device=DEV).bfloat16()
    pa.kv_append(kv, 0, new, new, seqs=room)
    out, lse = pa.attend_decode(kv, 0, q, room, with_lse=True)
    mine, shared = int(kv.table[0, 0]), int(kv.table[2, 0])
    assert mine == 2 and shared == 0 and kv.len[[0, 2, n_seqs - 1]].tolist() == [6, 5, 5]
    assert torch.equal(kv.K[:, :2], K[:, :2]) and torch.equal(kv.V[:, :2], V[:, :2]), "a page of others was written"
    assert np.array_equal(ko.k_from_pages(kv.K[0, mine].float().cpu().numpy())[5], new[2].float().cpu().numpy())
    empty = [0, 1, 3, 4, 5, 6]
    assert not bool(out[empty].any()) and bool(torch.isneginf(lse[empty]).all()) and bool(torch.isfinite(lse[2]).all())
    # the list over the one that it is made of
    pa.kv_trim(kv, i32(np.where(np.arange(n_seqs) == 1, 0, 100)))
    pa.kv_reserve(kv, i32(one - (np.arange(n_seqs) == 0)), seqs=seqs, seqs_served=seqs)
    assert seqs.tolist() == [n_seqs - 1, 2, -1, -1, -1, -1, 2]


@pytest.mark.parametrize("first", [0, 16])
def test_reserve_of_more_pages_than_32_bits_count(first):
    """4096 sequences that ask for whole rows of a table of 2^25 tokens: 2^33 pages of sixteen.  (The table's 34 GB are not touched: nobody has a token.)"""
    n_seqs, columns = 4096, 1 << 21
    kv = pa.KV(torch.zeros((1, 64, 1, 1, 4, 16, 8), dtype=torch.bfloat16, device=DEV), torch.zeros((1, 64, 1, 2, 32, 8), dtype=torch.bfloat16, device=DEV),
               torch.empty((n_seqs, columns), dtype=torch.int32, device=DEV), torch.zeros(n_seqs, dtype=torch.int32, device=DEV),
               torch.zeros(64, dtype=torch.int32, device=DEV), torch.full((2,), -1, dtype=torch.int32, device=DEV))
    want = np.full(n_seqs, 1 << 25, np.int32)
    want[0] = first                                                # one page, or no token
    want[4000:] = 1
    room = torch.empty(n_seqs, dtype=torch.int32, device=DEV)
    wbuf, ws = guarded_bytes(int(pa.lib().parse_kv_workspace_bytes(kv.c())))
    served = pa.kv_reserve(kv, i32(want), workspace=ws, seqs_served=room)
    check_guards(wbuf, "workspace")
    got = [0] if first else []
    assert np.flatnonzero(served.cpu().numpy()).tolist() == got and np.flatnonzero(room.cpu().numpy() >= 0).tolist() == got
    assert int(kv.len[0]) == first and not bool(kv.len[1:].any())
    assert kv.refs.tolist() == [len(got)] + [0] * 63 and kv.free_bits.tolist() == [-1 - len(got), -1]
    del kv
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("sign", [1, -1])
def test_values_near_the_type_s_largest(dtype, sign):
    """Scores of 0, then of 7.5 in powers of two, which is less than the running maximum may lag by: the sums hold 8 values of 1e37 and
    128 of 2^-7.5 of that, as they do with weights of at most 1."""
    n, d = 136, 32
    k, v = np.zeros((n, 1, d)), np.full((n, 1, d), sign * 1e37)
    k[128:, 0, 0] = 7.5
    case = Case(dtype, 1, d, 16, [n], seed=1)
    for j in range(n):
        case.write(0, j, k[j], rounded(v[j], dtype))
    q = np.zeros((1, 1, d)); q[0, 0, 0] = 1
    want = ko.attend_row(q[0], case.k[0], case.v[0], np.ones(n, bool), np.log(2.0))
    for out, lse in (pa.attend_decode(case.kv, 1, upload(q, dtype), scale=np.log(2.0), with_lse=True),
                     pa.attend_prefill(case.kv, 1, upload(q, dtype), scale=np.log(2.0), with_lse=True)):
        compare(case, out, lse, [(*want, n)], d)


@pytest.mark.parametrize("dtype,P,offsets", [("bf16", 64, True), ("bf16", 65, True), ("fp32", 65, True), ("bf16", 130, True), ("fp32", 300, True), ("bf16", 300, False),
                                             ("fp32", 70, False), ("bf16", 1000, True)])
def test_append_of_many_prompts(dtype, P, offsets):
    """Prompts that a workgroup finds by sums in LDS: empty ones, missing pages, sequences that the table does not have, several blocks a workgroup."""
    rng = np.random.default_rng(P)
    n_kv, n_q, d, page = 2, 3, 32, 16
    lens = rng.integers(1, 90, P)
    new = np.minimum(rng.choice([0, 1, 2, 15, 16, 17, 40], P), lens) if offsets else np.ones(P, np.int64)
    seqs = rng.permutation(P)                                      # prompt p is the table's row seqs[p]
    counts = -(-lens // page)
    ids = rng.permutation(int(counts.sum()))
    table, n, at = np.full((P, int(counts.max()) + 1), -1, np.int32), np.zeros(P, np.int32), 0
    for p in range(P):
        table[seqs[p], :counts[p]] = ids[at:at + counts[p]]; at += counts[p]
        n[seqs[p]] = lens[p]
    table[seqs[P // 2], counts[P // 2] - 1] = -1                   # the page of a prompt's last tokens is not there
    named = seqs.astype(np.int32); named[3], named[P - 5] = -1, P   # two prompts of no sequence
    off = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    rows = int(off[-1])
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    kv = pa.KV(torch.full((1, at, n_kv, 1, d // 8, 16, 8), 7.0, device=DEV, dtype=dt), torch.full((1, at, n_kv, 2, d, 8), 7.0, device=DEV, dtype=dt), i32(table), i32(n))
    x = rounded(rng.standard_normal((rows, n_q + 2 * n_kv, d)), dtype)
    fused, turn = upload(x, dtype), rope_table(90, d)
    buf, _, q_out = guarded(rows, n_q, d, fused, 16)
    pa.kv_append(kv, 0, fused[:, n_q:n_q + n_kv], fused[:, n_q + n_kv:], i32(off) if offsets else None, i32(named), q=fused[:, :n_q], q_out=q_out,
                 rope=torch.from_numpy(turn).to(DEV))
    check_guards(buf, "q_out")
    known = (named >= 0) & (named < P)
    pos = np.concatenate([np.where(known[p], lens[p] - new[p] + np.arange(new[p]), 0) for p in range(P)]).astype(int)
    angles = turn[pos].astype(np.float64)
    qk = ko.rotate(x[:, :n_q + n_kv], angles)
    # two products and a sum in 32 bits, the result rounded to the type
    tol = 2.0 ** -23 * np.concatenate([np.abs(x[:, :n_q + n_kv, :d // 2]) + np.abs(x[:, :n_q + n_kv, d // 2:])] * 2, 2) + (1.01 * 2.0 ** -8 * np.abs(qk) if dtype == "bf16" else 0)
    assert np.all(np.abs(q_out.double().cpu().numpy() - qk[:, :n_q]) <= tol[:, :n_q])
    K, V = ko.k_from_pages(kv.K[0].double().cpu().numpy()), ko.v_from_pages(kv.V[0].double().cpu().numpy())
    touched = np.zeros((at, page), bool)
    for p in np.flatnonzero(known):
        for t in range(new[p]):
            j, r = lens[p] - new[p] + t, off[p] + t
            id_ = table[seqs[p], j // page]
            if id_ < 0:
                continue
            touched[id_, j % page] = True
            assert np.all(np.abs(K[id_, j % page] - qk[r, n_q:]) <= tol[r, n_q:]) and np.array_equal(V[id_, j % page], x[r, n_q + n_kv:]), (p, t)
    assert np.all(K[~touched] == 7) and np.all(V[~touched] == 7), "a place of no new token was written"


@pytest.mark.parametrize("kv,n_q,d,lens,short", [(2, 8, 64, [300, 1, 77], True), (8, 8, 128, [40, 90, 33, 64] * 16, True), (1, 4, 32, [9000], False),
                                                 (1, 16, 128, [3000], False), (1, 2, 256, [500], False)])
def test_decode_keeps_what_the_rounding_of_a_weight_leaves(kv, n_q, d, lens, short):
    """bf16: a weight is multiplied as two bf16 numbers, 2^-16 of it lost at most; only the result is rounded to 2^-8.  Values whose mean is near 0 show the
    difference: with weights of one bf16 number the oracle itself is outside this bound, where rows are short (the bound grows with their number of sums)."""
    case = Case("bf16", kv, d, 16, lens, seed=n_q)
    q = rounded(np.random.default_rng(4).standard_normal((len(lens), n_q, d)), "bf16")
    out = pa.attend_decode(case.kv, 1, upload(q, "bf16")).double().cpu().numpy()
    over = 0
    for s, n in enumerate(lens):
        o, l, mag, big = ko.attend_row(q[s], case.k[s], case.v[s], case.there[s], d ** -0.5)
        tol, _ = bounds("fp32", d, n, o, l, mag, big)
        tol = tol + 1.01 * 2.0 ** -16 * mag + 1.01 * 2.0 ** -8 * (np.abs(o) + tol + 1.01 * 2.0 ** -16 * mag)
        assert np.all(np.abs(out[s] - o) <= tol), s
        for h in range(n_q):
            g = h // (n_q // kv)
            score = d ** -0.5 * (case.k[s][:, g] @ q[s, h])
            p = np.exp(score - score.max())
            over += int((np.abs(rounded(p, "bf16") @ case.v[s][:, g] / p.sum() - o[h]) > tol[h] - 1.01 * 2.0 ** -8 * np.abs(o[h])).sum())
    assert over > 0 or not short


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("window,sinks", [(2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (33, 2 ** 31 - 1)])
def test_decode_with_the_largest_window_and_sinks(dtype, window, sinks):
    run_decode(Case(dtype, 2, 64, 16, [1, 31, 32, 33, 40, 500, 1025], seed=3), 4, window, sinks)
