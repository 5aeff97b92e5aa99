"""Checks of the shared and selected attention and of the norm that need no GPU: every call refuses what it cannot take before anything is launched, and the
oracle is pinned to hand-computed values."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import step_oracle as so

pa = pytest.importorskip("paper_2605_08568_amd")
from test_kv_boundary import BAD_CACHES, EALIGN, EINVAL, ESHAPE, EWORKSPACE, FAKE, ODD, cache  # noqa: E402


def calls():
    L = pa.lib()
    ok = dict(layer=1, q=FAKE, qs=512, n_q=8, rows=3, seqs=FAKE, plan=FAKE, planb=1 << 40, scale=1.0, window=8, sinks=2, out=FAKE, outs=512, lse=FAKE, ws=FAKE, wsb=1 << 40,
              bounds=FAKE, off=FAKE, P=3, top=4, first=1, last=1, pages=FAKE)

    def wrap(f):
        def call(kv=None, **kw):
            return f(kv if kv is not None else cache(), {**ok, **kw})
        return call
    return {
        "plan": wrap(lambda kv, a: L.parse_shared_plan(kv, a["n_q"], a["rows"], a["seqs"], a["window"], a["sinks"], a["plan"], a["planb"], None)),
        "shared": wrap(lambda kv, a: L.parse_attend_shared(kv, a["layer"], a["q"], a["qs"], a["n_q"], a["rows"], a["seqs"], a["plan"], a["planb"], a["scale"], a["window"], a["sinks"],
                                                           a["out"], a["outs"], a["lse"], a["ws"], a["wsb"], None)),
        "bounds": wrap(lambda kv, a: L.parse_kv_bounds(kv, a["bounds"], a["layer"], a["off"], a["seqs"], a["P"], None)),
        "select": wrap(lambda kv, a: L.parse_select_pages(kv, a["bounds"], a["layer"], a["q"], a["qs"], a["n_q"], a["rows"], a["seqs"], a["top"], a["first"], a["last"],
                                                          a["pages"], a["ws"], a["wsb"], None)),
        "pages": wrap(lambda kv, a: L.parse_attend_pages(kv, a["layer"], a["q"], a["qs"], a["n_q"], a["rows"], a["seqs"], a["pages"], a["top"], a["scale"], a["out"],
                                                         a["outs"], a["lse"], a["ws"], a["wsb"], None)),
    }


def refused(call, status, bads):
    for bad in bads:
        assert call(**bad) == status, bad


def test_every_call_refuses_bad_caches():
    for name, call in calls().items():
        for bad, status in BAD_CACHES:
            assert call(cache(**bad)) == status, (name, bad)
    L = pa.lib()
    for bad in (cache(page=8), cache(d=40)):
        assert L.parse_shared_plan_bytes(bad, 8, 3) == 0 and L.parse_attend_shared_workspace_bytes(bad, 8, 3) == 0 and L.parse_kv_bounds_bytes(bad) == 0
        assert L.parse_select_pages_workspace_bytes(bad, 8, 3) == 0 and L.parse_attend_pages_workspace_bytes(bad, 8, 3, 4) == 0


@pytest.mark.parametrize("name", ["shared", "pages"])
def test_attention_refuses_bad_arguments(name):
    c = calls()[name]
    refused(c, EINVAL, [dict(q=None), dict(out=None), dict(n_q=0), dict(rows=0), dict(layer=-1), dict(scale=float("nan")), dict(scale=float("inf"))])
    refused(c, ESHAPE, [dict(layer=2), dict(n_q=6, qs=512), dict(qs=504), dict(outs=504), dict(n_q=65540), dict(rows=4097), dict(rows=4, seqs=None)])
    refused(c, EALIGN, [dict(q=ODD), dict(out=ODD), dict(lse=ODD), dict(seqs=ODD), dict(q=FAKE + 8), dict(qs=516), dict(outs=516), dict(ws=ODD)])
    refused(c, EWORKSPACE, [dict(ws=None), dict(wsb=0)])
    L = pa.lib()
    if name == "shared":
        assert c(wsb=L.parse_attend_shared_workspace_bytes(cache(), 8, 3) - 1) == EWORKSPACE
        refused(c, EINVAL, [dict(plan=None), dict(window=-1), dict(sinks=-1)])
        assert c(plan=ODD) == EALIGN and c(planb=L.parse_shared_plan_bytes(cache(), 8, 3) - 1) == EWORKSPACE
    else:
        assert c(wsb=L.parse_attend_pages_workspace_bytes(cache(), 8, 3, 4) - 1) == EWORKSPACE
        refused(c, EINVAL, [dict(pages=None), dict(top=0), dict(top=-5)])
        assert c(pages=ODD) == EALIGN and c(top=1 << 29) == ESHAPE
        assert c(cache(n_kv=1, page=256), rows=1, n_q=1, top=1 << 23) == ESHAPE and c(cache(n_kv=1, page=16), rows=1, n_q=1, top=1 << 27) == ESHAPE


def test_shared_plan_refuses_bad_arguments():
    c, L = calls()["plan"], pa.lib()
    refused(c, EINVAL, [dict(n_q=0), dict(rows=0), dict(window=-1), dict(sinks=-1)])
    refused(c, ESHAPE, [dict(n_q=6), dict(n_q=65540), dict(rows=4097), dict(rows=4, seqs=None)])
    refused(c, EALIGN, [dict(seqs=ODD), dict(plan=ODD)])
    need = L.parse_shared_plan_bytes(cache(), 8, 3)
    assert need > 0
    refused(c, EWORKSPACE, [dict(plan=None), dict(planb=need - 1)])


def test_shared_limits():
    """Pieces of a call, and the steps of all of them."""
    L = pa.lib()
    for n_q, rows, good in ((32, 4096, True), (4 * 16, 4096, True), (4 * 64, 4096, False), (4 * 64, 2000, True), (4096, 512, False), (4096, 64, True)):
        kv = cache(n_seqs=4096, n_kv=4)
        assert (L.parse_shared_plan_bytes(kv, n_q, rows) > 0) == good, (n_q, rows)
        assert (L.parse_attend_shared_workspace_bytes(kv, n_q, rows) > 0) == good, (n_q, rows)
        wide = dict(kv=kv, n_q=n_q, rows=rows, qs=n_q * 64, outs=n_q * 64)
        if not good:
            assert calls()["shared"](**wide) == ESHAPE and calls()["plan"](**wide) == ESHAPE
    for d, good in ((160, True), (192, False), (256, False)):
        kv = cache(n_seqs=4096, n_kv=4, d=d, dtype=0)
        assert (L.parse_shared_plan_bytes(kv, 4, 4096) > 0) == good and (L.parse_attend_shared_workspace_bytes(kv, 4, 3000) > 0), d
    long = cache(n_seqs=4096, max_pages=1 << 21)
    assert calls()["shared"](long, rows=4096, n_q=8) == ESHAPE


def test_shared_limit_of_steps_holds_for_plans_and_queries():
    """16 tokens a page, 4096 rows of 8 heads over 4 with keys, 128 columns a tile: 3 * (4096 * 2 / 128 + 2048 + 1) + 4096 = 10435 entries of max_pages / 2 steps each."""
    L = pa.lib()
    most = 2 * ((2 ** 31 - 1 - 2 ** 16) // 10435)
    for pages, good in ((most, True), (most + 2, False), (1 << 21, False)):
        kv = cache(n_seqs=4096, max_pages=pages)
        assert (L.parse_shared_plan_bytes(kv, 8, 4096) > 0) == good and (L.parse_attend_shared_workspace_bytes(kv, 8, 4096) > 0) == good, pages
        if not good:
            assert calls()["plan"](kv, rows=4096) == ESHAPE and calls()["shared"](kv, rows=4096) == ESHAPE


def test_bounds_refuse_bad_arguments():
    c = calls()["bounds"]
    refused(c, EINVAL, [dict(bounds=None), dict(P=0), dict(layer=-2)])
    refused(c, ESHAPE, [dict(layer=2), dict(P=4097), dict(P=4, seqs=None)])
    refused(c, EALIGN, [dict(bounds=ODD), dict(bounds=FAKE + 8), dict(off=ODD), dict(seqs=ODD)])
    assert c(cache(n_seqs=4096, max_pages=1 << 21), P=4096) == ESHAPE
    assert pa.lib().parse_kv_bounds_bytes(cache()) == 2 * 10 * 4 * 2 * 64 * 2


def test_select_refuses_bad_arguments():
    c = calls()["select"]
    refused(c, EINVAL, [dict(bounds=None), dict(q=None), dict(pages=None), dict(n_q=0), dict(rows=0), dict(layer=-1), dict(top=0), dict(first=-1), dict(last=0)])
    refused(c, ESHAPE, [dict(layer=2), dict(n_q=6), dict(n_q=65540), dict(rows=4097), dict(rows=4, seqs=None), dict(qs=504), dict(first=3, last=2), dict(first=2 ** 31 - 1, last=2 ** 31 - 1),
                        dict(top=2 ** 31 - 1)])
    refused(c, EALIGN, [dict(bounds=ODD), dict(q=ODD), dict(pages=ODD), dict(seqs=ODD), dict(qs=516), dict(ws=ODD)])
    refused(c, EWORKSPACE, [dict(ws=None), dict(wsb=pa.lib().parse_select_pages_workspace_bytes(cache(), 8, 3) - 1)])


def test_norm_refuses_bad_arguments():
    L = pa.lib()
    ok = dict(x=FAKE, xs=64, r=FAKE, rs=64, ro=FAKE, ros=64, dtype=1, w=FAKE, wt=1, rows=3, d=64, eps=1e-6, out=FAKE, outs=64, sc=None, block=0)

    def c(**kw):
        a = {**ok, **kw}
        return L.parse_rmsnorm(a["x"], a["xs"], a["r"], a["rs"], a["ro"], a["ros"], a["dtype"], a["w"], a["wt"], a["rows"], a["d"], a["eps"], a["out"], a["outs"], a["sc"],
                               a["block"], None)
    nan = float("nan")
    refused(c, EINVAL, [dict(x=None), dict(w=None), dict(out=None), dict(rows=0), dict(d=0), dict(eps=-1.0), dict(eps=nan), dict(eps=float("inf")), dict(dtype=2), dict(wt=-1),
                        dict(block=32), dict(sc=FAKE, block=0), dict(sc=FAKE, block=-1)])
    refused(c, ESHAPE, [dict(rows=(1 << 30) + 1), dict(d=60), dict(d=65544, xs=1 << 20, rs=1 << 20, ros=1 << 20, outs=1 << 20), dict(xs=56), dict(rs=56), dict(ros=56), dict(outs=56),
                        dict(sc=FAKE, block=16), dict(sc=FAKE, block=48), dict(sc=FAKE, block=128), dict(sc=FAKE, block=512)])
    refused(c, EALIGN, [dict(x=ODD), dict(r=ODD), dict(ro=ODD), dict(w=ODD), dict(out=ODD), dict(out=FAKE + 8), dict(xs=68), dict(rs=68), dict(ros=68), dict(outs=68),
                        dict(sc=ODD, block=64), dict(sc=FAKE, block=64, out=FAKE + 4), dict(sc=FAKE, block=64, outs=68)])


def test_the_binding_refuses_what_the_kernels_would_misread():
    kv = pa.KV(torch.zeros(2, 4, 3, 1, 4, 16, 8).bfloat16(), torch.zeros(2, 4, 3, 2, 32, 8).bfloat16(), torch.zeros(5, 6, dtype=torch.int32),
               torch.zeros(5, dtype=torch.int32))
    q = torch.zeros(5, 6, 32).bfloat16()
    bounds = pa.kv_bounds_empty(kv)
    assert tuple(bounds.shape) == (2, 4, 3, 2, 32)
    pages = torch.zeros(5, 3, 4, dtype=torch.int32)
    plan = torch.zeros(pa.shared_plan_bytes(kv, 6, 5), dtype=torch.uint8)
    for bad in (lambda: pa.attend_shared(kv, 0, q.float(), plan), lambda: pa.attend_shared(kv, 0, q, plan, pages.flatten()[:4]),
                lambda: pa.kv_bounds(kv, bounds[:1], 0), lambda: pa.kv_bounds(kv, bounds.float(), 0), lambda: pa.kv_bounds(kv, bounds, 0, pages.long().flatten()[:6]),
                lambda: pa.select_pages(kv, 0, bounds, q, 4, pages=pages[:4]), lambda: pa.select_pages(kv, 0, bounds, q, 5, pages=pages),
                lambda: pa.attend_pages(kv, 0, q, pages[:, :2]), lambda: pa.attend_pages(kv, 0, q, pages.long()), lambda: pa.attend_pages(kv, 0, q, pages.transpose(1, 2))):
        with pytest.raises(ValueError):
            bad()
    x, w = torch.zeros(4, 64), torch.zeros(64)
    for bad in (lambda: pa.rmsnorm(x, w[:8], 1e-6), lambda: pa.rmsnorm(x.t(), w[:4], 1e-6), lambda: pa.rmsnorm(x, w, 1e-6, residual=x[:3]),
                lambda: pa.rmsnorm(x, w, 1e-6, scales=torch.zeros(4, 3)), lambda: pa.rmsnorm(x, w, 1e-6, scales=torch.zeros(3, 1))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: pa.rmsnorm(x, w, 1e-6, residual=x.bfloat16()), lambda: pa.rmsnorm(x, w, 1e-6, out=x.bfloat16()), lambda: pa.rmsnorm(x, w, 1e-6, out=x, scales=torch.zeros(4, 1)),
                lambda: pa.rmsnorm(x.half(), w.half(), 1e-6)):
        with pytest.raises(TypeError):
            bad()


# ---- the oracle ------------------------------------------------------------------------------------------------------
def test_oracle_choice_by_hand():
    q = np.array([[1.0, -2.0], [0.0, 1.0]])
    b = np.array([[[0, 0], [1, 1]], [[-1, 0], [2, 3]], [[5, 5], [5, 5]], [[0, -4], [0, 4]], [[0, 0], [1, 1]], [[9, 9], [9, 9.0]]])
    # per page: max(lo, hi) - 2 lo_1 (or hi_1, whichever is larger) + max(lo_1, hi_1)
    score = [1 + 0 + 1, 2 + 0 + 3, 5 - 10 + 5, 0 + 8 + 4, 2, 0]
    there = np.ones(6, bool)
    for top, want in ((2, [0, 5]), (3, [0, 3, 5]), (4, [0, 1, 3, 5]), (5, [0, 1, 3, 4, 5])):
        got, gap = so.choose(q, b, there, top, 1, 1)
        assert got.tolist() == want and gap >= 0, (top, score)
    assert so.choose(q, b, there, 6, 1, 1)[0].tolist() == [0, 1, 2, 3, 4, 5]
    there[3] = False
    assert so.choose(q, b, there, 3, 1, 1)[0].tolist() == [0, 1, 5]
    b[4] = b[1]
    assert so.choose(q, b, there, 3, 1, 1)[0].tolist() == [0, 1, 5]


def test_oracle_score_bounds_every_key():
    rng = np.random.default_rng(0)
    k, q = rng.standard_normal((16, 1, 8)), rng.standard_normal((3, 8))
    b = so.page_bounds(k)[0]
    assert np.all(sum(np.maximum(r * b[0], r * b[1]).sum() for r in q) >= (k[:, 0] @ q.T).sum(1))
    assert np.array_equal(b[0], k.min((0, 1))) and np.array_equal(b[1], k.max((0, 1)))


def test_oracle_norm_and_format():
    s, y = so.rmsnorm(np.array([[3.0, 4.0]]), np.array([[0.0, 0.0]]), np.array([1.0, 2.0]), 0.0)
    assert np.allclose(y, [[3 / np.sqrt(12.5), 8 / np.sqrt(12.5)]]) and np.array_equal(s, [[3, 4]])
    v = so.e4m3_values()
    assert v[0] == 0 and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6 and v[56] == 1 and v[126] == 448 and np.all(np.diff(v) > 0)
