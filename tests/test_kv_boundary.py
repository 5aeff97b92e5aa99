"""Checks of the paged cache that need no GPU: every call refuses what it cannot take before anything is launched, and the oracle is
pinned to closed forms and hand-computed values."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import kv_oracle as ko

pa = pytest.importorskip("paper_2605_08568_amd")
from paper_2605_08568_amd import binding as B  # noqa: E402

FAKE = 0x1000                  # non-NULL, 16-byte aligned, never read: every check below fails first
ODD = 0x1002
EINVAL, ESHAPE, EALIGN, EWORKSPACE = -1, -2, -3, -5


def cache(**kw):
    a = dict(n_layers=2, n_pages=10, page=16, n_kv=4, d=64, dtype=1, n_seqs=3, max_pages=5, K=FAKE, V=FAKE, table=FAKE, len=FAKE, refs=FAKE,
             free_bits=FAKE)
    a.update(kw)
    return C.byref(B._KV(*a.values()))


BAD_CACHES = [(dict(K=None), EINVAL), (dict(V=None), EINVAL), (dict(table=None), EINVAL), (dict(len=None), EINVAL), (dict(dtype=2), EINVAL),
              (dict(n_layers=0), EINVAL), (dict(n_pages=0), EINVAL), (dict(n_kv=0), EINVAL), (dict(n_seqs=0), EINVAL), (dict(max_pages=-1), EINVAL),
              (dict(page=8), ESHAPE), (dict(page=48), ESHAPE), (dict(page=512), ESHAPE), (dict(d=48), ESHAPE), (dict(d=288), ESHAPE), (dict(d=0), ESHAPE),
              (dict(n_kv=1025), ESHAPE), (dict(n_seqs=4097), ESHAPE), (dict(max_pages=(1 << 21) + 1), ESHAPE), (dict(K=ODD), EALIGN),
              (dict(V=ODD), EALIGN), (dict(table=ODD), EALIGN), (dict(len=ODD), EALIGN)]


def calls():
    L = pa.lib()
    ok = dict(src=FAKE, n=2, new=FAKE, served=FAKE, ws=FAKE, wsb=1 << 40, keep=FAKE, window=8, sinks=2, layer=1, k=FAKE, ks=256, v=FAKE, vs=256, q=FAKE,
              qs=512, qo=FAKE, qos=512, n_q=8, rows=6, off=FAKE, seqs=FAKE, P=3, rope=FAKE, n_pos=9, scale=1.0, out=FAKE, outs=512, lse=FAKE, live=FAKE)

    def wrap(f):
        def call(kv=None, **kw):
            a = dict(ok); a.update(kw)
            return f(kv if kv is not None else cache(), a)
        return call
    return {
        "clear": wrap(lambda kv, a: L.parse_kv_clear(kv, None)),
        "fork": wrap(lambda kv, a: L.parse_kv_fork(kv, a["src"], FAKE, a["n"], None)),
        "reserve": wrap(lambda kv, a: L.parse_kv_reserve(kv, a["new"], a["served"], a["ws"], a["wsb"], None)),
        "trim": wrap(lambda kv, a: L.parse_kv_trim(kv, a["keep"], a["window"], a["sinks"], None)),
        "compact": wrap(lambda kv, a: L.parse_kv_compact(kv, a["live"], a["ws"], a["wsb"], None)),
        "append": wrap(lambda kv, a: L.parse_kv_append(kv, a["layer"], a["k"], a["ks"], a["v"], a["vs"], a["q"], a["qs"], a["qo"], a["qos"], a["n_q"], a["rows"],
                                                       a["off"], a["seqs"], a["P"], a["rope"], a["n_pos"], None)),
        "decode": wrap(lambda kv, a: L.parse_attend_decode(kv, a["layer"], a["q"], a["qs"], a["n_q"], a["rows"], a["seqs"], a["scale"], a["window"], a["sinks"],
                                                           a["out"], a["outs"], a["lse"], a["ws"], a["wsb"], None)),
        "prefill": wrap(lambda kv, a: L.parse_attend_prefill(kv, a["layer"], a["q"], a["qs"], a["n_q"], a["rows"], a["off"], a["seqs"], a["P"], a["scale"],
                                                             a["window"], a["sinks"], a["out"], a["outs"], a["lse"], a["ws"], a["wsb"], None)),
    }


def test_every_call_refuses_bad_caches():
    for name, call in calls().items():
        for bad, status in BAD_CACHES:
            assert call(cache(**bad)) == status, (name, bad)
    counting = ("clear", "fork", "reserve", "trim", "compact")
    for name in counting:
        assert calls()[name](cache(refs=None)) == EINVAL and calls()[name](cache(free_bits=None)) == EINVAL
        assert calls()[name](cache(refs=ODD)) == EALIGN
    L = pa.lib()
    assert L.parse_kv_clear(None, None) == EINVAL
    bad = cache(page=8)
    assert L.parse_kv_workspace_bytes(bad) == 0 and L.parse_attend_decode_workspace_bytes(bad, 8, 3) == 0
    assert L.parse_attend_prefill_workspace_bytes(bad, 8, 3, 3) == 0
    assert L.parse_attend_decode_workspace_bytes(cache(), 7, 3) == 0 and L.parse_attend_decode_workspace_bytes(cache(), 8, 0) == 0


def test_bookkeeping_refuses_bad_arguments():
    c = calls()
    assert c["fork"](src=None) == EINVAL and c["fork"](n=0) == EINVAL and c["fork"](n=1025) == ESHAPE and c["fork"](src=ODD) == EALIGN
    assert c["reserve"](new=None) == EINVAL and c["reserve"](new=ODD) == EALIGN and c["reserve"](served=ODD) == EALIGN
    for name in ("reserve", "compact"):
        need = pa.lib().parse_kv_workspace_bytes(cache())
        assert c[name](ws=None) == EWORKSPACE and c[name](wsb=need - 1) == EWORKSPACE and c[name](ws=ODD) == EALIGN
    assert c["compact"](live=ODD) == EALIGN
    assert c["trim"](window=-1) == EINVAL and c["trim"](sinks=-1) == EINVAL and c["trim"](keep=None, window=0) == EINVAL and c["trim"](keep=ODD) == EALIGN


def test_append_refuses_bad_arguments():
    c = calls()["append"]
    for bad in (dict(k=None), dict(v=None), dict(rows=0), dict(P=0), dict(layer=-1), dict(q=None), dict(qo=None), dict(n_q=0), dict(n_pos=0)):
        assert c(**bad) == EINVAL, bad
    for bad in (dict(layer=2), dict(P=4097), dict(seqs=None, P=4), dict(off=None), dict(ks=248), dict(vs=8), dict(qs=504), dict(qos=0), dict(rows=(1 << 24) + 1)):
        assert c(**bad) == ESHAPE, bad
    for bad in (dict(k=ODD), dict(v=ODD), dict(q=ODD), dict(qo=ODD), dict(rope=ODD), dict(off=ODD), dict(seqs=ODD), dict(k=FAKE + 4), dict(rope=FAKE + 4), dict(ks=260), dict(vs=260), dict(qs=516), dict(qos=516)):
        assert c(**bad) == EALIGN, bad


@pytest.mark.parametrize("name", ["decode", "prefill"])
def test_attention_refuses_bad_arguments(name):
    c = calls()[name]
    rows = dict(rows=3) if name == "decode" else {}
    for bad in (dict(q=None), dict(out=None), dict(n_q=0), dict(rows=0), dict(layer=-1), dict(window=-1), dict(sinks=-1), dict(scale=float("nan")),
                dict(scale=float("inf"))):
        assert c(**{**rows, **bad}) == EINVAL, bad
    for bad in (dict(layer=2), dict(n_q=6, qs=512), dict(qs=504), dict(outs=504), dict(n_q=65540)):
        assert c(**{**rows, **bad}) == ESHAPE, bad
    for bad in (dict(q=ODD), dict(out=ODD), dict(lse=ODD), dict(seqs=ODD), dict(q=FAKE + 8), dict(qs=516), dict(outs=516)):
        assert c(**{**rows, **bad}) == EALIGN, bad
    if name == "decode":
        assert c(rows=4097) == ESHAPE and c(rows=4, seqs=None) == ESHAPE
        assert c(rows=3, ws=None) == EWORKSPACE and c(rows=3, ws=ODD) == EALIGN
        assert c(rows=3, wsb=pa.lib().parse_attend_decode_workspace_bytes(cache(), 8, 3) - 1) == EWORKSPACE
    else:
        assert c(P=0) == EINVAL and c(P=4097) == ESHAPE and c(P=4, seqs=None) == ESHAPE and c(off=None) == ESHAPE
        assert c(n_q=4096, qs=1 << 19, outs=1 << 19, rows=1 << 15) == ESHAPE


def test_the_binding_refuses_what_the_kernels_would_misread():
    kv = pa.KV(torch.zeros(2, 4, 3, 1, 4, 16, 8).bfloat16(), torch.zeros(2, 4, 3, 2, 32, 8).bfloat16(), torch.zeros(5, 6, dtype=torch.int32),
               torch.zeros(5, dtype=torch.int32))
    assert (kv.n_layers, kv.n_pages, kv.n_kv, kv.page, kv.d, kv.n_seqs, kv.max_pages) == (2, 4, 3, 16, 32, 5, 6)
    c = kv.c()
    assert c.n_layers == 2 and c.refs is None and c.K == kv.K.data_ptr() and c.len == kv.len.data_ptr()
    K, V, t, n = kv.K, kv.V, kv.table, kv.len
    for bad in ((K, V[:, :3], t, n), (K, V.float(), t, n), (K, V, t.long(), n), (K, V, t, n[:4]), (K, V, t, n, torch.zeros(3, dtype=torch.int32)),
                (K[:, :, :, :, ::2], V, t, n), (K[0], V, t, n), (K, V, t.t().contiguous().t(), n)):
        with pytest.raises((ValueError, TypeError)):
            pa.KV(*bad)
    q = torch.zeros(4, 6, 32).bfloat16()
    for bad in (q.float(), q[:, :, :16], torch.zeros(4, 32, 6).bfloat16().transpose(1, 2), torch.zeros(4, 12, 32).bfloat16()[:, ::2]):
        with pytest.raises((ValueError, TypeError)):
            pa.attend_decode(kv, 0, bad, workspace=torch.zeros(1, dtype=torch.uint8))
    with pytest.raises(ValueError):
        pa.attend_decode(kv, 0, q, seqs=torch.zeros(4), workspace=torch.zeros(1, dtype=torch.uint8))
    with pytest.raises(ValueError):
        pa.attend_decode(kv, 0, q, out=q[:3], workspace=torch.zeros(1, dtype=torch.uint8))
    with pytest.raises(ValueError):
        pa.kv_append(kv, 0, q[:, :3], q[:3, 3:])
    with pytest.raises(ValueError):
        pa.kv_append(kv, 0, q[:, :3], q[:, 3:], rope=torch.zeros(3, 16))
    with pytest.raises(ValueError):
        pa.kv_trim(kv, torch.zeros(4, dtype=torch.int32))


# ---- the oracle -----------------------------------------------------------------------------------------------------
def test_layout_is_the_header_s():
    n_kv, d, page = 3, 32, 32
    x = np.arange(page * n_kv * d).reshape(page, n_kv, d)
    K, V = ko.k_to_pages(x).ravel(), ko.v_to_pages(x).ravel()
    for w in (0, 7, 8, 15, 16, 31):
        for h in range(n_kv):
            for i in (0, 5, 8, 31):
                assert K[(((h * (page // 16) + w // 16) * (d // 8) + i // 8) * 128) + (w % 16) * 8 + i % 8] == x[w, h, i]
                assert V[((h * (page // 8) + w // 8) * d + i) * 8 + w % 8] == x[w, h, i]
    assert np.array_equal(ko.k_from_pages(ko.k_to_pages(x)), x) and np.array_equal(ko.v_from_pages(ko.v_to_pages(x)), x)


def test_attention_closed_forms():
    rng = np.random.default_rng(0)
    v = rng.standard_normal((7, 2, 4))
    o, lse, mag, _ = ko.attend_row(np.zeros((4, 4)), rng.standard_normal((7, 2, 4)), v, np.ones(7, bool), 0.5)    # equal scores: the mean
    for h in range(4):
        assert np.allclose(o[h], v[:, h // 2].mean(0)) and np.isclose(lse[h], np.log(7)) and np.allclose(mag[h], np.abs(v[:, h // 2]).mean(0))
    k = np.zeros((2, 1, 2)); k[1, 0, 0] = 1
    q = np.array([[np.log(3.0), 0.0]])                                  # scores 0 and ln 3: weights 1/4 and 3/4
    o, lse, _, big = ko.attend_row(q, k, np.array([[[4.0, 0.0]], [[0.0, 4.0]]]), np.ones(2, bool), 1.0)
    assert np.allclose(o, [[1.0, 3.0]]) and np.isclose(lse[0], np.log(4)) and np.isclose(big[0], np.log(3))
    o, lse, _, _ = ko.attend_row(q, k, k, np.zeros(2, bool), 1.0)
    assert not o.any() and np.isneginf(lse[0])


def test_what_a_row_sees():
    there = np.ones(10, bool)
    assert list(np.flatnonzero(ko.visible(6, there, 0, 0))) == list(range(7))
    assert list(np.flatnonzero(ko.visible(6, there, 3, 0))) == [4, 5, 6]
    assert list(np.flatnonzero(ko.visible(6, there, 3, 2))) == [0, 1, 4, 5, 6]
    assert list(np.flatnonzero(ko.visible(1, there, 3, 4))) == [0, 1]                # sinks lie in the past only
    there[4:6] = False
    assert list(np.flatnonzero(ko.visible(6, there, 3, 1))) == [0, 6]
    assert not ko.visible(-1, there, 3, 4).any()


def test_rotation():
    x = np.array([[[1.0, 0.0, 0.0, 2.0]]])
    turn = np.array([[0.0, 1.0, 1.0, 0.0]])                              # a quarter turn of the first pair, none of the second
    assert np.allclose(ko.rotate(x, turn), [[[0.0, 0.0, 1.0, 2.0]]])


def test_bookkeeping_by_hand():
    p = ko.Pages(4, 3, 6, 16)
    copies, served = p.reserve([20, 5, 0, 0])
    assert copies == [] and served.tolist() == [1, 1, 0, 0] and p.table.tolist() == [[0, 1, -1], [2, -1, -1], [-1] * 3, [-1] * 3]
    p.fork([0, 0], [2, 3])
    assert p.refs.tolist() == [3, 3, 1, 0, 0, 0] and p.len.tolist() == [20, 5, 20, 20] and p.free_words().tolist() == [0b111000]
    copies, served = p.reserve([1, 0, 1, 1])                             # two copies of page 1, the third user keeps it
    assert copies == [(1, 3), (1, 4)] and p.table[:, 1].tolist() == [3, -1, 4, 1] and p.refs.tolist() == [3, 1, 1, 1, 1, 0]
    copies, served = p.reserve([0, 12, 12, 12])                          # one page is left: 1 takes it, 2 does not fit, 3 comes behind it
    assert served.tolist() == [0, 1, 0, 0] and p.table[1].tolist() == [2, 5, -1]
    p.trim([0, 100, 16, 21], 0, 0)
    assert p.len.tolist() == [0, 17, 16, 21] and p.refs.tolist() == [2, 1, 1, 0, 0, 1]
    assert p.compact() == ([(5, 3)], 4) and p.table.tolist() == [[-1] * 3, [2, 3, -1], [0, -1, -1], [0, 1, -1]]
    q = ko.Pages(1, 10, 10, 16)
    q.reserve([100])
    q.trim(None, 40, 4)                                                  # tokens 61.. are seen by the next one: pages 1 and 2 go, 0 has the sinks
    assert q.table[0].tolist() == [0, -1, -1, 3, 4, 5, 6, -1, -1, -1] and q.len[0] == 100


def test_reserve_with_a_list_refuses_bad_arguments():
    L = pa.lib()

    def call(kv=None, new=FAKE, served=FAKE, seqs=FAKE, P=3, out=FAKE, ws=FAKE, wsb=1 << 40):
        return L.parse_kv_reserve_seqs(kv if kv is not None else cache(), new, served, seqs, P, out, ws, wsb, None)
    for bad, status in BAD_CACHES + [(dict(refs=None), EINVAL), (dict(free_bits=ODD), EALIGN)]:
        assert call(cache(**bad)) == status, bad
    assert call(new=None) == EINVAL and call(out=None) == EINVAL and call(P=0) == EINVAL and call(P=-1) == EINVAL
    assert call(P=4097) == ESHAPE and call(seqs=None, P=4) == ESHAPE
    assert call(new=ODD) == EALIGN and call(served=ODD) == EALIGN and call(seqs=ODD) == EALIGN and call(out=ODD) == EALIGN and call(ws=ODD) == EALIGN
    assert call(ws=None) == EWORKSPACE and call(wsb=L.parse_kv_workspace_bytes(cache()) - 1) == EWORKSPACE
    kv = pa.KV(torch.zeros(2, 4, 3, 1, 4, 16, 8).bfloat16(), torch.zeros(2, 4, 3, 2, 32, 8).bfloat16(), torch.zeros(5, 6, dtype=torch.int32),
               torch.zeros(5, dtype=torch.int32))
    i = torch.zeros(5, dtype=torch.int32)
    for bad in (dict(seqs=i), dict(seqs=i[:3], seqs_served=i), dict(seqs=i, seqs_served=i.long()), dict(seqs_served=i.float())):
        with pytest.raises(ValueError):
            pa.kv_reserve(kv, i, i, torch.zeros(1, dtype=torch.uint8), **bad)


def test_decode_refuses_more_steps_than_it_can_count():
    """Blocks of 32 tokens over all rows are added up in 31 bits: the table says how many there may be, or the window where that is less.  A call that is
    let through stops at the missing workspace here."""
    L = pa.lib()

    def call(rows, columns, page=16, window=0, sinks=0):
        return L.parse_attend_decode(cache(n_seqs=4096, max_pages=columns, page=page), 0, FAKE, 512, 8, rows, FAKE, 1.0, window, sinks, FAKE, 512, None, None, 0, None)
    whole = 1 << 21                                                 # 2^25 tokens, 2^20 blocks
    assert call(4096, whole) == ESHAPE and call(2048, whole) == ESHAPE and call(4096, 1 << 17, 256) == ESHAPE
    assert call(2047, whole) == EWORKSPACE and call(4096, whole // 2 - 2) == EWORKSPACE and call(1, whole) == EWORKSPACE
    assert call(4096, whole, window=4096, sinks=4) == EWORKSPACE
    assert call(4096, whole, window=1 << 24, sinks=1 << 10) == ESHAPE and call(4096, whole, window=2 ** 31 - 1, sinks=2 ** 31 - 1) == ESHAPE
