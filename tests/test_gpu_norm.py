"""The root-mean-square norm against the float64 oracle: every width and type, rows apart, arrays that are one, 8 bits with scales."""
import numpy as np
import pytest
import torch

from oracle import step_oracle as so

pytestmark = pytest.mark.gpu

pa = pytest.importorskip("paper_2605_08568_amd")
from helpers import check_guards, guarded_bytes  # noqa: E402

DEV = "cuda"
TORCH = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
# In 32 bits: s is rounded once; the longest chain of the sum of squares is 8 columns of up to 8 pieces, 6 additions of lanes and 16 of wavefronts, each and every square
# half a step, so that the root is off by (64 + 6 + 16 + 1) / 2 of them; mean, eps, root, reciprocal, two products one each
STEPS = (64 + 6 + 16 + 1) / 2 + 1 + 6


def rows_of(rows, d, dtype, pad, fill=None):
    """[rows][d] inside a wider buffer between canaries: (whole, buffer, view)."""
    es = torch.empty((), dtype=dtype).element_size()
    buf, mid = guarded_bytes(rows * (d + pad) * es)
    whole = mid[:rows * (d + pad) * es].view(dtype).view(rows, d + pad)
    if fill is not None:
        whole[:, :d] = fill
    return buf, whole, whole[:, :d]


def check(got, y, dtype, what, floor=0.0):
    tol = np.abs(y) * (STEPS * 2.0 ** -24 + HALF[dtype] * (1 + 2.0 ** -15)) + floor + 2.0 ** -133
    off = np.abs(got.double().cpu().numpy() - y) - tol
    assert np.all(off <= 0), f"{what}: {off.max():.3e} over the bound, at {np.unravel_index(off.argmax(), off.shape)}"


def check_e4m3(out, scales, y, block):
    q, sc = out.double().cpu().numpy(), scales.double().cpu().numpy()
    rows, d = y.shape
    blocks = y.reshape(rows, -1, block)
    want = np.maximum(np.abs(blocks).max(2) / 448, 2.0 ** -120)
    assert np.all(np.abs(sc - want) <= want * (STEPS + 1) * 2.0 ** -24 + 2.0 ** -149), "scales"
    # half a step: 2^-4 of the value, below the smallest normal one 2^-10 of the scale; y, the reciprocal and the product are off by 32-bit steps
    off = np.abs(q.reshape(blocks.shape) * sc[..., None] - blocks)
    tol = np.maximum(np.abs(blocks) * 2.0 ** -4, 2.0 ** -10 * sc[..., None]) * (1 + 2.0 ** -16) + np.abs(blocks) * (STEPS + 3) * 2.0 ** -24
    assert np.all(off <= tol), f"values: {(off - tol).max():.3e} over the bound"
    assert np.all(np.isin(np.abs(q), so.e4m3_values()))


def run(dtype, rows, d, residual=True, wdtype=None, eps=1e-5, pads=(0, 0, 0, 0), block=None, seed=0, keep=True, scale=1.0):
    rng = np.random.default_rng(seed)
    t, wt = TORCH[dtype], TORCH[wdtype or dtype]
    x = torch.from_numpy(scale * rng.standard_normal((rows, d)).astype(np.float32)).to(t)
    r = torch.from_numpy((4 * scale * rng.standard_normal((rows, d))).astype(np.float32)).to(t) if residual else None
    w = torch.from_numpy((1 + 0.2 * rng.standard_normal(d)).astype(np.float32)).to(wt)
    s, y = so.rmsnorm(x.double().numpy(), r.double().numpy() if residual else None, w.double().numpy(), eps)
    bufs = {}
    bufs["x"], xw, xd = rows_of(rows, d, t, pads[0], x.to(DEV))
    rd = rout = None
    if residual:
        bufs["residual"], _, rd = rows_of(rows, d, t, pads[1], r.to(DEV))
    if keep:
        bufs["residual_out"], kw, rout = rows_of(rows, d, t, pads[2])
        marked = kw[:, d:].clone()
    scales = None
    bufs["out"], ow, out = rows_of(rows, d, t if block is None else torch.float8_e4m3fn, pads[3])
    behind = ow.view(torch.uint8)[:, d * out.element_size():].clone()
    if block is not None:
        bufs["scales"], mid = guarded_bytes(rows * (d // block) * 4)
        scales = mid[:rows * (d // block) * 4].view(torch.float32).view(rows, d // block)
    pa.rmsnorm(xd, w.to(DEV), eps, rd, rout, out, scales)
    for what, b in bufs.items():
        check_guards(b, what)
    assert torch.equal(ow.view(torch.uint8)[:, d * out.element_size():], behind), "stores between the rows"
    assert torch.equal(xd.cpu().view(torch.uint8 if dtype == "bf16" else torch.uint8), x.view(torch.uint8)) or not xd.is_contiguous()
    if keep:
        assert torch.equal(rout.cpu(), (x.float() + r.float()).to(t) if residual else x), "residual_out"
        assert torch.equal(kw[:, d:], marked)
    if block is None:
        check(out, y, dtype, "out")
    else:
        check_e4m3(out, scales, y, block)


SIZES = [8, 24, 64, 512, 520, 1024, 1032, 2048, 2056, 4096, 4104, 8192, 8200, 16384, 16392, 32768, 32776, 65536]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", SIZES)
def test_widths(dtype, d):
    run(dtype, 5, d, seed=d)
    run(dtype, 3, d, residual=False, keep=False, seed=d + 1)


@pytest.mark.parametrize("dtype,wdtype", [("bf16", "fp32"), ("fp32", "bf16")])
@pytest.mark.parametrize("d", [64, 1024, 4096, 16384])
def test_weights_of_the_other_type(dtype, wdtype, d):
    run(dtype, 4, d, wdtype=wdtype, seed=d)
    run(dtype, 4, d, wdtype=wdtype, block=d, seed=d)


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 63, 257, 5000])
def test_rows_apart(rows):
    run("bf16", rows, 136, pads=(8, 16, 24, 32), seed=rows)
    run("fp32", rows, 72, pads=(4, 8, 12, 16), seed=rows)
    run("bf16", rows, 256, pads=(8, 16, 24, 8), block=32, seed=rows)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,block", [(8, 8), (32, 32), (96, 32), (512, 64), (1000, 1000), (1024, 128), (2048, 256), (4096, 4096), (4096, 128), (4352, 256), (8192, 32), (16640, 64),
                                     (11008, 256), (32768, 128), (65536, 65536), (65536, 256)])
def test_eight_bits(dtype, d, block):
    run(dtype, 3, d, block=block, seed=d + block)


def test_arrays_that_are_one():
    """The stream updated in place, the norm written over its input."""
    torch.manual_seed(1)
    x, r, w = torch.randn(37, 768, device=DEV).bfloat16(), torch.randn(37, 768, device=DEV).bfloat16(), torch.rand(768, device=DEV).bfloat16()
    kept = torch.empty_like(x)
    want = pa.rmsnorm(x, w, 1e-6, r, kept)
    a, b = x.clone(), r.clone()
    assert pa.rmsnorm(a, w, 1e-6, b, b, a) is a
    assert torch.equal(a, want) and torch.equal(b, kept)
    a = x.clone()
    out = pa.rmsnorm(a, w, 1e-6, r, a)
    assert torch.equal(out, want) and torch.equal(a, kept)


def test_values_at_the_ends():
    """Rows of zeros, tiny and huge rows, NaN and infinities in one row only."""
    w = torch.ones(256, device=DEV)
    x = torch.randn(8, 256, device=DEV)
    x[1], x[2, 7], x[3, 9] = 0, torch.nan, torch.inf
    x[4] *= 1e-18
    x[5] *= 1e18
    out = pa.rmsnorm(x, w, 1e-6)
    _, y = so.rmsnorm(x.double().cpu().numpy(), None, np.ones(256), 1e-6)
    good = [0, 1, 4, 5, 6, 7]
    check(out[good], y[good], "fp32", "out")
    assert bool(out[2].isnan().all()) and bool(out[3, 9].isnan()) and bool((out[3][torch.arange(256) != 9] == 0).all())
    scales = torch.empty(8, 2, device=DEV)
    q = pa.rmsnorm(x, w, 1e-6, scales=scales)
    check_e4m3(q[good], scales[good], y[good], 128)
    assert bool((q[1].float() == 0).all()) and bool((scales[1] == 2.0 ** -120).all())
    assert bool(q[2].float().isnan().all()) and bool(scales[2].isnan().all())
    q = pa.rmsnorm(x[:1] * 0, w, 0.0, scales=torch.empty(1, 1, device=DEV))
    assert bool(q.float().isnan().all())                           # 0 / 0, as the formula has it


def test_small_weights_keep_their_scale():
    x, w = torch.randn(4, 128, device=DEV), torch.full((128,), 2.0 ** -126, device=DEV)
    scales = torch.empty(4, 1, device=DEV)
    q = pa.rmsnorm(x, w, 1e-6, scales=scales)
    _, y = so.rmsnorm(x.double().cpu().numpy(), None, w.double().cpu().numpy(), 1e-6)
    assert bool((scales == 2.0 ** -120).all())
    assert np.all(np.abs(q.double().cpu().numpy() * 2.0 ** -120 - y) <= np.maximum(np.abs(y) * 2.0 ** -4, 2.0 ** -130) * 1.01 + 2.0 ** -149)


@pytest.mark.parametrize("block", [None, 8])
def test_more_rows_than_a_launch_takes(block):
    """The rows on both sides of the seam, at the end, and those between that repeat them."""
    seam, d = 1 << 21, 8
    some = torch.from_numpy(np.random.default_rng(3).standard_normal((64, d)).astype(np.float32)).bfloat16()
    x = some.to(DEV).repeat(seam // 64 + 1, 1)[:seam + 37].contiguous()
    w = torch.ones(d, device=DEV, dtype=torch.bfloat16)
    res, scales = torch.empty_like(x), None if block is None else torch.full((len(x), d // block), np.nan, device=DEV)
    out = pa.rmsnorm(x, w, 1e-5, x, res, None, scales)
    s, y = so.rmsnorm(some.double().numpy(), some.double().numpy(), np.ones(d), 1e-5)
    if block is None:
        check(out[:64], y, "bf16", "out")
    else:
        check_e4m3(out[:64], scales[:64], y, block)
    assert torch.equal(res, 2 * x), "twice a number of bf16 is one"
    for t in (out.view(torch.uint8), scales):
        if t is not None:
            assert torch.equal(t[64:], t[:-64]), "equal rows, equal results"


def test_graph_and_stream():
    torch.manual_seed(2)
    x, r, w = torch.randn(100, 4096, device=DEV).bfloat16(), torch.randn(100, 4096, device=DEV).bfloat16(), torch.rand(4096, device=DEV).bfloat16()
    kept, out = torch.empty_like(x), torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pa.rmsnorm(x, w, 1e-6, r, kept, out)
    torch.cuda.current_stream().wait_stream(side)
    want = pa.rmsnorm(x, w, 1e-6, r)
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pa.rmsnorm(x, w, 1e-6, r, kept, out)
    for i in range(5):
        x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, pa.rmsnorm(x, w, 1e-6, r)) and torch.equal(kept, (x.float() + r.float()).bfloat16())
