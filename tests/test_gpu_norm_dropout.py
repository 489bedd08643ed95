"""Dropout, and the root-mean-square norm with the residual's addition, against their formulas in 64 bits: widths, types,
strides, masks to the element, outputs in 8 bits, gradients, rows and values at the ends of their ranges."""
import numpy as np
import pytest

import block_reference as ref
from gpu_common import require_gpu
from paper_2609_37899_amd import soma

pytestmark = pytest.mark.gpu

TYPES = [("float32", "float32"), ("bfloat16", "bfloat16"), ("bfloat16", "float32")]
SEED, STEP, LAYER = 0x123456789ABCDEF, (5 << 32) + 7, 9


def both(torch, x, dtype, pad=0, shift=0):
    """On the GPU (rows `pad` elements longer, starting at element `shift`), and as it is stored in 64 bits."""
    dt = getattr(torch, dtype)
    y = torch.from_numpy(x.astype(np.float32)).to(dt)
    if pad or shift:
        n, w = x.shape
        flat = torch.full((n * (w + pad) + shift + 16,), float("nan"), dtype=dt, device="cuda")
        view = flat[shift:shift + n * (w + pad)].view(n, w + pad)[:, :w]
        view.copy_(y)
    else:
        view = y.cuda()
    return view, y.double().numpy()


def near(got, exact, err, dtype, name):
    step = ref.half_step(dtype)
    got = got.double().cpu().numpy()
    tol = err * (1 + step) + step * np.abs(exact) + 1e-37
    bad = ~(np.abs(got - exact) <= tol)
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size}, worst {np.nanmax(np.abs(got - exact) / tol):.2f} of the bound"


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,width", [(1, 1), (3, 8), (7, 13), (5, 1000), (300, 361), (1, 70001)])
@pytest.mark.parametrize("p", [0.0, 1e-6, 0.1, 0.999])
@pytest.mark.parametrize("residual", [False, True])
def test_dropout(dtype, rows, width, p, residual):
    torch = require_gpu()
    g = np.random.default_rng(1)
    x, x64 = both(torch, g.standard_normal((rows, width)), dtype)
    r, r64 = both(torch, g.standard_normal((rows, width)), dtype) if residual else (None, 0)
    plan = soma.Dropout(rows, width, x.dtype, p)
    y = torch.full_like(x, 7.0)
    plan.forward(x, y, r, SEED, STEP, LAYER)
    torch.cuda.synchronize()
    factor = ref.keep(rows, width, p, SEED, STEP, LAYER)
    exact = ref.drop(x64, factor)
    near(y, exact + r64, ref.U * (2 * np.abs(exact) + np.abs(exact + r64)), dtype, "y")
    if not residual:
        assert np.array_equal(y.double().cpu().numpy() == 0, (exact == 0) | (x64 == 0))
    # gradients go the same way, in place too
    d = x.clone()
    plan.backward(d, d, SEED, STEP, LAYER)
    torch.cuda.synchronize()
    near(d, exact, ref.U * 2 * np.abs(exact), dtype, "dx")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("width", [64, 37])
@pytest.mark.parametrize("pad,shift", [(1, 0), (8, 8), (3, 1), (0, 2)])
def test_dropout_strides(dtype, width, pad, shift):
    """The same bits as from contiguous rows."""
    torch = require_gpu()
    g = np.random.default_rng(2)
    a, b = g.standard_normal((50, width)), g.standard_normal((50, width))
    plan = soma.Dropout(50, width, getattr(torch, dtype), 0.3)
    out = []
    for k in (dict(), dict(pad=pad, shift=shift)):
        y = torch.zeros(50, width, dtype=plan.dtype, device="cuda")
        plan.forward(both(torch, a, dtype, **k)[0], y, both(torch, b, dtype, **k)[0], SEED, 1, 0)
        out.append(y)
    torch.cuda.synchronize()
    assert torch.equal(*out)


def test_masks_differ_and_keep_their_share():
    """By seed, step and layer; the share that is kept within 6 deviations.  (The upper halves of seed and step enter
    as their exclusive or, so that 2^32 more of one is, by definition, 2^32 more of the other.)"""
    torch = require_gpu()
    n, w, p = 4096, 1024, 0.3
    plan = soma.Dropout(n, w, torch.bfloat16, p)
    x = torch.ones(n, w, dtype=torch.bfloat16, device="cuda")
    masks = []
    for where in ((1, 1, 1), (2, 1, 1), (1, 2, 1), (1, 1, 2), (1 + (1 << 32), 1, 1), (1, 1 + (1 << 33), 1)):
        y = torch.empty_like(x)
        plan.forward(x, y, None, *where)
        masks.append(y != 0)
    kept = round(65536 * (1 - p)) / 65536
    for i, m in enumerate(masks):
        assert abs(m.double().mean().item() - kept) < 6 * (kept * (1 - kept) / (n * w)) ** 0.5
        for other in masks[:i]:
            both_kept = (m & other).double().mean().item()
            assert abs(both_kept - kept * kept) < 6 * (kept * kept / (n * w)) ** 0.5


def test_what_is_dropped_counts_as_zero():
    torch = require_gpu()
    factor = ref.keep(10, 100, 0.5, SEED, STEP, LAYER)
    x = torch.zeros(10, 100, device="cuda")
    x[torch.from_numpy(factor == 0).cuda()] = float("nan")
    x[0, torch.from_numpy(factor[0] == 0).cuda()] = float("inf")
    y, r = torch.full_like(x, 7.0), torch.randn(10, 100, device="cuda")
    soma.Dropout(10, 100, torch.float32, 0.5).forward(x, y, r, SEED, STEP, LAYER)
    n = soma.RmsNorm(10, 100, torch.float32, drop=0.5)
    total, z = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    n.forward(x, torch.ones(100, device="cuda"), z, r, total, None, SEED, STEP, LAYER)
    torch.cuda.synchronize()
    assert torch.equal(y, r) and torch.equal(total, r) and torch.isfinite(z).all()


def test_dropout_beyond_2_32_elements():
    """Counters past 32 bits of elements: the last rows against the reference."""
    torch = require_gpu()
    rows, width = 2**22 + 3, 1031
    x = torch.ones(rows, width, dtype=torch.bfloat16, device="cuda")
    soma.Dropout(rows, width, torch.bfloat16, 0.25).forward(x, x, None, SEED, STEP, LAYER)
    for first in (0, 2**32 // width - 5, rows - 10):
        got = x[first:first + 10].double().cpu().numpy()
        assert np.array_equal(got != 0, ref.keep(10, width, 0.25, SEED, STEP, LAYER, first) != 0)


def make(torch, types, rows, width, p, residual=True, seed=0, **kw):
    g = np.random.default_rng(seed)
    T, S = types
    x, w = {}, {}
    x["x"], w["x"] = both(torch, g.standard_normal((rows, width)), T, **kw)
    x["residual"], w["residual"] = both(torch, 2 * g.standard_normal((rows, width)), S, **kw) if residual else (None, None)
    gain = (1 + 0.1 * g.standard_normal(width)).astype(np.float32)
    x["gain"], w["gain"] = torch.from_numpy(gain).cuda(), gain.astype(np.float64)
    x["dy"], w["dy"] = both(torch, g.standard_normal((rows, width)), T)
    x["dtotal"], w["dtotal"] = both(torch, g.standard_normal((rows, width)), S)
    w["factor"] = ref.keep(rows, width, p, SEED, STEP, LAYER)
    return x, w


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("rows,width", [(1, 1), (5, 2), (9, 63), (1, 512), (70, 500), (33, 512), (6, 509), (5, 1000), (6, 1024),
                                        (3, 2047), (4, 2048), (3, 3000), (2, 4097), (2, 8192), (2, 8185), (2, 16384), (1, 16383),
                                        (6000, 40), (5000, 361)])
@pytest.mark.parametrize("p", [0.0, 0.2])
def test_norm(types, rows, width, p):
    torch = require_gpu()
    T, S = types
    x, w = make(torch, types, rows, width, p)
    plan = soma.RmsNorm(rows, width, getattr(torch, T), getattr(torch, S), eps=1e-5, drop=p)
    total, y = torch.full_like(x["dtotal"], 7.0), torch.full_like(x["dy"], 7.0)
    where = SEED, STEP, LAYER
    plan.forward(x["x"], x["gain"], y, x["residual"], total, None, *where)
    torch.cuda.synchronize()
    eps = np.float64(np.float32(1e-5))
    want = ref.norm(w["x"], w["residual"], w["gain"], eps, w["factor"])
    near(total, want["total"], want["total_err"], S, "total")
    near(y, want["y"], want["y_err"], T, "y")
    dr, dx, dg = torch.full_like(total, 7.0), torch.full_like(y, 7.0), torch.full_like(x["gain"], 7.0)
    plan.backward(total, x["gain"], x["dy"], x["dtotal"], dr, dx, dg, *where)
    torch.cuda.synchronize()
    back = ref.norm_backward(total.double().cpu().numpy(), w["gain"], w["dy"], w["dtotal"], eps, w["factor"])
    near(dr, back["dresidual"], back["dresidual_err"], S, "dresidual")
    near(dx, back["dx"], back["dx_err"], T, "dx")
    near(dg, back["dgain"], back["dgain_err"], "float32", "dgain")


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("width", [96, 77])
def test_norm_in_place_strided_and_left_out(types, width):
    """total over residual, dresidual over dtotal, strided rows, single outputs, no residual: the same bits."""
    torch = require_gpu()
    T, S = types
    x, w = make(torch, types, 41, width, 0.3)
    plan = soma.RmsNorm(60, width, getattr(torch, T), getattr(torch, S), drop=0.3)
    where = SEED, STEP, LAYER
    total, y = torch.empty_like(x["dtotal"]), torch.empty_like(x["dy"])
    plan.forward(x["x"], x["gain"], y, x["residual"], total, None, *where)
    dr, dx, dg = torch.empty_like(total), torch.empty_like(y), torch.empty_like(x["gain"])
    plan.backward(total, x["gain"], x["dy"], x["dtotal"], dr, dx, dg, *where)
    r, y2 = x["residual"].clone(), torch.empty_like(y)
    plan.forward(x["x"], x["gain"], y2, r, r, None, *where)
    assert torch.equal(r, total) and torch.equal(y, y2)
    d = x["dtotal"].clone()
    plan.backward(total, x["gain"], x["dy"], d, d, None, None, *where)
    assert torch.equal(d, dr)
    dx2, dg2 = torch.empty_like(dx), torch.empty_like(dg)
    plan.backward(total, x["gain"], x["dy"], x["dtotal"], None, dx2, None, *where)
    plan.backward(total, x["gain"], x["dy"], x["dtotal"], None, None, dg2, *where)
    assert torch.equal(dx2, dx) and torch.equal(dg2, dg)
    for pad, shift in ((1, 0), (8, 8), (5, 3)):
        s, _ = make(torch, types, 41, width, 0.3, pad=pad, shift=shift)
        y2, t2 = torch.empty_like(y), torch.empty_like(total)
        plan.forward(s["x"], x["gain"], y2, s["residual"], t2, None, *where)
        assert torch.equal(t2, total) and torch.equal(y, y2)
    y3, t3 = torch.empty_like(y), torch.empty_like(total)
    plan.forward(x["x"], x["gain"], y2, None, t2, None, *where)
    plan.forward(x["x"], x["gain"], y3, torch.zeros_like(total), t3, None, *where)
    plan.backward(total, x["gain"], x["dy"], None, dr, None, None, *where)
    plan.backward(total, x["gain"], x["dy"], torch.zeros_like(total), d, None, None, *where)
    torch.cuda.synchronize()
    assert torch.equal(t2, t3) and torch.equal(y2, y3) and torch.equal(dr, d)


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("rows,width", [(1, 1), (64, 512), (9, 361), (5, 2049), (3, 4096), (2, 16384)])
def test_norm_in_8_bits(types, rows, width):
    """Scales from the largest magnitude of a row; codes to the nearest: half a step of e4m3 (a quarter of 2^-6 below its
    normal values, 2^-10), after two divisions and a product in fp32."""
    torch = require_gpu()
    T, S = types
    x, w = make(torch, types, rows, width, 0.0)
    plan = soma.RmsNorm(rows, width, getattr(torch, T), getattr(torch, S))
    total = torch.full_like(x["dtotal"], 7.0)
    codes = torch.full((rows, width), 7.0, device="cuda").to(torch.float8_e4m3fn)
    scale = torch.full((rows,), 7.0, device="cuda")
    plan.forward(x["x"], x["gain"], codes, x["residual"], total, scale)
    torch.cuda.synchronize()
    want = ref.norm(w["x"], w["residual"], w["gain"], np.float64(np.float32(1e-5)), w["factor"])
    near(total, want["total"], want["total_err"], S, "total")
    top = np.abs(want["y"]).max(1)
    near(scale, top / 448, want["y_err"].max(1) / 448 + 3 * ref.U * top / 448, "float32", "scale")
    exact = want["y"] / (top[:, None] / 448)
    got = codes.double().cpu().numpy()
    err = (want["y_err"] + want["y_err"].max(1, keepdims=True)) / (top[:, None] / 448) + 6 * ref.U * np.abs(exact)
    assert (np.abs(got - exact) <= 2.0**-4 * np.abs(exact) + 2.0**-10 + err * 1.1).all()
    assert (np.abs(got).max(1) == 448).all()


@pytest.mark.parametrize("small", [1e-36, 1e-38, 1e-40, 1e-44])
def test_norm_in_8_bits_below_the_normal_numbers(small):
    """Rows whose scale would be no normal number: 2^-126 (one with half its columns 0 is just above it), and codes as near as they come. y is off by a few u, and by a
    step of 2^-149 where it is subnormal itself; its code by half a step, 2^-4 of it or 2^-10."""
    torch = require_gpu()
    x, w = make(torch, ("float32", "float32"), 5, 100, 0.0, residual=False)
    x["x"][2], w["x"][2] = 0.0, 0.0
    x["x"][3, ::2], w["x"][3, ::2] = 0.0, 0.0
    gain = torch.full((100,), small, device="cuda")
    plan = soma.RmsNorm(5, 100, torch.float32)
    codes, scale = torch.empty(5, 100, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(5, device="cuda")
    plan.forward(x["x"], gain, codes, None, None, scale)
    torch.cuda.synchronize()
    exact = w["x"] / np.sqrt((w["x"] ** 2).mean(1, keepdims=True) + np.float64(np.float32(1e-5))) * np.float64(np.float32(small))
    got, scale = codes.double().cpu().numpy(), scale.double().cpu().numpy()
    want = np.where(np.arange(5) == 2, 0.0, np.maximum(np.abs(exact).max(1) / 448, 2.0**-126))
    assert (np.abs(scale - want) <= np.where(want > 2.0**-126, 60 * ref.U * want, 0.0)).all()
    at = exact / np.maximum(want, 2.0**-126)[:, None]
    assert (np.abs(got[:2] - at[:2]) <= 2.0**-4 * np.abs(at[:2]) + 2.0**-10 + 60 * ref.U * np.abs(at[:2]) + 2.0**-22).all()
    assert (got[2] == 0).all() and (got[3, ::2] == 0).all()
    assert (np.abs(got[3:] - at[3:]) <= 2.0**-4 * np.abs(at[3:]) + 2.0**-10 + 60 * ref.U * np.abs(at[3:]) + 2.0**-22).all()


@pytest.mark.parametrize("rows,width", [(2100, 1101), (1100, 2051), (1030, 4099), (520, 8195)])
def test_norm_gradient_over_rows_of_a_block(rows, width):
    """More rows than blocks, at widths whose rows begin anywhere: the gain's gradient over all of them."""
    torch = require_gpu()
    x, w = make(torch, ("float32", "float32"), rows, width, 0.0)
    plan = soma.RmsNorm(rows, width, torch.float32)
    total, y, dr, dg = torch.empty_like(x["x"]), torch.empty_like(x["x"]), torch.empty_like(x["x"]), torch.empty_like(x["gain"])
    plan.forward(x["x"], x["gain"], y, x["residual"], total)
    plan.backward(total, x["gain"], x["dy"], x["dtotal"], dr, None, dg)
    torch.cuda.synchronize()
    eps = np.float64(np.float32(1e-5))
    want = ref.norm(w["x"], w["residual"], w["gain"], eps, w["factor"])
    near(y, want["y"], want["y_err"], "float32", "y")
    back = ref.norm_backward(total.double().cpu().numpy(), w["gain"], w["dy"], w["dtotal"], eps, w["factor"])
    near(dr, back["dresidual"], back["dresidual_err"], "float32", "dresidual")
    near(dg, back["dgain"], back["dgain_err"], "float32", "dgain")


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("width", [5, 61, 509, 1001, 2051, 4099, 8195])
def test_norm_rows_beside_rows_that_are_not_finite(types, width):
    """Groups of eight that lie across two rows: what is not finite in one never reaches the other, nor do an array's
    neighbours in memory."""
    torch = require_gpu()
    T, S = types
    rows = 9
    x, _ = make(torch, types, rows, width, 0.0)
    plan = soma.RmsNorm(rows, width, getattr(torch, T), getattr(torch, S))

    def run(bad):
        a = {}
        for n in ("x", "residual", "dy", "dtotal"):          # NaN in front of and behind each array
            whole = torch.full((rows * width + 32,), float("nan"), dtype=x[n].dtype, device="cuda")
            a[n] = whole[16:16 + rows * width].view(rows, width)
            a[n].copy_(x[n])
        if bad:
            a["x"][1::2], a["dy"][1::2] = float("nan"), float("inf")
        gain = torch.full((width + 16,), float("nan"), device="cuda")[8:8 + width]
        gain.copy_(x["gain"])
        y, codes = torch.empty_like(a["x"]), torch.empty(rows, width, dtype=torch.float8_e4m3fn, device="cuda")
        t, s = torch.empty_like(a["residual"]), torch.empty(rows, device="cuda")
        plan.forward(a["x"], gain, codes, a["residual"], t, s)
        plan.forward(a["x"], gain, y, a["residual"], t)
        dr, dx = torch.empty_like(t), torch.empty_like(y)
        plan.backward(t, gain, a["dy"], a["dtotal"], dr, dx)
        torch.cuda.synchronize()
        return y, codes.float(), s, t, dr, dx

    for a, b in zip(run(False), run(True)):
        assert torch.isfinite(a).all() and torch.equal(a[::2], b[::2])


def test_norm_of_more_rows_than_one_launch_takes():
    """A wave a row: 2^25 rows a launch.  y = gain x / sqrt(x^2 + eps) in fp32: roundings of the square, its sum with eps
    (half of theirs is left by the root), the root, its reciprocal and two products, 6 u, and one for the division."""
    torch = require_gpu()
    n = 2**25 + 7
    x = torch.randn(n, 1, device="cuda")
    y, t = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    soma.RmsNorm(n, 1, torch.float32, eps=0.25).forward(x, torch.full((1,), 1.5, device="cuda"), y, None, t)
    torch.cuda.synchronize()
    assert torch.equal(t, x)
    want = 1.5 * x.double() / (x.double() ** 2 + 0.25).sqrt()
    assert ((y.double() - want).abs() <= 7 * 2.0**-24 * want.abs() + 1e-37).all()


def test_norm_rows_of_zeros_and_not_finite():
    """A row's values reach no other row; zeros give zeros, also without eps in 8 bits' scale."""
    torch = require_gpu()
    x, _ = make(torch, ("float32", "float32"), 6, 100, 0.0, residual=False)
    plan = soma.RmsNorm(6, 100, torch.float32)
    y, t = torch.empty_like(x["x"]), torch.empty_like(x["x"])
    plan.forward(x["x"], x["gain"], y, None, t)
    bad = x["x"].clone()
    bad[1, 3], bad[2, 99], bad[4] = float("nan"), float("inf"), 0.0
    z = torch.empty_like(y)
    plan.forward(bad, x["gain"], z, None, t)
    codes, scale = torch.empty(6, 100, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(6, device="cuda")
    plan.forward(bad, x["gain"], codes, None, None, scale)
    dr, dg = torch.empty_like(y), torch.empty_like(x["gain"])
    plan.backward(t, x["gain"], x["dy"], None, dr, None, dg)
    torch.cuda.synchronize()
    for r in (0, 3, 5):
        assert torch.equal(y[r], z[r]) and torch.isfinite(dr[r]).all() and torch.isfinite(scale[r])
    assert torch.isnan(z[1]).all() and (z[4] == 0).all() and torch.isnan(scale[1]) and torch.isnan(scale[2]) and scale[4] == 0
    assert (codes[4].float() == 0).all() and torch.isfinite(dr[4]).all()


def test_no_rows():
    torch = require_gpu()
    plan = soma.RmsNorm(5, 30, torch.bfloat16, torch.float32)
    x, t, g = (torch.zeros(0, 30, dtype=d, device="cuda") for d in (torch.bfloat16, torch.float32, torch.float32))
    gain, dg = torch.ones(30, device="cuda"), torch.full((30,), 7.0, device="cuda")
    plan.forward(x, gain, x.clone(), t, t.clone())
    plan.backward(t, gain, x, g, g.clone(), x.clone(), dg)
    soma.Dropout(5, 30, torch.bfloat16, 0.5).forward(x, x.clone())
    torch.cuda.synchronize()
    assert (dg == 0).all()


def test_captured_steps_draw_anew():
    """A step held on the device and counted up in the graph: every replay's mask is that step's."""
    torch = require_gpu()
    x, w = make(torch, ("bfloat16", "float32"), 40, 200, 0.4)
    plan, drop = soma.RmsNorm(40, 200, torch.bfloat16, torch.float32, drop=0.4), soma.Dropout(40, 200, torch.bfloat16, 0.4)
    step = torch.full((1,), 6, dtype=torch.int64, device="cuda")
    total, y, dr, dx = (torch.empty_like(t) for t in (x["dtotal"], x["dy"], x["dtotal"], x["dy"]))
    dg, z = torch.empty_like(x["gain"]), torch.empty_like(y)

    def run(step):
        plan.forward(x["x"], x["gain"], y, x["residual"], total, None, SEED, step, 1)
        plan.backward(total, x["gain"], x["dy"], x["dtotal"], dr, dx, dg, SEED, step, 1)
        drop.forward(x["x"], z, None, SEED, step, 2)

    run(step)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step += 1
        run(step)
    for n in (7, 8, 9):
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (total, y, dr, dx, dg, z)]
        run(n)
        torch.cuda.synchronize()
        for a, b in zip(got, (total, y, dr, dx, dg, z)):
            assert torch.equal(a, b)
        factor = ref.keep(40, 200, 0.4, SEED, n, 2)
        assert np.array_equal(got[5].double().cpu().numpy() != 0, (factor != 0) & (w["x"] != 0))


def test_on_another_stream():
    torch = require_gpu()
    x, _ = make(torch, ("float32", "float32"), 100, 333, 0.1)
    plan = soma.RmsNorm(100, 333, torch.float32, drop=0.1)
    side = torch.cuda.Stream()
    out = []
    for stream in (None, side):
        total, y, dr, dx, dg = (torch.empty_like(x[k]) for k in ("x", "x", "x", "x", "gain"))
        torch.cuda.synchronize()
        plan.forward(x["x"], x["gain"], y, x["residual"], total, None, SEED, STEP, LAYER, stream=stream)
        plan.backward(total, x["gain"], x["dy"], x["dtotal"], dr, dx, dg, SEED, STEP, LAYER, stream=stream)
        torch.cuda.synchronize()
        out.append((total, y, dr, dx, dg))
    for a, b in zip(*out):
        assert torch.equal(a, b)
