"""Cross entropy of a linear head and its gradients against 64 bits: sizes around every tile and piece, types,
strides, rows without a target, values that are not finite, captured and repeated calls."""
import numpy as np
import pytest

import train_reference as ref
from gpu_common import require_gpu
from paper_2609_37899_amd import soma

pytestmark = pytest.mark.gpu


def make(torch, dtype, R, V, K, ignored=0.0, pad=(0, 0), shift=(0, 0), seed=0, scale=1.0):
    g = np.random.default_rng(seed)
    dt = getattr(torch, dtype)

    def rows(n, pad, shift, s):
        flat = torch.zeros(n * (K + pad) + shift + 8, dtype=dt, device="cuda")
        flat.fill_(float("nan"))                       # nothing between the rows is read
        y = flat[shift:shift + n * (K + pad)].view(n, K + pad)[:, :K]
        y.copy_(torch.from_numpy((g.standard_normal((n, K)) * s).astype(np.float32)))
        return y

    t = g.integers(0, V, R).astype(np.int32)
    t[g.random(R) < ignored] = -1
    w = (g.standard_normal(R) * 0.1).astype(np.float32)
    return {"f": rows(R, pad[0], shift[0], scale), "E": rows(V, pad[1], shift[1], 1.5 / np.sqrt(K)),
            "targets": torch.from_numpy(t).cuda(), "w": torch.from_numpy(w).cuda()}


def run(torch, plan, x, stream=None):
    R, dt = x["f"].shape[0], x["f"].dtype
    y = {k: torch.full((R,), 7.0, device="cuda") for k in ("loss", "lse")}
    y["df"] = torch.full((R, plan.width), 7.0, dtype=dt, device="cuda")
    y["dE"] = torch.full((plan.vocab, plan.width), 7.0, dtype=dt, device="cuda")
    plan.loss(x["f"], x["E"], x["targets"], y["loss"], y["lse"], stream=stream)
    plan.grad(x["f"], x["E"], x["targets"], y["lse"], x["w"], y["df"], y["dE"], stream=stream)
    return y


def host(t):
    return t.double().cpu().numpy()


def check(x, y, dtype, names=("loss", "lse", "df", "dE")):
    want = ref.cross_entropy(host(x["f"]), host(x["E"]), host(x["targets"]).astype(np.int64), host(x["w"]))
    K = x["f"].shape[1]
    # Each product of a sum is off by 2 u and every addition by u, accumulators of at most K / 32 + 32 in a row; fp32
    # operands are off by 4 u more (2^-22).  A sum of n such terms' errors is far below n u: sqrt is not relied on.
    n = {"loss": K / 32 + 40, "lse": K / 32 + 40}
    for name in names:
        got, exact = host(y[name]), want[name]
        terms = n.get(name, x["f"].shape[0] / 32 + x["E"].shape[0] / 32 + K / 32 + 40)
        tol = terms * ref.U * want[name + "_fp32"] + 1e-37
        if name in ("df", "dE"):
            if dtype == "bfloat16":
                tol = tol + 2.0 ** -8 * (1 + 2.0 ** -8) * want[name + "_g16"]
            else:
                tol = tol + want[name + "_tiny"]
            tol = tol * (1 + 2.0 ** -8) + ref.half_step(dtype) * np.abs(exact)
        bad = ~(np.abs(got - exact) <= tol)            # NaN counts as wrong
        assert not bad.any(), (f"{name}: {bad.sum()} of {bad.size}, worst {np.nanmax(np.abs(got - exact) / tol):.3g} of "
                               f"the bound, not finite {np.sum(~np.isfinite(got))}")
        if name in ("df", "dE") and exact.size:
            # and as a whole: errors of the type's size, not of the bounds' sums
            rel = np.linalg.norm(got - exact) / max(np.linalg.norm(exact), 1e-300)
            assert rel <= (6e-3 if dtype == "bfloat16" else 2e-5), (name, rel)
    return want


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("R,V,K", [
    (1, 1, 1), (1, 2, 8), (3, 5, 7), (1, 1000, 64), (16, 257, 100), (17, 256, 32), (64, 64, 64), (65, 129, 65),
    (300, 256, 512), (130, 1003, 361), (700, 300, 40), (256, 8192, 64), (40, 8193, 48), (90, 17000, 33),
    (1024, 9000, 128), (2100, 600, 257)])
def test_matches_reference(dtype, R, V, K):
    torch = require_gpu()
    x = make(torch, dtype, R, V, K, ignored=0.2 if R > 1 else 0.0)
    plan = soma.CrossEntropy(R, V, K, getattr(torch, dtype))
    y = run(torch, plan, x)
    torch.cuda.synchronize()
    check(x, y, dtype)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_large_tiles(dtype):
    """Sizes at which every product runs on the large tiles, one with shares of its columns and one with several
    items a block."""
    torch = require_gpu()
    R, V, K = 4096, 8400, 512
    x = make(torch, dtype, R, V, K, ignored=0.1)
    y = run(torch, soma.CrossEntropy(R, V, K, getattr(torch, dtype)), x)
    torch.cuda.synchronize()
    check(x, y, dtype)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("R", [5, 200])
@pytest.mark.parametrize("pad,shift", [((1, 0), (0, 0)), ((0, 3), (1, 1)), ((8, 8), (0, 0)), ((8, 4), (8, 4))])
def test_strides_and_alignment(dtype, R, pad, shift):
    torch = require_gpu()
    x = make(torch, dtype, R, 333, 72, 0.2, pad, shift)
    y = run(torch, soma.CrossEntropy(R, 333, 72, getattr(torch, dtype)), x)
    torch.cuda.synchronize()
    check(x, y, dtype)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("R", [6, 150])
def test_rows_without_a_target_count_for_nothing(dtype, R):
    """NaN, infinities and the type's lowest value in their f, and NaN in their weight, reach nothing; all rows
    without a target give zeros."""
    torch = require_gpu()
    V, K = 500, 40
    x = make(torch, dtype, R, V, K)
    x["targets"][:5] = -1
    for k, v in enumerate((float("nan"), float("inf"), -float("inf"), torch.finfo(x["f"].dtype).min)):
        x["f"][k] = v
    x["w"][1] = float("nan")
    y = run(torch, soma.CrossEntropy(R, V, K, getattr(torch, dtype)), x)
    torch.cuda.synchronize()
    x["f"][:5] = 0
    x["w"][:5] = 0
    check(x, y, dtype)
    assert (y["df"][:5] == 0).all() and (y["loss"][:5] == 0).all() and (y["lse"][:5] == 0).all()
    x["targets"][:] = -1
    y = run(torch, soma.CrossEntropy(R, V, K, getattr(torch, dtype)), x)
    torch.cuda.synchronize()
    assert all((y[k] == 0).all() for k in y)


@pytest.mark.parametrize("R", [4, 100])
def test_bad_targets_and_values_that_are_not_finite(R):
    torch = require_gpu()
    V, K = 300, 64
    for dtype in ("float32", "bfloat16"):
        plan = soma.CrossEntropy(R, V, K, getattr(torch, dtype))
        x = make(torch, dtype, R, V, K)
        x["targets"][2] = V                    # out of range: its loss is NaN, and the gradients that it enters
        y = run(torch, plan, x)
        torch.cuda.synchronize()
        assert torch.isnan(y["loss"][2]) and torch.isfinite(y["loss"][[0, 1, 3]]).all()
        assert torch.isfinite(y["lse"]).all()
        assert torch.isnan(y["df"][2]).all() and torch.isfinite(y["df"][[0, 1, 3]]).all()
        assert torch.isnan(y["dE"]).all()
        x = make(torch, dtype, R, V, K)
        x["f"][1, 3] = float("nan")            # a row with a target: its own results, and dE
        y = run(torch, plan, x)
        torch.cuda.synchronize()
        assert torch.isnan(y["loss"][1]) and torch.isfinite(y["loss"][[0, 2, 3]]).all()
        assert torch.isnan(y["df"][1]).all() and torch.isfinite(y["df"][[0, 2, 3]]).all()


@pytest.mark.parametrize("scale", [1e-20, 1e-4, 300.0])
def test_magnitudes(scale):
    """fp32 operands far from 1: the arrays' scales hold their precision.  (Logits reach 4 * 300.)"""
    torch = require_gpu()
    x = make(torch, "float32", 200, 700, 96, scale=scale)
    y = run(torch, soma.CrossEntropy(200, 700, 96, torch.float32), x)
    torch.cuda.synchronize()
    check(x, y, "float32")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_one_gradient_only_and_no_rows(dtype):
    torch = require_gpu()
    R, V, K = 100, 9000, 72
    x = make(torch, dtype, R, V, K, 0.1)
    plan = soma.CrossEntropy(R, V, K, getattr(torch, dtype))
    y = run(torch, plan, x)
    df, dE = torch.zeros_like(y["df"]), torch.zeros_like(y["dE"])
    plan.grad(x["f"], x["E"], x["targets"], y["lse"], x["w"], df, None)
    plan.grad(x["f"], x["E"], x["targets"], y["lse"], x["w"], None, dE)
    torch.cuda.synchronize()
    assert torch.equal(df, y["df"]) and torch.equal(dE, y["dE"])
    # fewer rows on the same plan, down to none: no row, no gradient
    for n in (40, 3, 0):
        z = {k: v[:n] if k != "E" else v for k, v in x.items()}
        y = run(torch, plan, z)
        torch.cuda.synchronize()
        if n:
            check(z, y, dtype)
        else:
            assert (y["dE"] == 0).all()


def test_gradient_against_differences():
    """df and dE against central differences of the weighted loss in 64 bits."""
    torch = require_gpu()
    R, V, K = 20, 50, 12
    x = make(torch, "float32", R, V, K)
    y = run(torch, soma.CrossEntropy(R, V, K, torch.float32), x)
    torch.cuda.synchronize()
    f, E, t, w = host(x["f"]), host(x["E"]), x["targets"].cpu().numpy(), host(x["w"])
    rng = np.random.default_rng(2)
    eps = 1e-5
    for name, a in (("df", f), ("dE", E)):
        for _ in range(10):
            i, j = rng.integers(a.shape[0]), rng.integers(K)
            keep = a[i, j]
            at = []
            for s in (eps, -eps):
                a[i, j] = keep + s
                at.append(np.sum(w * ref.cross_entropy(f, E, t)["loss"]))
            a[i, j] = keep
            num = (at[0] - at[1]) / (2 * eps)
            assert abs(num - float(y[name][i, j])) <= 1e-6 + 1e-5 * abs(num), name


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_captured_on_another_stream_and_repeated(dtype):
    torch = require_gpu()
    R, V, K = 300, 8500, 80
    x = make(torch, dtype, R, V, K, 0.1)
    plan, eager = (soma.CrossEntropy(R, V, K, getattr(torch, dtype)) for _ in range(2))
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    y = run(torch, plan, x, stream=st)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.loss(x["f"], x["E"], x["targets"], y["loss"], y["lse"])
        plan.grad(x["f"], x["E"], x["targets"], y["lse"], x["w"], y["df"], y["dE"])
    for k in range(3):
        z = make(torch, dtype, R, V, K, 0.1, seed=5 + k)
        for name in x:
            x[name].copy_(z[name])
        graph.replay()
        torch.cuda.synchronize()
        e = run(torch, eager, z)
        torch.cuda.synchronize()
        for name in y:
            assert torch.equal(y[name], e[name]), (k, name)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("R,V,K", [
    (17, 100, 64), (32, 777, 512), (33, 1000, 136), (49, 20000, 8), (64, 1, 96), (65, 5003, 1024), (100, 50, 72),
    (128, 3000, 64), (129, 3000, 64), (32, 300, 2304), (33, 300, 2304), (64, 70, 2304), (7, 65, 4616), (20, 65, 1200)])
def test_loss_of_some_rows(dtype, R, V, K):
    """Rows that take the head from memory as it lies, in one or two passes, and the numbers around those limits."""
    torch = require_gpu()
    x = make(torch, dtype, R, V, K, ignored=0.2)
    x["f"][3] = torch.where(x["targets"][3] < 0, float("inf"), x["f"][3])
    plan = soma.CrossEntropy(R, V, K, getattr(torch, dtype), grad=False)
    y = {k: torch.full((R,), 7.0, device="cuda") for k in ("loss", "lse")}
    plan.loss(x["f"], x["E"], x["targets"], y["loss"], y["lse"])
    torch.cuda.synchronize()
    want = ref.cross_entropy(host(x["f"]), host(x["E"]), host(x["targets"]).astype(np.int64))
    # a product and every addition are off by 2 u: accumulators of at most K / 4 in a row, and those of the exponentials
    for name in y:
        assert np.all(np.abs(host(y[name]) - want[name]) <= (K / 4 + 40) * ref.U * want[name + "_fp32"] + 1e-37), name
    # fewer rows in the same plan, to the same bits where the passes are alike, else within the bound
    n = R - 1
    loss, lse = torch.full((n,), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda")
    plan.loss(x["f"][:n], x["E"], x["targets"][:n], loss, lse)
    torch.cuda.synchronize()
    assert np.all(np.abs(host(loss) - want["loss"][:n]) <= (K / 4 + 40) * ref.U * want["loss_fp32"][:n] + 1e-37)
    assert np.all(np.abs(host(lse) - want["lse"][:n]) <= (K / 4 + 40) * ref.U * want["lse_fp32"][:n] + 1e-37)
