"""Cross entropy with values at the ends of their ranges, and on each of the ways that its sizes choose between."""
import numpy as np
import pytest

import train_reference as ref
from gpu_common import require_gpu
from paper_2609_37899_amd import soma
from test_gpu_cross_entropy import check, host, make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("R,V", [(6, 300), (150, 300), (300, 9000)])
@pytest.mark.parametrize("weight", [float("inf"), -float("inf"), float("nan")])
def test_a_weight_that_is_not_finite_is_its_rows_alone(dtype, R, V, weight):
    """df of the other rows is what it is without that row; its own, and dE, which it enters, are not finite."""
    torch = require_gpu()
    x = make(torch, dtype, R, V, 48)
    plan = soma.CrossEntropy(R, V, 48, getattr(torch, dtype))
    others = torch.arange(R, device="cuda") != 2
    for w in (x["w"].clone(), torch.zeros(R, device="cuda")):
        x["w"] = w.clone()
        x["w"][2] = 0.0
        want = run(torch, plan, x)
        x["w"][2] = weight
        got = run(torch, plan, x)
        torch.cuda.synchronize()
        assert torch.isfinite(want["df"]).all()
        assert torch.equal(got["df"][others], want["df"][others])
        assert not torch.isfinite(got["df"][2]).any() and not torch.isfinite(got["dE"]).any()


@pytest.mark.parametrize("dtype,R,V,K", [
    ("bfloat16", 65, 9000, 1024), ("bfloat16", 100, 9000, 1024), ("bfloat16", 128, 9000, 1024), ("bfloat16", 97, 16391, 513),
    ("float32", 33, 5003, 1024), ("float32", 45, 5003, 1024), ("float32", 63, 8200, 513)])
def test_loss_of_rows_in_two_passes(dtype, R, V, K):
    """Heads above 16 MiB, of which 65 to 128 rows (fp32: 33 to 64) take two readings: whole second passes and passes of
    fewer rows than their tiles."""
    torch = require_gpu()
    x = make(torch, dtype, R, V, K, ignored=0.2)
    assert V * K * x["E"].element_size() >= 1 << 24
    x["f"][3] = torch.where(x["targets"][3] < 0, float("inf"), x["f"][3])
    plan = soma.CrossEntropy(R, V, K, getattr(torch, dtype), grad=False)
    for n in (R, R - 1, (64 if dtype == "bfloat16" else 32) + 1):
        y = {k: torch.full((n,), 7.0, device="cuda") for k in ("loss", "lse")}
        plan.loss(x["f"][:n], x["E"], x["targets"][:n], y["loss"], y["lse"])
        torch.cuda.synchronize()
        want = ref.cross_entropy(host(x["f"][:n]), host(x["E"]), host(x["targets"][:n]).astype(np.int64))
        # a product and every addition are off by 2 u: accumulators of at most K / 4 in a row, and those of the exponentials
        for name in y:
            assert np.all(np.abs(host(y[name]) - want[name]) <= (K / 4 + 40) * ref.U * want[name + "_fp32"] + 1e-37), name


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("R,V,K", [(8200, 8193, 24), (2048, 17000, 1024)])
def test_gradients_over_several_pieces(dtype, R, V, K):
    """More than 8,192 rows, whose pieces are 8,192 of the vocabulary; and a df of large tiles that is the sum of shares
    and of pieces, the last one of too few columns for all shares."""
    torch = require_gpu()
    x = make(torch, dtype, R, V, K, ignored=0.1)
    y = run(torch, soma.CrossEntropy(R, V, K, getattr(torch, dtype)), x)
    torch.cuda.synchronize()
    check(x, y, dtype)
