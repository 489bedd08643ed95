"""Cross entropy with values at the ends of their ranges, and on each of the ways that its sizes choose between."""
import numpy as np
import pytest

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
