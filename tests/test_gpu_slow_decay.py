"""A decay's power over many rows: what the documentation allows it to be off by, whether one block walks them or pieces.

Rows of zeros leave a state a^n s0 (and its gradient a^n dsT), rounded once for every chunk of 32 rows (fp32) or 64
(bf16) on its way.  Those roundings, of states with mantissas of their own, have no common sign: of N states' relative
errors the mean has a deviation of at most chunks 2^-24 / sqrt(N).  What is left of the mean is the power's error, the
same for all of them: at most (3 |n log a| + 8) 2^-23."""
import math

import pytest

from gpu_common import require_gpu
from paper_2609_37899_amd import soma

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("heads,width", [(512, 4), (2, 64)], ids=["whole", "pieces"])
@pytest.mark.parametrize("log_decay,rows", [(-1e-7, 16384), (-3e-6, 16384), (-3e-6, 200000), (-1e-4, 16384), (-2e-4, 100000),
                                            (-0.02, 1000), (-0.03, 1000)])
def test_power_over_many_rows(dtype, heads, width, log_decay, rows):
    torch = require_gpu()
    dt = getattr(torch, dtype)
    rows = min(rows, 2**27 // (heads * width))
    plan = soma.LinearAttention(rows, 1, heads, width, width, dt)
    assert (plan._bytes > 0) == (heads == 2)
    zero = torch.zeros(rows, heads * width, dtype=dt, device="cuda")
    out = [torch.empty_like(zero) for _ in range(3)]
    l = torch.full((heads,), log_decay, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(11)
    s0, dsT = (torch.rand(1, heads, width, width, device="cuda", generator=gen) + 0.5 for _ in range(2))
    sT, ds0 = torch.empty_like(s0), torch.empty_like(s0)
    plan.forward(zero, zero, zero, l, out[0], s0, sT)
    plan.backward(zero, zero, zero, l, zero, *out, s0, dsT, ds0)
    torch.cuda.synchronize()
    nl = rows * l[0].double().item()
    chunks = rows / (32 if dtype == "float32" else 64)
    bound = (3 * abs(nl) + 8) * 2.0**-23 + 6 * chunks * 2.0**-24 / math.sqrt(s0.numel())
    for name, got, start in (("sT", sT, s0), ("ds0", ds0, dsT)):
        off = (got.double() / (start.double() * math.exp(nl)) - 1).mean().item()
        assert abs(off) <= bound, f"{name}: off by {off:.2e}, {abs(off) / bound:.2f} of the bound"
