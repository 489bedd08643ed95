"""AdamW at the ends of its ranges, and on blocks of either size."""
import numpy as np
import pytest

import train_reference as ref
from gpu_common import require_gpu
from paper_2609_37899_amd import soma

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rounding", ["nearest", "random"])
@pytest.mark.parametrize("bits", [0x7FC0, 0xFFC0, 0x7FFF, 0xFFFF, 0x7F80, 0xFF80])
def test_codes_of_gradients_that_are_not_finite(bits, rounding):
    """NaN of either sign and any payload, and infinities: m's code is NaN, v's the largest."""
    torch = require_gpu()
    p = torch.zeros(600, device="cuda", dtype=torch.bfloat16)
    grad = torch.ones(600, device="cuda", dtype=torch.bfloat16)
    grad.view(torch.int16)[300] = bits - (bits & 0x8000) * 2
    assert not torch.isfinite(grad[300])
    plan = soma.AdamW([p], [grad], bits=8, rounding=rounding)
    plan.step(1, 1e-3)
    torch.cuda.synchronize()
    m, v = (x.cpu().numpy() for x in plan.state[0][:2])
    assert m[300] & 127 == 127 and v[300] == 255
    assert not torch.isfinite(p[300]) and torch.isfinite(p[:300]).all() and torch.isfinite(p[301:]).all()
