"""The gated linear recurrence at the ends of its ranges, against 64 bits."""
import numpy as np
import pytest

import train_reference as ref
from gpu_common import require_gpu
from paper_2609_37899_amd import soma

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("offsets", [False, True])
def test_no_rows(dtype, offsets):
    """Every sequence keeps its state and passes its gradient on; nothing else is written."""
    torch = require_gpu()
    S, H, dt = 5, 70, getattr(torch, dtype)
    plan = soma.GatedScan(0, S, H, dt)
    gates, h = (torch.zeros((0, k * H), dtype=dt, device="cuda") for k in (4, 1))
    off = torch.zeros(S + 1, dtype=torch.int32, device="cuda") if offsets else None
    c0, dcT = torch.randn(S, H, device="cuda"), torch.randn(S, H, device="cuda")
    cT, dc0 = torch.zeros(S, H, device="cuda"), torch.zeros(S, H, device="cuda")
    states = plan.new_states()
    plan.forward(gates, h, c0, cT, states, off)
    plan.backward(gates, states, h, torch.zeros((0, 4 * H), dtype=dt, device="cuda"), c0, dcT, dc0, off)
    torch.cuda.synchronize()
    assert torch.equal(cT, c0) and torch.equal(dc0, dcT)
