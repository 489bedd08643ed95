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


@pytest.mark.parametrize("bits", [32, 8])
def test_rates_that_fp32_does_not_hold_are_refused(bits):
    """delta of 0 in fp32 would make 0 / 0 of an element without gradients; rates beyond fp32's range are infinite."""
    torch = require_gpu()
    p, grad = torch.ones(300, device="cuda"), torch.zeros(300, device="cuda")
    for delta in (1e-46, 1e39):
        plan = soma.AdamW([p], [grad], bits=bits, delta=delta)
        with pytest.raises(soma.SomaError):
            plan.step(1, 1e-3)
    plan = soma.AdamW([p], [grad], bits=bits, delta=1e-44)       # fp32's smallest values are among them
    for lr in (1e39, -1e39, 3e38):                               # 3e38 / (1 - 0.9)
        with pytest.raises(soma.SomaError):
            plan.step(1, lr)
    plan.step(1, 1e-3)
    torch.cuda.synchronize()
    assert torch.allclose(p, torch.full_like(p, 1 - 1e-5))       # the decay alone


def test_a_plan_is_not_made_in_a_capture_and_leaves_it_whole():
    torch = require_gpu()
    n = 300
    p, grad = torch.ones(n, device="cuda"), torch.ones(n, device="cuda")
    q = p.clone()
    moments = [(torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")) for _ in range(2)]
    plan, eager = soma.AdamW([p], [grad], moments=moments[:1]), soma.AdamW([q], [grad], moments=moments[1:])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.step(1, 1e-3)
        with pytest.raises(soma.SomaError, match="captured"):
            soma.AdamW([p], [grad], moments=moments[:1])
        plan.step(2, 1e-3)
    for _ in range(3):
        graph.replay()
        for t in (1, 2):
            eager.step(t, 1e-3)
        torch.cuda.synchronize()
        assert torch.equal(p, q) and all(torch.equal(a, b) for a, b in zip(*moments))
