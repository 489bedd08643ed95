"""Errors that the device's runtime remembers from a call of the program's own are not taken for the operators'."""
import ctypes

import pytest

from gpu_common import require_gpu
from paper_2609_37899_amd import soma

pytestmark = pytest.mark.gpu


def test_an_error_before_is_not_the_operators():
    torch = require_gpu()
    path = next(line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line)
    hip = ctypes.CDLL(path)
    n, H = 600, 16
    gates, h, dg = torch.randn(n, 4 * H, device="cuda"), torch.zeros(n, H, device="cuda"), torch.zeros(n, 4 * H, device="cuda")
    c = torch.zeros(1, H, device="cuda")
    scan, step = soma.GatedScan(n, 1, H, torch.float32), soma.GatedScan(1, 1, H, torch.float32)
    states = scan.new_states()
    f, E, t = torch.randn(200, H, device="cuda"), torch.randn(30, H, device="cuda"), torch.zeros(200, dtype=torch.int32, device="cuda")
    loss, lse, df, dE = (torch.zeros(s, device="cuda") for s in ((200,), (200,), (200, H), (30, H)))
    ce = soma.CrossEntropy(200, 30, H, torch.float32)
    p = torch.zeros(300, device="cuda")
    adamw = [soma.AdamW([p], [torch.ones(300, device="cuda")], bits=bits) for bits in (32, 8)]
    m, v = torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda")
    calls = [lambda: scan.forward(gates, h, None, None, states), lambda: scan.backward(gates, states, h, dg),
             lambda: step.step(gates[:1], None, c, h[:1]), lambda: ce.loss(f, E, t, loss, lse),
             lambda: ce.loss(f[:5], E, t[:5], loss[:5], lse[:5]), lambda: ce.grad(f, E, t, lse, loss, df, dE),
             lambda: ce.grad(f[:0], E, t[:0], lse[:0], loss[:0], None, dE),
             lambda: adamw[0].step(1, 1e-3), lambda: adamw[1].step(1, 1e-3), lambda: adamw[1].moments([m], [v])]
    torch.cuda.synchronize()
    for call in calls:
        assert hip.hipSetDevice(99) != 0                 # no such device: refused, and remembered
        try:
            call()
        finally:
            hip.hipGetLastError()
    torch.cuda.synchronize()
    assert (dE == 0).all() and torch.isfinite(p).all() and torch.isfinite(dg).all()
