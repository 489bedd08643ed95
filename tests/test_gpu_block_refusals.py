"""What the classes of a residual block's operators refuse, and errors that are not theirs."""
import ctypes

import pytest

from gpu_common import require_gpu
from paper_2609_37899_amd import soma

pytestmark = pytest.mark.gpu


def z(*shape, dtype=None):
    import torch
    return torch.zeros(*shape, dtype=dtype or torch.float32, device="cuda")


def test_linear_attention():
    torch = require_gpu()
    plan = soma.LinearAttention(10, 2, 4, 8, 6, torch.float32, kv_heads=2)
    q, k, v, l, o = z(10, 32), z(10, 16), z(10, 12), z(4), z(10, 24)
    s = z(2, 4, 8, 6)
    off = torch.tensor([0, 3, 10], dtype=torch.int32, device="cuda")
    plan.forward(q, k, v, l, o, s, s, off)
    bad_type, bad_shape = (TypeError,), (ValueError,)
    for err, args in ((bad_type, (q.cpu(), k, v, l, o)), (bad_type, (q.bfloat16(), k, v, l, o)), (bad_type, (q, k, v, l.double(), o)),
                      (bad_shape, (q, k, v, z(2), o)), (bad_shape, (q, k[:, :8], v, l, o)), (bad_shape, (q, k, v, l, o[:9])),
                      (bad_shape, (z(11, 32), z(11, 16), z(11, 12), l, z(11, 24))), (bad_type, (q.view(-1), k, v, l, o)),
                      (bad_shape, (q.t().contiguous().t(), k, v, l, o)), (bad_shape, (q, k, v, l, z(10, 48)[:, ::2]))):
        with pytest.raises(err):
            plan.forward(*args)
    with pytest.raises(ValueError):
        plan.forward(q, k, v, l, o, s[:1])
    with pytest.raises(TypeError):
        plan.forward(q, k, v, l, o, None, s.bfloat16())
    with pytest.raises(TypeError):
        plan.forward(q, k, v, l, o, offsets=off.long())
    with pytest.raises(ValueError):
        plan.forward(q, k, v, l, o, offsets=off[:2])
    with pytest.raises(soma.SomaError):
        plan.forward(q[:9], k[:9], v[:9], l, o[:9])                # no offsets: a multiple of the sequences
    with pytest.raises(soma.SomaError):
        plan.step(q, k, v, l, s, s, o)                             # a row for every sequence
    flat = z(10 * 32 + 10 * 24)
    with pytest.raises(soma.SomaError):
        plan.forward(flat[:320].view(10, 32), k, v, l, flat[300:540].view(10, 24))
    g = z(10, 32), z(10, 16), z(10, 12)
    with pytest.raises(soma.SomaError):
        plan.backward(q, k, v, l, o, g[0], k, g[2])
    no = soma.LinearAttention(10, 2, 4, 8, 6, torch.float32, kv_heads=2, grad=False)
    with pytest.raises(ValueError):
        no.backward(q, k, v, l, o, *g)
    torch.cuda.synchronize()


def test_norm_and_dropout():
    torch = require_gpu()
    plan = soma.RmsNorm(10, 16, torch.bfloat16, torch.float32, drop=0.1)
    b, f, gain = z(10, 16, dtype=torch.bfloat16), z(10, 16), z(16)
    y = torch.zeros_like(b)
    plan.forward(b, gain, y, f, f)
    for err, args, kw in ((TypeError, (f, gain, y), {}), (TypeError, (b, gain.bfloat16(), y), {}), (ValueError, (b, z(15), y), {}),
                          (TypeError, (b, gain, f), {}), (TypeError, (b, gain, y), {"residual": b}), (ValueError, (b, gain, y[:9]), {}),
                          (TypeError, (b, gain, y), {"scale": z(10)}), (ValueError, (z(11, 16, dtype=torch.bfloat16), gain, y), {}),
                          (ValueError, (b, gain, y), {"layer": -1}), (TypeError, (b, gain, y), {"step": z(1)}),
                          (ValueError, (b, gain, y), {"step": torch.zeros(2, dtype=torch.int64, device="cuda")}),
                          (soma.SomaError, (b, gain, b), {})):
        with pytest.raises(err):
            plan.forward(*args, **kw)
    wide = z(10, 20)
    with pytest.raises(ValueError):
        plan.forward(b, gain, y, wide[:, :16], wide[:, :16])       # total has contiguous rows
    with pytest.raises(soma.SomaError):
        plan.backward(f, gain, y)                                  # nothing wanted
    with pytest.raises(soma.SomaError):
        plan.backward(f, gain, y, None, f)                         # dresidual over total
    with pytest.raises(TypeError):
        plan.backward(f, gain, f, None, z(10, 16))
    d = soma.Dropout(10, 16, torch.float32, 0.5)
    for err, args in ((TypeError, (b, f)), (ValueError, (f[:, :8], f)), (ValueError, (z(11, 16), z(11, 16))), (ValueError, (f, wide[:, :16]))):
        with pytest.raises(err):
            d.forward(*args)
    flat = z(200)
    with pytest.raises(soma.SomaError):
        d.forward(flat[:160].view(10, 16), flat[16:176].view(10, 16))
    torch.cuda.synchronize()


def test_sampler():
    torch = require_gpu()
    plan = soma.Sampler(8, 100, torch.float32)
    logits, u, tokens = z(8, 100), z(8), z(8, dtype=torch.int32)
    plan.sample(logits, u, tokens)
    for err, args, kw in ((TypeError, (logits.bfloat16(), u, tokens), {}), (ValueError, (logits[:, :99], u, tokens), {}),
                          (ValueError, (z(9, 100), z(9), z(9, dtype=torch.int32)), {}), (TypeError, (logits, u, tokens.long()), {}),
                          (ValueError, (logits, u[:7], tokens), {}), (TypeError, (logits, u, tokens), {"top_k": u}),
                          (TypeError, (logits, u, tokens), {"top_p": 0.9}), (ValueError, (logits, u, tokens), {"temperature": z(1)}),
                          (TypeError, (logits.view(-1), u, tokens), {}), (soma.SomaError, (logits, u, tokens), {"logprob": u})):
        with pytest.raises(err):
            plan.sample(*args, **kw)
    torch.cuda.synchronize()


def test_an_error_before_is_not_the_operators():
    """Errors that the device's runtime remembers from a call of the program's own are not taken for theirs."""
    torch = require_gpu()
    path = next(line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line)
    hip = ctypes.CDLL(path)
    n, E, H = 300, 16, 2
    x, l = torch.randn(n, H * E, device="cuda"), torch.full((H,), -0.1, device="cuda")
    out = [torch.zeros_like(x) for _ in range(4)]
    la, one = soma.LinearAttention(n, 1, H, E, E, torch.float32), soma.LinearAttention(1, 1, H, E, E, torch.float32)
    s = z(1, H, E, E)
    norm, drop, gain = soma.RmsNorm(n, H * E, torch.float32, drop=0.5), soma.Dropout(n, H * E, torch.float32, 0.5), z(H * E) + 1
    codes, scale = torch.zeros(n, H * E, dtype=torch.float8_e4m3fn, device="cuda"), z(n)
    u, tokens = z(n), z(n, dtype=torch.int32)
    few, many = soma.Sampler(n, H * E, torch.float32), soma.Sampler(2, 5000, torch.float32)
    logits, dgain = torch.randn(2, 5000, device="cuda"), z(H * E)
    u2, tokens2 = u[:2].clone(), tokens[:2].clone()
    x1, o1 = x[:1].clone(), z(1, H * E)
    calls = [lambda: la.forward(x, x, x, l, out[0], s, s), lambda: la.backward(x, x, x, l, out[0], *out[1:], s),
             lambda: one.step(x1, x1, x1, l, s, s, o1), lambda: norm.forward(x, gain, out[0], x, out[1]),
             lambda: norm.forward(x, gain, codes, None, None, scale), lambda: norm.backward(out[1], gain, x, None, out[2], out[3], dgain),
             lambda: drop.forward(x, out[3]), lambda: few.sample(x, u, tokens), lambda: many.sample(logits, u2, tokens2)]
    torch.cuda.synchronize()
    for call in calls:
        assert hip.hipSetDevice(99) != 0                 # no such device: refused, and remembered
        try:
            call()
        finally:
            hip.hipGetLastError()
    torch.cuda.synchronize()
    assert all(torch.isfinite(t).all() for t in out) and (tokens >= 0).all()
