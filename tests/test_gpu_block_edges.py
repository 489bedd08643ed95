"""Calls of a residual block's operators at the ends of what they allow: no rows, outputs in place of inputs."""
import numpy as np
import pytest

import block_reference as ref
from gpu_common import require_gpu
from paper_2609_37899_amd import soma
from test_gpu_norm_dropout import LAYER, SEED, STEP, both, make, near

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("offsets", [False, True])
def test_linear_attention_of_no_rows(dtype, offsets):
    """States are kept, with and without offsets, in place too; without states there is nothing to do."""
    torch = require_gpu()
    dt = getattr(torch, dtype)
    plan = soma.LinearAttention(1000, 2, 4, 16, 24, dt, kv_heads=2)
    q, k, v, o = (torch.zeros(0, w, dtype=dt, device="cuda") for w in (64, 32, 48, 96))
    l = torch.full((4,), -0.1, device="cuda")
    off = torch.zeros(3, dtype=torch.int32, device="cuda") if offsets else None
    s, d = torch.randn(2, 4, 16, 24, device="cuda"), torch.randn(2, 4, 16, 24, device="cuda")
    sT, ds0 = torch.full_like(s, 7.0), torch.full_like(s, 7.0)
    s2, d2 = s.clone(), d.clone()
    plan.forward(q, k, v, l, o, s, sT, off)
    plan.forward(q, k, v, l, o, s2, s2, off)
    plan.forward(q, k, v, l, o, offsets=off)
    grads = [torch.zeros_like(t) for t in (q, k, v)]
    plan.backward(q, k, v, l, o, *grads, s, d, ds0, off)
    plan.backward(q, k, v, l, o, *grads, s, d2, d2, off)
    plan.backward(q, k, v, l, o, *grads, offsets=off)
    torch.cuda.synchronize()
    assert torch.equal(sT, s) and torch.equal(s2, s) and torch.equal(ds0, d) and torch.equal(d2, d)


def test_dropout_in_place_of_the_residual():
    """10 rows of 20, x 24 apart: y over the residual, and over x where its rows lie side by side."""
    torch = require_gpu()
    g = np.random.default_rng(6)
    x, x64 = both(torch, g.standard_normal((10, 20)), "float32", pad=4)
    r, r64 = both(torch, g.standard_normal((10, 20)), "float32")
    plan = soma.Dropout(10, 20, torch.float32, 0.1)
    y, c = r.clone(), x.contiguous()
    plan.forward(x, y, y, SEED, STEP, LAYER)
    plan.forward(c, c, r, SEED, STEP, LAYER)
    torch.cuda.synchronize()
    exact = ref.drop(x64, ref.keep(10, 20, 0.1, SEED, STEP, LAYER))
    near(y, exact + r64, ref.U * (2 * np.abs(exact) + np.abs(exact + r64)), "float32", "y")
    assert torch.equal(y, c)


def test_norm_in_place():
    """10 rows of 20, no multiple of 8: total over the residual, dresidual over dtotal."""
    torch = require_gpu()
    x, _ = make(torch, ("bfloat16", "float32"), 10, 20, 0.0)
    plan = soma.RmsNorm(10, 20, torch.bfloat16, torch.float32)
    total, y, r = torch.empty_like(x["residual"]), torch.empty_like(x["dy"]), x["residual"].clone()
    y2, dr, d = torch.empty_like(y), torch.empty_like(total), x["dtotal"].clone()
    plan.forward(x["x"], x["gain"], y, x["residual"], total)
    plan.forward(x["x"], x["gain"], y2, r, r)
    plan.backward(total, x["gain"], x["dy"], x["dtotal"], dr)
    plan.backward(total, x["gain"], x["dy"], d, d)
    torch.cuda.synchronize()
    assert torch.equal(r, total) and torch.equal(y, y2) and torch.equal(d, dr)


@pytest.mark.parametrize("sequences,heads", [(20485, 819), (65535, 256)])
def test_linear_attention_of_as_many_blocks_as_a_launch_has(sequences, heads):
    """2^24 - 1 blocks of 256 threads, and 2^24 - 256: o = scale q (k v + a s0) and its gradients.  A term is at the most a
    product of the matrix cores (which may cut: 2 u), one of a vector's lanes (1 u), a power of the decay (its exponent
    of 0.72 rounded twice, 1.1 u, and 2 u of its own), and the sum of both terms (2 u): 9 u."""
    torch = require_gpu()
    assert sequences * heads in (2**24 - 1, 2**24 - 256)
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, v, do = (torch.randn(sequences, heads, device="cuda", generator=g) for _ in range(4))
    s0, dsT = (torch.randn(sequences, heads, 1, 1, device="cuda", generator=g) for _ in range(2))
    l = torch.full((heads,), -0.5, device="cuda")
    a = l.double().exp()
    o, dq, dk, dv = (torch.full_like(q, 7.0) for _ in range(4))
    sT, ds0 = torch.full_like(s0, 7.0), torch.full_like(s0, 7.0)
    plan = soma.LinearAttention(sequences, sequences, heads, 1, 1, torch.float32, scale=0.5)
    plan.forward(q, k, v, l, o, s0, sT)
    plan.backward(q, k, v, l, do, dq, dk, dv, s0, dsT, ds0)
    torch.cuda.synchronize()

    def near(got, one, two):
        want, size = one + two, one.abs() + two.abs()
        assert ((got.double() - want).abs() <= 9 * 2.0**-24 * size + 1e-37).all()

    Q, K, V, D = (t.double() for t in (q, k, v, do))
    S, G = s0.double().view_as(q), dsT.double().view_as(q)
    near(o, 0.5 * Q * K * V, 0.5 * a * Q * S)
    near(sT.view_as(q), K * V, a * S)
    near(dq, 0.5 * D * V * K, 0.5 * a * D * S)
    near(dk, 0.5 * V * D * Q, V * G)
    near(dv, 0.5 * K * D * Q, K * G)
    near(ds0.view_as(q), 0.5 * a * Q * D, a * G)
