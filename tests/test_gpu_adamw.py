"""AdamW over many tensors against 64 bits: types, sizes, alignment, moments in 32 and in 8 bits."""
import numpy as np
import pytest

import train_reference as ref
from gpu_common import require_gpu
from paper_2609_37899_amd import soma

pytestmark = pytest.mark.gpu

SIZES = [1, 3, 4, 255, 256, 257, 4095, 4096, 4097, 10001, 0, 70000]
B1, B2, DELTA = 0.9, 0.999, 1e-8


def make(torch, ptype, gtype, bits, sizes, shift=0, seed=0):
    """Tensors that start `shift` elements into their memory."""
    g = np.random.default_rng(seed)

    def dev(x, dtype):
        y = torch.zeros(x.size + shift + 8, dtype=dtype, device="cuda")[shift:shift + x.size]
        y.copy_(torch.from_numpy(x))
        return y

    x = {"p": [], "g": [], "state": []}
    for k, n in enumerate(sizes):
        x["p"].append(dev(g.standard_normal(n).astype(np.float32), getattr(torch, ptype)))
        x["g"].append(dev((g.standard_normal(n) * 10.0 ** (k % 5 - 4)).astype(np.float32), getattr(torch, gtype)))
        if bits == 32:
            x["state"].append((dev((g.standard_normal(n) * 0.1).astype(np.float32), torch.float32),
                               dev((g.random(n) * 0.01).astype(np.float32), torch.float32)))
        else:
            b = -(-n // 256)
            codes = g.integers(0, 256, n).astype(np.uint8)
            codes[(codes & 127) == 127] = 5          # no NaN among the first moments
            x["state"].append((dev(codes, torch.uint8), dev(g.integers(0, 256, n).astype(np.uint8), torch.uint8),
                               dev((g.random(b) * 1e-3).astype(np.float32), torch.float32),
                               dev((g.random(b) * 1e-2).astype(np.float32), torch.float32)))
    return x


def arrays(state):
    return [t.cpu().numpy().copy() for t in state]


def expect(x, decay, t, lr, scale):
    out = []
    for p, g, s, w in zip(x["p"], x["g"], x["state"], decay):
        m, v = ref.moments_of(*arrays(s))
        out.append(ref.adamw(p.double().cpu().numpy(), g.double().cpu().numpy(), m, v, t, lr, B1, B2, DELTA, w, scale)
                   + (p.double().cpu().numpy(),))
    return out


def check_tensor(p, state, want, ptype, lr):
    np1, m, v, before = want
    got = p.double().cpu().numpy()
    # p: the product with 1 - lr decay, the update's ten roundings (sums of its terms' size), one to p's type
    tol = 4 * ref.U * np.abs(before) + 16 * ref.U * np.abs(np1 - before) + ref.half_step(ptype) * np.abs(np1) + 1e-37
    # lr decay p is part of np1 - before; a step near delta or with opposite terms: sqrt(v) carries 4 u
    assert np.all(np.abs(got - np1) <= tol + 16 * ref.U * lr * 4), np.max(np.abs(got - np1) / tol)
    gm, gv = ref.moments_of(*arrays(state))
    if len(state) == 2:
        # m's two terms may cancel: roundings of their size; v's have one sign
        assert np.all(np.abs(gm - m) <= 4 * ref.U * np.abs(m) + M_TERMS * ref.U)
        assert np.all(np.abs(gv - v) <= 6 * ref.U * v + 1e-44)
        return
    block = np.arange(m.size) // 256
    top_m = np.array([np.abs(m[block == b]).max() for b in range(block[-1] + 1)]) if m.size else np.zeros(0)
    r, gr = np.sqrt(v), np.sqrt(gv)
    top_r = np.array([r[block == b].max() for b in range(block[-1] + 1)]) if m.size else np.zeros(0)
    # half a step of e4m3 (3 bits of mantissa; subnormals of 2^-9 under the scale top / 448) and fp32's own error
    slack = 1 + 64 * ref.U
    assert np.all(np.abs(gm - m) <= (2.0 ** -4 * np.abs(m) + top_m[block] / 448 * 2.0 ** -10) * slack + M_TERMS * ref.U)
    # half a step of a root's code (4 bits of mantissa); the smallest code for what lies below it
    smallest = top_r[block] / 1.9375 * 17 / 16 * 2.0 ** -15
    assert np.all(np.abs(gr - r) <= np.maximum(2.0 ** -5 * r * slack + 8 * ref.U * r, smallest * slack))
    assert np.all((gr > 0) == (r > 0))


M_TERMS = 8.0        # |beta1 m| + |(1 - beta1) g| never exceeds this here: its roundings where the two cancel


@pytest.mark.parametrize("ptype,gtype", [("float32", "float32"), ("float32", "bfloat16"), ("bfloat16", "float32"),
                                         ("bfloat16", "bfloat16")])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [0, 1])
def test_matches_reference(ptype, gtype, bits, shift):
    torch = require_gpu()
    x = make(torch, ptype, gtype, bits, SIZES, shift)
    decay = [0.1 * (k % 3) for k in range(len(SIZES))]
    copies = [torch.zeros(n, dtype=torch.bfloat16, device="cuda") if k % 2 else None for k, n in enumerate(SIZES)]
    plan = soma.AdamW(x["p"], x["g"], bits=bits, weight_decay=decay, betas=(B1, B2), delta=DELTA, moments=x["state"],
                      copies=copies)
    scale = torch.tensor([0.5], device="cuda")
    for t in (1, 2, 1000):
        want = expect(x, decay, t, 1e-2, 0.5)
        plan.step(t, 1e-2, scale)
        torch.cuda.synchronize()
        for p, s, w in zip(x["p"], x["state"], want):
            check_tensor(p, s, w, ptype, 1e-2)
    outs = [[torch.zeros(n, device="cuda") for n in SIZES] for _ in range(2)]
    plan.moments(*outs)
    torch.cuda.synchronize()
    for k, s in enumerate(x["state"]):
        m, v = ref.moments_of(*arrays(s))
        assert np.all(np.abs(outs[0][k].cpu().numpy() - m) <= ref.U * np.abs(m))
        assert np.all(np.abs(outs[1][k].cpu().numpy() - v) <= 3 * ref.U * v + 1e-44)
        if copies[k] is not None:
            # the copy is the new parameter before its own rounding
            c, p = copies[k].double().cpu().numpy(), x["p"][k].double().cpu().numpy()
            assert np.all(np.abs(c - p) <= (2.0 ** -8 + ref.U) * np.abs(p))


@pytest.mark.parametrize("bits", [32, 8])
def test_from_zero_moments(bits):
    """The first update from zeros moves every parameter by lr against its gradient's sign, whatever the gradient's
    size within a block: a second moment that is not zero never becomes zero."""
    torch = require_gpu()
    n = 1000
    p = torch.zeros(n, device="cuda")
    g = (10.0 ** torch.linspace(-5, 2, n)).cuda() * torch.where(torch.arange(n).cuda() % 2 == 0, 1.0, -1.0)
    plan = soma.AdamW([p], [g], bits=bits, weight_decay=0.0)
    plan.step(1, 1e-3)
    torch.cuda.synchronize()
    # |g| / (|g| + delta), |g| >= 1e-5, delta = 1e-8
    assert torch.allclose(p, -1e-3 * torch.sign(g), rtol=1.1e-3, atol=0)
    before = p.clone()
    plan.step(2, 1e-3)
    torch.cuda.synchronize()
    assert torch.isfinite(p).all()
    # v is at least what the code keeps of it, so no step passes the exact one by more than the codes' half steps
    assert ((p - before).abs() <= 1e-3 * 1.2).all()


@pytest.mark.parametrize("ptype", ["float32", "bfloat16"])
def test_ordinary_blocks_as_any_other(ptype):
    """Moments in 8 bits take a shorter way where a block of 256 holds ordinary values only.  The same tensors, aligned
    and one element further on (which never takes it), blocks of every kind side by side."""
    torch = require_gpu()
    n = 4096 * 3 + 77
    x, y = (make(torch, ptype, ptype, 8, [n], shift) for shift in (0, 1))
    for z in (x, y):
        m, v, _, _ = z["state"][0]
        v.clamp_(min=1)                                   # no code 0
        g = z["g"][0]
        for k, (gv, mv, vv) in enumerate([(0.0, 0, 0), (1e-30, 0, 0), (1e18, 1, 1), (0.0, 40, 30), (float("inf"), 1, 1),
                                          (float("nan"), 1, 1), (1e-12, 0, 1), (3e38, 126, 255), (1e-14, 0, 0)]):
            b = slice(256 * (3 * k + 1), 256 * (3 * k + 2) if k % 2 else 256 * (3 * k + 1) + 5)
            g[b], m[b], v[b] = gv, mv, vv
    before = x["p"][0].double()
    plans = [soma.AdamW(z["p"], z["g"], bits=8, weight_decay=0.1, moments=z["state"]) for z in (x, y)]
    for t in (1, 2):
        for plan in plans:
            plan.step(t, 1e-2)
        torch.cuda.synchronize()
        a, b = x["p"][0].double(), y["p"][0].double()
        # the quotients differ by a reciprocal's 2 u and two roundings, the products by two, the root by 2 u at most,
        # then p's own roundings (its type's whole step where one falls the other way), and the first update's again
        tol = t * (8 * ref.U * (b - before).abs() + (2 * ref.U + 2 * ref.half_step(ptype)) * b.abs())
        same = torch.isfinite(b)
        assert torch.equal(torch.isfinite(a), same)
        assert ((a - b).abs()[same] <= tol[same]).all()
        for u, w in zip(x["state"][0][:2], y["state"][0][:2]):
            assert torch.equal(u, w)
        for u, w in zip(x["state"][0][2:], y["state"][0][2:]):
            assert ((u - w).abs() <= 4 * ref.U * w).all()


def test_non_finite_gradients_stay_their_own():
    torch = require_gpu()
    for bits in (32, 8):
        for bad in (float("nan"), float("inf"), -float("inf")):
            x = make(torch, "float32", "float32", bits, [600])
            y = make(torch, "float32", "float32", bits, [600])
            x["g"][0][300] = bad
            y["g"][0][300] = 0.0
            for z in (x, y):
                soma.AdamW(z["p"], z["g"], bits=bits, moments=z["state"]).step(1, 1e-3)
            torch.cuda.synchronize()
            keep = np.arange(600) != 300
            assert not torch.isfinite(x["p"][0][300])
            gx, gy = (ref.moments_of(*arrays(z["state"][0])) for z in (x, y))
            assert not np.isfinite(gx[0][300])
            assert np.array_equal(x["p"][0].cpu().numpy()[keep], y["p"][0].cpu().numpy()[keep])
            # the others' codes follow the largest finite value of the block: that of y unless element 300 held it
            other = np.arange(600) // 256 != 300 // 256
            assert np.array_equal(gx[0][other], gy[0][other]) and np.array_equal(gx[1][other], gy[1][other])
            assert np.isfinite(gx[0][keep]).all() and np.isfinite(gx[1][keep]).all()


def test_many_tensors_captured_and_on_another_stream():
    """450 tensors (their outputs take several launches), a captured step replayed against the eager one."""
    torch = require_gpu()
    sizes = [(37 * k) % 1000 + 1 for k in range(450)]
    x, y = (make(torch, "bfloat16", "bfloat16", 8, sizes) for _ in range(2))
    a, b = (soma.AdamW(z["p"], z["g"], bits=8, moments=z["state"]) for z in (x, y))
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    a.step(5, 1e-3, stream=st)
    b.step(5, 1e-3)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step(6, 1e-3)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        b.step(6, 1e-3)
        torch.cuda.synchronize()
        for k in range(len(sizes)):
            assert torch.equal(x["p"][k], y["p"][k])
            assert all(torch.equal(s, t) for s, t in zip(x["state"][k], y["state"][k]))
    outs = [[torch.zeros(n, device="cuda") for n in sizes] for _ in range(2)]
    a.moments(*outs)
    torch.cuda.synchronize()
    for k, s in enumerate(x["state"]):
        m, _ = ref.moments_of(*arrays(s))
        assert np.all(np.abs(outs[0][k].cpu().numpy() - m) <= ref.U * np.abs(m)), k


def test_refusals_and_closed_plans():
    torch = require_gpu()
    x = make(torch, "float32", "float32", 32, [100, 7])
    plan = soma.AdamW(x["p"], x["g"], moments=x["state"])
    before = [p.clone() for p in x["p"]]
    for bad in (dict(t=0, lr=1e-3), dict(t=1, lr=float("nan")), dict(t=1, lr=float("inf"))):
        with pytest.raises(soma.SomaError):
            plan.step(**bad)
    for bad in (dict(betas=(1.0, 0.999)), dict(betas=(0.9, -0.1)), dict(delta=0.0), dict(delta=float("nan"))):
        other = soma.AdamW(x["p"], x["g"], moments=x["state"], **bad)
        with pytest.raises(soma.SomaError):
            other.step(1, 1e-3)
    with pytest.raises(TypeError):
        plan.step(1, 1e-3, torch.ones(1, dtype=torch.float64, device="cuda"))
    with pytest.raises(ValueError):
        plan.step(1, 1e-3, torch.ones(2, device="cuda"))
    out = [torch.zeros(100, device="cuda"), torch.zeros(7, device="cuda")]
    for bad in (out[:1], [out[0], torch.zeros(8, device="cuda")], [out[0], torch.zeros(14, device="cuda")[::2]]):
        with pytest.raises(ValueError):
            plan.moments(bad, out)
    with pytest.raises(TypeError):
        plan.moments(out, [out[0], torch.zeros(7)])
    with pytest.raises(TypeError):
        plan.moments(out, [out[0].half(), out[1]])
    with pytest.raises(soma.SomaError):                    # the same tensor twice
        soma.AdamW(x["p"][:1] * 2, x["g"][:1] * 2)
    with pytest.raises(soma.SomaError):
        soma.AdamW(x["p"], x["p"])
    with pytest.raises(ValueError):
        soma.AdamW([torch.zeros(8, 8, device="cuda").t()], [torch.zeros(8, 8, device="cuda")])
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(x["p"], before))
    plan.close()
    with pytest.raises(RuntimeError):
        plan.step(1, 1e-3)


@pytest.mark.parametrize("bits", [32, 8])
def test_moments_from_zeros_used_on_another_stream(bits):
    """Moments that the plan makes itself, of many odd sizes, from the first step on on a stream of their own."""
    torch = require_gpu()
    sizes = [1, 0, 255, 300, 5000, 3]
    x = make(torch, "float32", "float32", 32, sizes)
    zero = [(torch.zeros(n, device="cuda"),) * 2 for n in sizes]
    want = expect(dict(x, state=zero), [0.0] * len(sizes), 1, 1e-2, 1.0)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    plan = soma.AdamW(x["p"], x["g"], bits=bits, weight_decay=0.0, betas=(B1, B2), delta=DELTA)
    plan.step(1, 1e-2, stream=st)
    torch.cuda.synchronize()
    for p, s, w in zip(x["p"], plan.state, want):
        assert s[0].numel() == p.numel() and all(t.data_ptr() % 256 == 0 for t in s)
        check_tensor(p, s, w, "float32", 1e-2)
