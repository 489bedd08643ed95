"""Moments in 8 bits rounded at random: the codes of one step against the formula, bit for bit, and the averages that a
run of many steps has to follow."""
import numpy as np
import pytest

import train_reference as ref
from gpu_common import require_gpu
from paper_2609_37899_amd import soma

F = np.float32
B1, B2 = 0.9, 0.999
M0, M1, W0, W1 = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85
LOW = np.uint64(0xFFFFFFFF)


def philox(c0, c1, c2, c3, k0, k1):
    """Philox4x32-10 of arrays of counters: four arrays of words."""
    x = [np.asarray(c, np.uint64) + np.zeros_like(np.asarray(c0, np.uint64)) for c in (c0, c1, c2, c3)]
    k0, k1 = int(k0), int(k1)
    for _ in range(10):
        p0, p1 = x[0] * np.uint64(M0), x[2] * np.uint64(M1)
        x = [(p1 >> np.uint64(32)) ^ x[1] ^ np.uint64(k0), p1 & LOW, (p0 >> np.uint64(32)) ^ x[3] ^ np.uint64(k1), p0 & LOW]
        k0, k1 = (k0 + W0) & 0xFFFFFFFF, (k1 + W1) & 0xFFFFFFFF
    return x


def test_philox_here_is_the_oracles(oracle_mod):
    for c, k in (((0, 0, 0, 0), (0, 0)), ((7, 3, 101, 1), (0xDEADBEEF, 0x12345678)), ((2**32 - 1,) * 4, (2**32 - 1,) * 2)):
        assert [int(w[0]) for w in philox(np.array([c[0]]), *c[1:], *k)] == [int(w) for w in oracle_mod.philox(c, k)]


def test_refusals_on_the_host():
    torch = pytest.importorskip("torch")
    assert soma.load().soma_adamw_set_rounding(None, 1, 0) == soma.SOMA_EINVAL
    x = torch.zeros(4)
    with pytest.raises(ValueError):
        soma.AdamW([x], [x.clone()], bits=8, rounding="up")


def draws(n, tensor, t, seed):
    """(v's, m's) draws of a tensor's n elements."""
    q = np.arange(-(-n // 4), dtype=np.uint64)
    w = np.stack(philox(q & LOW, tensor, t & 0xFFFFFFFF, q >> np.uint64(32), seed & 0xFFFFFFFF, (seed >> 32) ^ (t >> 32)), 1)
    w = w.reshape(-1)[:n]
    return w >> np.uint64(12), w & np.uint64(0xFFF)


def neighbours(table, y):
    """The table's values around y (upper: the largest for what lies above it)."""
    at = np.clip(np.searchsorted(table, y, side="right") - 1, 0, len(table) - 1)
    return at, table[at], table[np.minimum(at + 1, len(table) - 1)]


def expected_codes(codes_m, codes_v, sm, sv, g, tensor, t, seed):
    """Codes and scales of one step's moments in fp32, one rounding for every operation as the kernel has them."""
    n = g.size
    block = np.arange(n) // 256
    e = ref.e4m3_values()
    values = np.concatenate([e, [np.nan], -e, [np.nan]]).astype(F)
    r = ref.root_values().astype(F)[codes_v] * sv[block]
    m = F(B1) * (values[codes_m] * sm[block]) + F(1 - B1) * g
    v = F(B2) * (r * r) + F(1 - B2) * (g * g)
    root = np.sqrt(v)

    def top(x):
        y = np.zeros(-(-n // 256) * 256, F)
        y[:n] = x
        return y.reshape(-1, 256).max(1)

    tm, tr = top(np.abs(m)), top(root)
    with np.errstate(divide="ignore"):
        fm, fr = (np.where(x > F(1e-35), F(c) * (F(1) / x), F(0)).astype(F) for x, c in ((tm, 448), (tr, 1.9375)))
    dv, dm = draws(n, tensor, t, seed)
    a = np.abs(m * fm[block]).astype(np.float64)
    at, lo, hi = neighbours(e, a)
    with np.errstate(invalid="ignore", divide="ignore"):
        up = (dm + 0.5) / 4096 < np.where(hi > lo, (a - lo) / (hi - lo), 0.0)
    cm = (at + up).astype(np.uint8) | np.where(np.signbit(m), 128, 0).astype(np.uint8)
    y = (root * fr[block]).astype(np.float64)
    at, lo, hi = neighbours(ref.root_values(), y)
    with np.errstate(invalid="ignore", divide="ignore"):
        up = (dv + 0.5) / 2**20 < np.where(hi > lo, (y**2 - lo**2) / (hi**2 - lo**2), 0.0)
    cv = np.where(y > 0, np.maximum(at + up, 1), 0).astype(np.uint8)
    return cm, cv, tm * F(1 / 448), tr * F(1 / 1.9375)


def chunk_of(plan, sizes):
    """The elements of a block that the plan chose, from the size of its tables."""
    for chunk in (1024, 4096):
        blocks = sum(-(-n // chunk) for n in sizes)
        if plan.workspace.numel() == (len(sizes) * 80 + 255) // 256 * 256 + (blocks * 8 + 255) // 256 * 256:
            return chunk


def state_of(torch, g, n, shift):
    def dev(x, dtype):
        y = torch.zeros(x.size + shift, dtype=dtype, device="cuda")[shift:]
        y.copy_(torch.from_numpy(x))
        return y

    b = -(-n // 256)
    codes = g.integers(0, 256, n).astype(np.uint8)
    codes[(codes & 127) == 127] = 5
    root = g.integers(0, 256, n).astype(np.uint8)
    root[:512] = 0                                   # blocks that are not ordinary, and ones that are
    root[512:n // 2] |= 1
    return (dev(codes, torch.uint8), dev(root, torch.uint8),
            dev((g.random(b) * 1e-3 + 1e-4).astype(F), torch.float32), dev((g.random(b) * 1e-2 + 1e-3).astype(F), torch.float32))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("sizes,shift,chunk", [
    ([1, 255, 257, 5000, 0, 70001], 0, 1024), ([1, 255, 257, 5000, 0, 70001], 1, 1024),
    ([4099, 4_300_001], 0, 4096), ([4099, 4_300_001], 1, 4096)])
def test_codes_are_the_formulas(dtype, sizes, shift, chunk):
    torch = require_gpu()
    g = np.random.default_rng(3)
    dt = getattr(torch, dtype)
    p = [torch.zeros(n + shift, device="cuda", dtype=dt)[shift:] for n in sizes]
    grads = [torch.zeros(n + shift, device="cuda", dtype=dt)[shift:] for n in sizes]
    for x in grads:
        x.copy_(torch.from_numpy((g.standard_normal(x.numel()) * 10.0 ** g.integers(-4, 0)).astype(F)))
    state = [state_of(torch, g, n, shift) for n in sizes]
    seed, t = 0x1234567890ABCDEF, 2**32 + 77
    plan = soma.AdamW(p, grads, bits=8, weight_decay=0.0, betas=(B1, B2), moments=state, rounding="random", seed=seed)
    assert chunk_of(plan, sizes) == chunk
    before = [[x.cpu().numpy().copy() for x in s] for s in state]
    plan.step(t, 1e-3)
    torch.cuda.synchronize()
    for k, (s, b) in enumerate(zip(state, before)):
        if sizes[k] == 0:
            continue
        cm, cv, sm, sv = expected_codes(*b, grads[k].float().cpu().numpy(), k, t, seed)
        got = [x.cpu().numpy() for x in s]
        # A root or a block's factor of the short way may be off by one last bit (one in a million, and of a block 256
        # elements at once): a probability moves by 2^-18 then.  In fp32 a comparison may fall the other way where the
        # draw is within 2^-20 of the border.  So one code of neighbours in 2^16 elements may differ.
        for name, x, want in (("m", got[0].astype(int), cm.astype(int)), ("v", got[1].astype(int), cv.astype(int))):
            d = np.abs(x - want)
            # m's codes 0 and 128 are the zeros of either sign
            d = np.where((x & 127) + (want & 127) == 0, 0, d) if name == "m" else d
            assert d.max() <= 1 and (d > 0).sum() <= 1 + d.size / 2**16, (name, k, (d > 0).sum(), d.max())
        assert np.all(np.abs(got[2] - sm) <= 4 * ref.U * sm) and np.all(np.abs(got[3] - sv) <= 4 * ref.U * sv)


@pytest.mark.gpu
@pytest.mark.parametrize("n,chunk", [(256 * 64, 1024), (4096 * 1030, 4096)])
def test_averages_are_followed(n, chunk):
    """One element of 256 keeps its gradient, the others' has fallen tenfold: after 3,000 updates their v is where the
    recursion puts it.  (Rounded to nearest it stays where it was.)"""
    torch = require_gpu()
    lead = torch.arange(n, device="cuda") % 256 == 0
    grad = torch.where(lead, 1.0, 0.1) * torch.where(torch.arange(n, device="cuda") % 3 == 0, -1.0, 1.0)
    b = n // 256
    state = (torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.full((n,), 255, dtype=torch.uint8, device="cuda"),
             torch.zeros(b, device="cuda"), torch.full((b,), 1 / 1.9375, device="cuda"))       # m = 0, v = 1
    p = torch.zeros(n, device="cuda")
    plan = soma.AdamW([p], [grad], bits=8, weight_decay=0.0, betas=(B1, B2), moments=[state], rounding="random", seed=9)
    assert chunk_of(plan, [n]) == chunk
    m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    for t in range(1, 3001):
        plan.step(t, 1e-6)
        if t in (5, 300, 3000):
            plan.moments([m], [v])
            torch.cuda.synchronize()
            want_v = 0.01 + (1.0 - 0.01) * B2**t
            want_m = 0.1 * (1 - B1**t)
            for name, x, want in (("v", v[~lead], want_v), ("m", m[~lead] * torch.sign(grad[~lead]), want_m)):
                x = x.double() / want
                # the mean of independent elements, each expected where the recursion is; fp32 and the draws' 2^-12
                # steps shift it by far less than a thousandth
                assert abs(float(x.mean()) - 1) <= 5 * float(x.std()) / x.numel()**0.5 + 1e-3, (name, t, float(x.mean()))
                assert float(x.std()) <= 0.5, (name, t, float(x.std()))
    assert torch.isfinite(p).all()


@pytest.mark.gpu
def test_same_seed_same_bits_captured_and_of_two_plans():
    torch = require_gpu()
    g = np.random.default_rng(4)
    n = 9000

    def make():
        r = np.random.default_rng(5)
        return torch.zeros(n, device="cuda"), torch.from_numpy(r.standard_normal(n).astype(F)).cuda()

    runs = []
    for seed in (1, 1, 2):
        p, grad = make()
        plan = soma.AdamW([p], [grad], bits=8, rounding="random", seed=seed)
        if len(runs) == 1:                            # the second: a graph whose update is replayed
            plan.step(1, 1e-3)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                plan.step(2, 1e-3)
            for _ in range(3):
                graph.replay()
                torch.cuda.synchronize()
        else:
            for t in (1, 2, 2, 2):
                plan.step(t, 1e-3)
                torch.cuda.synchronize()
        runs.append([p] + list(plan.state[0]))
    assert all(torch.equal(a, b) for a, b in zip(runs[0], runs[1]))
    assert not torch.equal(runs[0][2], runs[2][2])
