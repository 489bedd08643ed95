"""The 64-bit references themselves: gradients against central differences, and a recurrence row by row."""
import numpy as np
import pytest

import block_reference as ref


@pytest.mark.parametrize("heads,shared", [(2, 1), (3, 3)])
def test_linear_attention_is_its_recurrence_and_its_gradients_are_differences(heads, shared):
    g = np.random.default_rng(3)
    lengths, dk, dv, scale = [5, 0, 1, 7], 3, 4, 0.7
    rows = sum(lengths) + 2
    x = {"q": g.standard_normal((rows, heads, dk)), "k": g.standard_normal((rows, shared, dk)),
         "v": g.standard_normal((rows, shared, dv)), "s0": g.standard_normal((4, heads, dk, dv))}
    log_decay = np.array([-0.3, 0.0, -np.inf])[:heads]
    do, dsT = g.standard_normal((rows, heads, dv)), g.standard_normal((4, heads, dk, dv))

    def run(x, **kw):
        return ref.linear_attention(x["q"], x["k"], x["v"], log_decay, lengths, x["s0"], scale, **kw)

    out = run(x, do=do, dsT=dsT)
    at = 0
    for n, T in enumerate(lengths):
        S = x["s0"][n].copy()
        for t in range(at, at + T):
            for h in range(heads):
                j = h // (heads // shared)
                S[h] = np.exp(log_decay[h]) * S[h] + np.outer(x["k"][t, j], x["v"][t, j])
                assert np.allclose(out["o"][t, h], scale * x["q"][t, h] @ S[h], rtol=1e-12, atol=1e-12)
        assert np.allclose(out["sT"][n], S, rtol=1e-12, atol=1e-12)
        at += T
    assert np.isnan(out["o"][at:]).all() and np.isnan(out["dq"][at:]).all()

    def loss(x):
        y = run(x)
        return (y["o"][:at] * do[:at]).sum() + (y["sT"] * dsT).sum()

    for name, grad in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("s0", "ds0")):
        for i in g.permutation(out[grad].size)[:12]:
            i = np.unravel_index(i, out[grad].shape)
            if np.isnan(out[grad][i]):
                continue
            y = {k: v.copy() for k, v in x.items()}
            y[name][i] += 1e-4
            z = {k: v.copy() for k, v in x.items()}
            z[name][i] -= 1e-4
            # quadratic and cubic terms: the difference is exact up to 64-bit roundings and 1e-8 of the third order
            assert abs((loss(y) - loss(z)) / 2e-4 - out[grad][i]) < 1e-6 * (1 + abs(out[grad][i])), (name, i)


def test_norm_gradients_are_differences():
    g = np.random.default_rng(5)
    x, r, gain = g.standard_normal((4, 7)), g.standard_normal((4, 7)), 1 + 0.1 * g.standard_normal(7)
    dy, dt = g.standard_normal((4, 7)), g.standard_normal((4, 7))
    factor = ref.keep(4, 7, 0.4, 12345, 3, 1)
    out = ref.norm_backward(ref.norm(x, r, gain, 1e-3, factor)["total"], gain, dy, dt, 1e-3, factor)

    def loss(x, r, gain):
        y = ref.norm(x, r, gain, 1e-3, factor)
        return (y["y"] * dy).sum() + (y["total"] * dt).sum()

    for name, which in (("dx", 0), ("dresidual", 1), ("dgain", 2)):
        for i in np.ndindex(out[name].shape):
            a = [x.copy(), r.copy(), gain.copy()]
            b = [x.copy(), r.copy(), gain.copy()]
            a[which][i] += 1e-5
            b[which][i] -= 1e-5
            # third derivatives of a root of O(1): 1e-10 times some hundred, and 64-bit roundings over 1e-5
            assert abs((loss(*a) - loss(*b)) / 2e-5 - out[name][i]) < 1e-7


def test_mask_is_the_framework_s_philox(oracle_mod):
    """The generator's words against the oracle's."""
    g = np.random.default_rng(1)
    ctr = g.integers(0, 2**32, (50, 4), dtype=np.uint64)
    key = g.integers(0, 2**32, 2, dtype=np.uint64)
    mine = ref.philox(ctr, key)
    theirs = np.array([oracle_mod.philox(tuple(int(v) for v in c), tuple(int(v) for v in key)) for c in ctr], dtype=np.uint64)
    assert np.array_equal(mine, theirs)


def test_sample_by_hand():
    l = np.log(np.array([0.1, 0.4, 0.1, 0.4]))
    assert [ref.sample(l, u)[0] for u in (0.0, 0.099, 0.101, 0.499, 0.501, 0.599, 0.601, 0.999, 1.0)] == [0, 0, 1, 1, 2, 2, 3, 3, 3]
    assert ref.sample(l, 0.7, temperature=0)[0] == 1
    assert ref.sample(l, 0.999, top_k=1)[0] == 1 and ref.sample(l, 0.999, top_k=3)[0] == 3
    assert ref.sample(l, 0.01, top_k=3)[0] == 0 and ref.sample(l, 0.5, top_k=2, top_p=0.4)[0] == 1
    assert ref.sample(l, 0.999, top_p=0.3)[0] == 1 and ref.sample(l, 0.001, top_p=0.85)[0] == 0
    assert ref.sample(l, 0.999, min_p=0.5)[0] == 3 and ref.sample(l, 0.0, min_p=0.5)[0] == 1
    assert ref.sample(np.full(3, -np.inf), 0.5)[0] == -1 and ref.sample(np.array([np.nan, 1.0, -np.inf]), 0.9)[0] == 1
    assert [ref.sample(np.array([np.inf, 1.0, np.inf]), u)[0] for u in (0.2, 0.9)] == [0, 2]
