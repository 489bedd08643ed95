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
