"""64-bit references of a residual block's operators, written from their formulas, and what fp32 arithmetic may differ
from them by, in roundings u = 2^-24."""
import numpy as np

U = 2.0 ** -24


def half_step(dtype):
    """Largest rounding to a type, relative to the value."""
    return {"float32": U, "bfloat16": 2.0 ** -8, "float8_e4m3fn": 2.0 ** -4}[dtype]


def linear_attention(q, k, v, log_decay, lengths, s0, scale, dtype="float32", do=None, dsT=None):
    """q [rows][H][dk], k [rows][K][dk], v [rows][K][dv] in float64.  Every pair of rows of a sequence and head.  Returns o,
    sT (and dq, dk, dv, ds0), each with its bound under the name + "_err"; rows behind the last sequence are NaN.

    Bounds, of the sum of the magnitudes of a result's terms, a term being one q_t k_s v_s or one through s0: a dot
    product over w columns is off by w u times two (the matrix cores may cut instead of round), a chunk's products by 64 u
    twice over, each power of a decay over n rows by 2 u n |log a| and 3 u, of which there are 3 and one more for every 32
    rows, as is a sum into the state (12 u).  bf16 adds the two parts that the products of a chunk and the state enter
    with, 2^-15, not in the states themselves.  Gradients of shared heads add their sum."""
    rows, H, dk = q.shape
    K, dv = v.shape[1], v.shape[2]
    share = H // K
    parts = 2.0 ** -15 if dtype == "bfloat16" else 0.0
    shapes = {"o": (rows, H, dv)}
    if do is not None:
        shapes.update(dq=(rows, H, dk), dk=(rows, K, dk), dv=(rows, K, dv))
    out = {}
    for name, shape in shapes.items():
        out[name], out[name + "_err"] = np.full(shape, np.nan), np.zeros(shape)
    used = sum(lengths)
    for name in shapes:
        out[name][:used] = 0.0
    out["sT"], out["sT_err"] = s0.copy(), np.zeros_like(s0)
    if do is not None:
        out["ds0"], out["ds0_err"] = dsT.copy(), np.zeros_like(dsT)
    first = 0
    a = np.abs
    for n, T in enumerate(lengths):
        at = slice(first, first + T)
        first += T
        if T == 0:
            continue
        t = np.arange(T, dtype=np.float64)
        apart = t[:, None] - t[None, :]
        past = apart >= 0
        for h in range(H):
            j, l = h // share, log_decay[h]

            def power(m):
                with np.errstate(invalid="ignore"):
                    return np.where(m == 0, 1.0, np.exp(l * m))

            def off(m):                     # relative error of a term that m rows lie between
                ml = np.where(power(m) > 0, m, 0) * (a(l) if np.isfinite(l) else 0.0)
                return U * (2 * (dk + dv) + 4 * 64 + share + 40 + 2 * ml + 15 * (m / 32))

            qh, kh, vh, S = q[at, h], k[at, j], v[at, j], s0[n, h]
            D = np.where(past, power(np.maximum(apart, 0)), 0.0) * scale
            E = np.where(past, off(np.maximum(apart, 0)) + parts, 0.0) * a(D)
            front, tail = power(t + 1) * scale, power(T - 1 - t)
            ef, et = (off(t + 1) + parts) * a(front), off(T - 1 - t) * tail
            A, Aa = qh @ kh.T, a(qh) @ a(kh).T
            out["o"][at, h] = (A * D) @ vh + front[:, None] * (qh @ S)
            out["o_err"][at, h] = (Aa * E) @ a(vh) + ef[:, None] * (a(qh) @ a(S))
            whole, ew = power(np.float64(T)), off(np.float64(T)) * power(np.float64(T))
            out["sT"][n, h] = whole * S + (kh * tail[:, None]).T @ vh
            out["sT_err"][n, h] = ew * a(S) + (a(kh) * et[:, None]).T @ a(vh)
            if do is None:
                continue
            g, G = do[at, h], dsT[n, h]
            dA, dAa = g @ vh.T, a(g) @ a(vh).T
            out["dq"][at, h] = (dA * D) @ kh + front[:, None] * (g @ S.T)
            out["dq_err"][at, h] = (dAa * E) @ a(kh) + ef[:, None] * (a(g) @ a(S).T)
            ets = et + parts * tail
            out["dk"][at, j] += (dA * D).T @ qh + tail[:, None] * (vh @ G.T)
            out["dk_err"][at, j] += (dAa * E).T @ a(qh) + ets[:, None] * (a(vh) @ a(G).T)
            out["dv"][at, j] += (A * D).T @ g + tail[:, None] * (kh @ G)
            out["dv_err"][at, j] += (Aa * E).T @ a(g) + ets[:, None] * (a(kh) @ a(G))
            out["ds0"][n, h] = whole * G + (qh * front[:, None]).T @ g
            out["ds0_err"][n, h] = ew * a(G) + (a(qh) * (off(t + 1) * a(front))[:, None]).T @ a(g)
    return out
