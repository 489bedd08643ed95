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


def philox(ctr, key):
    """Philox4x32-10 of counters [n][4] and one key, uint64 arrays of 32-bit words."""
    x = [ctr[:, i].astype(np.uint64) for i in range(4)]
    k0, k1 = int(key[0]), int(key[1])
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(b >> np.uint64(32)) ^ x[1] ^ np.uint64(k0), b & low, (a >> np.uint64(32)) ^ x[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(x, 1)


def keep(rows, width, p, seed, step, layer, first=0):
    """The factor of every element of rows first .. first + rows - 1: 0, or 65536 / (65536 - cut)."""
    cut = round(p * 65536)
    lo, hi = first * width, (first + rows) * width
    b = np.arange(lo // 8, -(-hi // 8), dtype=np.uint64)
    s, t = int(seed) % 2**64, int(step) % 2**64
    ctr = np.stack([b & np.uint64(0xFFFFFFFF), np.full_like(b, layer), np.full_like(b, t & 0xFFFFFFFF), b >> np.uint64(32)], 1)
    w = philox(ctr, (s & 0xFFFFFFFF, (s >> 32) ^ (t >> 32)))
    fields = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], 2).reshape(-1)
    kept = fields[lo - lo // 8 * 8:][:hi - lo] >= cut
    return (kept * (65536 / (65536 - cut))).reshape(rows, width)


def drop(x, factor):
    """What is dropped counts as 0, whatever it is."""
    return np.where(factor == 0, 0.0, x) * factor


def norm(x, residual, gain, eps, factor):
    """total and y, and their bounds before they are rounded to their types.

    The factor carries 1 u, its product and the sum 1 each; the mean of squares at most 64 u (sums of up to 40 terms a
    lane and 10 halvings), half of it in the root; root, division, products: 6."""
    t = drop(x, factor) + (0 if residual is None else residual)
    et = U * (2 * np.abs(drop(x, factor)) + np.abs(t))
    n = x.shape[1]
    square = (t * t).mean(1, keepdims=True) + eps
    inv = 1 / np.sqrt(square)
    y = gain * t * inv
    ei = 40 * U + (np.abs(t) * et).sum(1, keepdims=True) / n / square
    return {"total": t, "total_err": et, "y": y, "y_err": np.abs(gain) * inv * et + (ei + 6 * U) * np.abs(y)}


def norm_backward(t, gain, dy, dtotal, eps, factor):
    """From the total as it is stored: dresidual, dx, dgain and their bounds."""
    rows, n = t.shape
    inv = 1 / np.sqrt((t * t).mean(1, keepdims=True) + eps)
    x, h = t * inv, dy * gain
    m, ma = (h * x).mean(1, keepdims=True), np.abs(h * x).mean(1, keepdims=True)
    d = (0 if dtotal is None else dtotal) + inv * (h - x * m)
    size = inv * (np.abs(h) + np.abs(x) * np.abs(m))
    e = U * (100 * size + 2 * np.abs(d) + 120 * inv * np.abs(x) * ma)
    # a lane's rows one after another, waves, blocks in 16 columns
    return {"dresidual": d, "dresidual_err": e, "dx": drop(d, factor), "dx_err": (e + 2 * U * np.abs(d)) * factor,
            "dgain": (dy * x).sum(0), "dgain_err": U * (100 + rows / 512 + 64) * np.abs(dy * x).sum(0)}


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row: (token, its share's logarithm, how near u comes to another token, in shares)."""
    l = np.where(np.isnan(logits), -np.inf, logits.astype(np.float64))
    top = l.max()
    if top == -np.inf:
        return -1, -np.inf, 1.0
    order = np.argsort(-l, kind="stable")
    if not temperature > 0:
        return int(order[0]), 0.0, 1.0
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(l == top, 1.0, np.where((l == -np.inf) | (top == np.inf), 0.0, np.exp((l - top) / temperature)))
    order = order[l[order] > -np.inf]
    near = 1.0
    if top_k > 0:
        order = order[:top_k]
    if top_p < 1:
        before = np.cumsum(w[order]) - w[order]
        limit = max(float(top_p), 0.0) * w[order].sum()
        if order.size > 1:                 # the first stays whatever the limit
            near = min(near, np.abs(before[1:] - limit).min() / w[order].sum())
        stay = before < limit
        stay[0] = True
        order = order[stay]
    if min_p > 0:
        order = order[w[order] >= min(float(min_p), 1.0)]
    order = np.sort(order)
    run = np.cumsum(w[order])
    share = run / run[-1]
    u = min(max(float(u), 0.0), 1.0)
    at = min(int(np.searchsorted(share, u, side="right")), int(np.nonzero(w[order])[0][-1]))
    near = min(near, np.abs(share[:-1] - u).min() if share.size > 1 else 1.0)
    return int(order[at]), float(np.log(w[order[at]] / run[-1])), near
