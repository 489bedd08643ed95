"""64-bit references of the first-order operators, written from their formulas, and what fp32 arithmetic may
differ from them by.

Bounds count roundings: u = 2^-24 for every fp32 operation and for each correctly rounded elementary function, 2 u
for the hardware's exponential and reciprocal.  An exponential's argument x log2(e) carries 2 u |x| (the constant's
rounding and the product's), which the exponential turns into as much relative error."""
import numpy as np

U = 2.0 ** -24


def half_step(dtype):
    """Largest rounding to a type, relative to the value."""
    return {"float32": U, "bfloat16": 2.0 ** -8}[dtype]


def sigmoid(x):
    return 0.5 * (1.0 + np.tanh(0.5 * x))


def scan(gates, lengths, c0, dh=None, dcT=None):
    """gates [rows][4H] (float64), lengths of the sequences.  Returns a dict of h, cT (and dgates, dc0), each with its
    bound under the name + "_err"; rows behind the last sequence are NaN in h and dgates."""
    rows, H = gates.shape[0], gates.shape[1] // 4
    out = {"h": np.full((rows, H), np.nan), "h_err": np.zeros((rows, H)), "cT": c0.copy(), "cT_err": np.zeros_like(c0)}
    if dh is not None:
        out.update(dgates=np.full((rows, 4 * H), np.nan), dgates_err=np.zeros((rows, 4 * H)), dc0=dcT.copy(),
                   dc0_err=np.zeros_like(dcT))
    at = 0
    for s, n in enumerate(lengths):
        x = gates[at:at + n].reshape(n, 4, H)
        xi, xf, xg, xo = (x[:, k] for k in range(4))
        i, f, o, g = sigmoid(xi), sigmoid(xf), sigmoid(xo), np.tanh(xg)
        # sigma = 1 / (1 + e^-x): (2 |x| + 2) u e^-x / (1 + e^-x) from the exponential, u from the sum, 2 u + 0.5 u
        # from the reciprocal and the rounding
        ri, rf, ro = ((2 * np.abs(y) + 6) * U for y in (xi, xf, xo))
        # tanh = (1 - e) / (1 + e), e = e^-2|x|: absolute, at most (4 |x| + 2) u e + u + 4 u tanh
        tg = 8 * U
        c = np.empty((n + 1, H))
        ec = np.zeros((n + 1, H))
        c[0] = c0[s]
        for t in range(n):
            b = i[t] * g[t]
            c[t + 1] = f[t] * c[t] + b
            # maps of rows are composed in another order: 4 u more for each product and sum
            ec[t + 1] = f[t] * ec[t] + (rf[t] + 6 * U) * (np.abs(f[t] * c[t])) + (ri[t] + 6 * U) * np.abs(b) + tg * i[t]
        tc = np.tanh(c[1:])
        etc = ec[1:] + tg
        out["h"][at:at + n] = o * tc
        out["h_err"][at:at + n] = o * etc + (ro + U) * np.abs(o * tc)
        out["cT"][s], out["cT_err"][s] = c[n], ec[n]
        if dh is not None:
            d = dh[at:at + n]
            q, eq = dcT[s].copy(), np.zeros(H)
            for t in range(n - 1, -1, -1):
                w = 1 - tc[t] ** 2
                uu = d[t] * o[t] * w
                eu = np.abs(d[t] * o[t]) * (2 * etc[t] + 2 * U) + (ro[t] + 3 * U) * np.abs(uu)
                l, el = uu + q, eu + eq + 4 * U * (np.abs(uu) + np.abs(q))
                for k, (coef, err) in enumerate((
                        (g[t] * i[t] * (1 - i[t]), tg * 0.25 + np.abs(g[t]) * (2 * ri[t] * i[t] + 2 * U)),
                        (c[t] * f[t] * (1 - f[t]), ec[t] * 0.25 + np.abs(c[t]) * (2 * rf[t] * f[t] + 2 * U)),
                        (i[t] * (1 - g[t] ** 2), (ri[t] + 3 * U) * i[t] + 2 * tg * i[t]))):
                    out["dgates"][at + t, k * H:(k + 1) * H] = l * coef
                    out["dgates_err"][at + t, k * H:(k + 1) * H] = el * np.abs(coef) + np.abs(l) * (err + 3 * U * np.abs(coef))
                coef = tc[t] * o[t] * (1 - o[t])
                out["dgates"][at + t, 3 * H:] = d[t] * coef
                out["dgates_err"][at + t, 3 * H:] = np.abs(d[t]) * (etc[t] * 0.25 + 2 * ro[t] * o[t] + 5 * U)
                q, eq = f[t] * l, f[t] * el + (rf[t] + 6 * U) * np.abs(f[t] * l)
            out["dc0"][s], out["dc0_err"][s] = q, eq
        at += n
    return out


def e4m3_values():
    """The 127 values of e4m3 from 0 on."""
    v = [k * 2.0 ** -9 for k in range(8)] + [(1 + k / 8) * 2.0 ** (e - 7) for e in range(1, 16) for k in range(8)]
    return np.array(v[:127])


def root_values():
    return np.array([0.0] + [(16 + k % 16) * 2.0 ** (k // 16 - 19) for k in range(1, 256)])


def moments_of(m, v, m_scale=None, v_scale=None):
    """Values of moments as they are held (fp32, or codes with scales)."""
    if m_scale is None:
        return m.astype(np.float64), v.astype(np.float64)
    block = np.arange(m.size) // 256
    e = e4m3_values()
    table = np.concatenate([e, [np.nan], -e, [np.nan]])
    return (table[m] * m_scale.astype(np.float64)[block],
            (root_values()[v] * v_scale.astype(np.float64)[block]) ** 2)


def adamw(p, g, m, v, t, lr, b1, b2, delta, decay, scale=1.0):
    g = g * scale
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    return (1 - lr * decay) * p - lr * (m / (1 - b1 ** t)) / (np.sqrt(v / (1 - b2 ** t)) + delta), m, v


def cross_entropy(f, E, targets, w=None):
    """f [R][K], E [V][K] (float64), targets; rows with a negative target are left out.  Returns a dict of loss, lse
    (and df, dE) with bounds under the name + "_err" in units that the caller scales: "<name>_fp32", sums of absolute
    products (times 2^-24 and a small count), and "<name>_g16", what rounding the softmax's part to bf16 may add;
    "<name>_tiny" is the bound of what parts of fp32 operands in fp16's subnormals may add."""
    has = targets >= 0
    f = np.where(has[:, None], f, 0.0)
    at = np.where(has, targets, 0)
    l = f @ E.T
    mag = np.abs(f) @ np.abs(E).T                      # sums of absolute products
    top = l.max(1, keepdims=True)
    lse = (top + np.log(np.exp(l - top).sum(1, keepdims=True)))[:, 0]
    rows = np.arange(len(at))
    p = np.exp(l - lse[:, None])
    out = {"lse": np.where(has, lse, 0.0), "loss": np.where(has, lse - l[rows, at], 0.0)}
    # an error of every logit of e_l = d mag_rv moves lse by at most its average over p
    out["lse_fp32"] = np.where(has, (p * mag).sum(1) + np.abs(lse), 0.0)
    out["loss_fp32"] = np.where(has, (p * mag).sum(1) + mag[rows, at] + np.abs(out["loss"]) + np.abs(lse), 0.0)
    if w is None:
        return out
    w = np.where(has, w, 0.0)
    g = p.copy()
    g[rows, at] -= 1.0
    g *= w[:, None]
    out["df"], out["dE"] = g @ E, g.T @ f
    # a logit's error e_l changes p by p (e_l + its row's lse error); then the product's own sums
    gl = np.abs(w)[:, None] * p * (mag + (p * mag).sum(1, keepdims=True) + 2 * np.abs(l - lse[:, None]) + 1.0)
    out["df_fp32"] = gl @ np.abs(E) + np.abs(g) @ np.abs(E)
    out["dE_fp32"] = gl.T @ np.abs(f) + np.abs(g).T @ np.abs(f)
    # fp32 operands are two fp16 parts of x s, s a power of two that brings the array's largest to 2^13 or more: where
    # the second part is subnormal its rounding is 2^-25, so x is off by up to 2^-25 / s <= 2^-38 of the largest.
    # (G's largest counts as max |w|.)
    tiny = 2.0 ** -38
    c, mf, mE = np.abs(w).max(), np.abs(f).max(), np.abs(E).max()
    el = tiny * (mf * np.abs(E).sum(1)[None, :] + mE * np.abs(f).sum(1)[:, None])
    gt = np.abs(w)[:, None] * p * (el + (p * el).sum(1, keepdims=True)) + c * tiny
    out["df_tiny"] = gt @ np.abs(E) + tiny * mE * np.abs(g).sum(1, keepdims=True)
    out["dE_tiny"] = gt.T @ np.abs(f) + tiny * mf * np.abs(g).sum(0)[:, None]
    out["df_g16"], out["dE_g16"] = np.abs(g) @ np.abs(E), np.abs(g).T @ np.abs(f)
    return out
