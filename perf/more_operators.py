"""The operators of a residual block without recurrent products, in training and in serving, as they are timed and
compared:

* linear attention with a decay for each head (``soma.LinearAttention``): a recurrence whose state is a matrix, in
  chunks for prompts and training, with its backward pass and its form for single tokens;
* root-mean-square norm with the residual's addition (``soma.RmsNorm``), the branch dropped out at random on its way,
  its backward pass, and its output in 8 bits with a scale for each row;
* dropout from the counter-based generator (``soma.Dropout``), whose mask is never stored;
* the draw of the next token from logits (``soma.Sampler``) with temperature, top-k, top-p and min-p, from given random
  numbers.

``run`` computes them from elementary torch operations, or, where ``own`` is set, through the framework's entry points.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}
EPS = 1e-5                       # of the norm
CHUNK = 128                      # rows that the plain linear attention takes at once


def _la(call, sequences, length, heads, kv_heads, key_width, value_width, dtype, ragged=False, pad=0, name=None):
    """call: "step" (one token for every sequence), "forward" or "train" (forward and backward); ragged: sequences of
    different lengths, some empty, ``length`` rows on average, and rows behind the last one; pad: elements between the end
    of a row of q, k or v and the next."""
    c = {"op": "la", "call": call, "sequences": sequences, "length": length, "heads": heads, "kv_heads": kv_heads,
         "key_width": key_width, "value_width": value_width, "dtype": dtype, "ragged": ragged, "pad": pad}
    return dict(c, name=name) if name else c


def _norm(call, rows, width, dtype, sum_dtype, drop=0.0, name=None):
    """call: "forward", "codes" (forward with the output in 8 bits) or "train" (forward and backward); sum_dtype: type of
    the residual and of the sum; drop: probability of dropping an element of the branch."""
    c = {"op": "norm", "call": call, "rows": rows, "width": width, "dtype": dtype, "sum_dtype": sum_dtype, "drop": drop}
    return dict(c, name=name) if name else c


def _drop(rows, width, dtype, drop, residual, name=None):
    c = {"op": "drop", "rows": rows, "width": width, "dtype": dtype, "drop": drop, "residual": residual}
    return dict(c, name=name) if name else c


def _sample(rows, vocab, dtype, top_k, top_p, min_p, pad=0, name=None):
    """Filters are switched on by truth values; each row has its own settings."""
    c = {"op": "sample", "rows": rows, "vocab": vocab, "dtype": dtype, "top_k": top_k, "top_p": top_p, "min_p": min_p,
         "pad": pad}
    return dict(c, name=name) if name else c


def listed():
    return [
        # One token for each of 64 sequences that are being generated: eight
        # states of 64 x 64 each, read and written.
        _la("step", 64, 1, 8, 8, 64, 64, "bfloat16", name="la_token"),
        # A training batch at the default workload's width: 64 windows of 1,024
        # tokens, H = 512 as 8 heads of 64.
        _la("train", 64, 1024, 8, 8, 64, 64, "bfloat16", name="la_train_h512"),
        # Documents of different lengths behind one another, empty ones among
        # them, widths nobody rounded, keys and values shared by all heads.
        _la("train", 37, 600, 5, 1, 45, 77, "float32", ragged=True, pad=3, name="la_ragged_odd"),
        # One prompt of 16,384 tokens on its way into a state.
        _la("forward", 1, 16384, 16, 16, 128, 128, "bfloat16", name="la_prompt"),
        # The norm of one token for each of 64 sequences, in 8 bits for the
        # product that follows.
        _norm("codes", 64, 512, "bfloat16", "bfloat16", name="norm_token"),
        # The wide control's width, which no vector load divides.
        _norm("train", 22000, 361, "float32", "float32", drop=0.25, name="norm_odd_d361"),
        # A training batch: branches in bfloat16, the residual's sum in fp32,
        # a tenth of the branch dropped.
        _norm("train", 65536, 512, "bfloat16", "float32", drop=0.1, name="norm_train_h512"),
        # Long prompts through a wide layer that is served in 8 bits.
        _norm("codes", 16384, 4096, "bfloat16", "bfloat16", name="norm_codes_d4096"),
        # Dropout of one small batch: launches and latency count.
        _drop(64, 512, "float32", 0.1, False, name="drop_small"),
        # Dropout of a training batch's branch and its addition to the residual.
        _drop(65536, 1024, "bfloat16", 0.1, True, name="drop_train"),
        # The next byte of 64 sequences.
        _sample(64, 256, "float32", True, True, True, name="sample_bytes"),
        # The next token of 256 sequences from a vocabulary of 50,257.
        _sample(256, 50257, "bfloat16", True, True, True, name="sample_50k"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("la", "la", "la", "norm", "norm", "drop", "sample", "sample"))
    dtype = rng.choice(sorted(DTYPES))
    if kind == "la":
        call = rng.choice(("step", "forward", "train", "train"))
        while True:
            n = _log_int(rng, 1, 256)
            t = 1 if call == "step" else _log_int(rng, 1, 16384)
            kv = rng.choice((1, 1, 2, 3, 4, 8))
            heads = kv * rng.choice((1, 1, 2, 3, 4))
            dk, dv = (rng.choice((rng.choice((16, 32, 64, 128)), _log_int(rng, 8, 192))) for _ in range(2))
            c = _la(call, n, t, heads, kv, dk, dv, dtype, call != "step" and rng.random() < 0.5, rng.choice((0, 0, 1, 8)))
            w = work(c)
            # fp32 products cost several times bfloat16's in either form; a
            # ragged batch's plain form is filled up to its longest sequence
            cost = w["flops"] * (8 if dtype == "float32" else 1) * (3 if c["ragged"] else 1)
            if w["bytes"] <= 7e8 and cost <= 1.5e11 and n * heads * dk * dv <= 2 ** 25:
                return c
    if kind == "norm":
        call = rng.choice(("forward", "codes", "train", "train"))
        sum_dtype = "float32" if dtype == "float32" else rng.choice(sorted(DTYPES))
        while True:
            c = _norm(call, _log_int(rng, 1, 65536), _log_int(rng, 16, 8192), dtype, sum_dtype,
                      rng.choice((0.0, 0.1, rng.uniform(0.0, 0.6))))
            if c["rows"] * c["width"] <= 65536 * 512:
                return c
    if kind == "drop":
        while True:
            c = _drop(_log_int(rng, 1, 65536), _log_int(rng, 1, 8192), dtype, rng.uniform(0.01, 0.6), rng.random() < 0.5)
            if c["rows"] * c["width"] <= 65536 * 1024 // (2 if dtype == "float32" else 1):
                return c
    while True:
        c = _sample(_log_int(rng, 1, 512), _log_int(rng, 2, 131072), dtype, rng.random() < 0.5, rng.random() < 0.5,
                    rng.random() < 0.3, rng.choice((0, 0, 1, 8)))
        if c["rows"] * c["vocab"] <= 256 * 50257:
            return c


# --------------------------------------------------------------------------
# Sizes

def _lengths(c):
    """Rows of every sequence, and of the whole array."""
    n, t = c["sequences"], c["length"]
    if not c["ragged"]:
        return [t] * n, n * t
    # Lengths between 0 and about three times the mean, a fixed pattern.
    share = [((7 * i + 3) % 11) ** 2 for i in range(n)]
    share[0] = max(1, share[0])
    scale = n * t / sum(share)
    lengths = [0 if i % 9 == 5 else int(s * scale) for i, s in enumerate(share)]
    return lengths, sum(lengths) + 5


def _size(name):
    return 2 if name == "bfloat16" else 4


def work(case):
    c = case
    e = _size(c["dtype"])
    if c["op"] == "la":
        lengths, _ = _lengths(c)
        n, dk, dv = sum(lengths), c["key_width"], c["value_width"]
        keys, values = c["kv_heads"] * dk, c["kv_heads"] * dv
        q, o = c["heads"] * dk, c["heads"] * dv
        state = len(lengths) * c["heads"] * dk * dv * 4
        # the recurrence itself: a state's update, and its product with a query
        flops = 5.0 * n * c["heads"] * dk * dv
        if c["call"] == "train":            # states: in and out, and the same of their gradients
            return {"bytes": float(n * e * (3 * q + 3 * keys + 3 * values + 2 * o) + 5 * state), "flops": 3.6 * flops}
        return {"bytes": float(n * e * (q + keys + values + o) + 2 * state), "flops": flops}
    if c["op"] == "norm":
        n, s = c["rows"] * c["width"], _size(c["sum_dtype"])
        if c["call"] == "train":            # x, residual, dy and dtotal in; sum (read back), y, dresidual and dx out
            return {"bytes": float(n * (4 * e + 5 * s) + 8 * c["width"]), "flops": 18.0 * n}
        return {"bytes": float(n * (e + 2 * s + (1 if c["call"] == "codes" else e)) + 4 * c["rows"]), "flops": 6.0 * n}
    if c["op"] == "drop":
        n = c["rows"] * c["width"]
        return {"bytes": float(n * e * (3 if c["residual"] else 2)), "flops": 2.0 * n}
    return {"bytes": float(c["rows"] * (c["vocab"] * e + 28)), "flops": 10.0 * c["rows"] * c["vocab"]}


# --------------------------------------------------------------------------
# Inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) & 0x7FFFFFFF)
    return g


def _normal(n, width, dtype, g, scale=1.0, pad=0):
    """[n][width], rows ``width + pad`` elements apart."""
    x = torch.empty((n, width + pad), device="cuda", dtype=torch.float32)
    x.normal_(0.0, scale, generator=g)
    return x.to(dtype)[:, :width]


def _inputs_la(c, g):
    lengths, rows = _lengths(c)
    S, H, K, dk, dv = c["sequences"], c["heads"], c["kv_heads"], c["key_width"], c["value_width"]
    dt = DTYPES[c["dtype"]]
    s = {"q": _normal(rows, H * dk, dt, g, pad=c["pad"]), "k": _normal(rows, K * dk, dt, g, pad=c["pad"]),
         "v": _normal(rows, K * dv, dt, g, pad=c["pad"])}
    # Heads remember from 8 tokens to 1,024, geometrically apart; a seed moves
    # all of them a little.
    at = torch.arange(H, device="cuda", dtype=torch.float64) / max(1, H - 1)
    move = torch.rand(1, device="cuda", generator=g, dtype=torch.float64)
    s["log_decay"] = torch.log1p(-2.0 ** (-3.0 - 7.0 * at - 0.5 * move)).float()
    s["s0"] = torch.empty((S, H, dk, dv), device="cuda").normal_(0.0, 1.0, generator=g)
    off = torch.tensor([0] + lengths, dtype=torch.int64).cumsum(0).to(torch.int32).cuda()
    s["offsets"] = off if c["ragged"] else None
    s["lengths"] = (off[1:] - off[:-1]).long()
    s["scale"] = 1.0 / math.sqrt(dk)
    s["o"] = torch.zeros((rows, H * dv), device="cuda", dtype=dt)
    s["sT"] = torch.zeros_like(s["s0"])
    if c["call"] == "train":
        s["do"] = _normal(rows, H * dv, dt, g)
        s["dsT"] = torch.empty_like(s["s0"]).normal_(0.0, 1.0, generator=g)
        s["ds0"] = torch.zeros_like(s["s0"])
        s["dq"], s["dk"], s["dv"] = (torch.zeros((rows, w), device="cuda", dtype=dt) for w in (H * dk, K * dk, K * dv))
    return s


def _inputs_norm(c, g):
    R, W, dt, sdt = c["rows"], c["width"], DTYPES[c["dtype"]], DTYPES[c["sum_dtype"]]
    s = {"x": _normal(R, W, dt, g), "residual": _normal(R, W, sdt, g, 2.0),
         "gain": torch.empty(W, device="cuda").normal_(1.0, 0.1, generator=g),
         "seed": int(torch.randint(0, 2 ** 62, (1,), device="cuda", generator=g)), "step": 7, "layer": 3,
         "total": torch.zeros((R, W), device="cuda", dtype=sdt)}
    if c["call"] == "codes":
        s["y"] = torch.zeros((R, W), device="cuda", dtype=torch.float8_e4m3fn)
        s["scale"] = torch.zeros(R, device="cuda")
    else:
        s["y"] = torch.zeros((R, W), device="cuda", dtype=dt)
    if c["call"] == "train":
        s["dy"], s["dtotal"] = _normal(R, W, dt, g), _normal(R, W, sdt, g)
        s["dresidual"] = torch.zeros((R, W), device="cuda", dtype=sdt)
        s["dx"] = torch.zeros((R, W), device="cuda", dtype=dt)
        s["dgain"] = torch.zeros(W, device="cuda")
    return s


def _inputs_drop(c, g):
    R, W, dt = c["rows"], c["width"], DTYPES[c["dtype"]]
    return {"x": _normal(R, W, dt, g), "residual": _normal(R, W, dt, g, 2.0) if c["residual"] else None,
            "y": torch.zeros((R, W), device="cuda", dtype=dt),
            "seed": int(torch.randint(0, 2 ** 62, (1,), device="cuda", generator=g)), "step": 12, "layer": 1}


def _inputs_sample(c, g):
    R, V, dt = c["rows"], c["vocab"], DTYPES[c["dtype"]]

    def between(lo, hi):
        return lo + (hi - lo) * torch.rand(R, device="cuda", generator=g)

    s = {"logits": _normal(R, V, dt, g, 2.5, c["pad"]), "u": torch.rand(R, device="cuda", generator=g),
         "temperature": between(0.6, 1.3), "tokens": torch.zeros(R, device="cuda", dtype=torch.int32),
         "logprob": torch.zeros(R, device="cuda")}
    s["temperature"][::8] = 0.0             # some callers want the likeliest token
    s["top_k"] = torch.exp(between(0.0, math.log(V))).to(torch.int32) if c["top_k"] else None
    s["top_p"] = between(0.5, 1.0) if c["top_p"] else None
    s["min_p"] = between(0.0, 0.1) if c["min_p"] else None
    return s


INPUTS = {"la": _inputs_la, "norm": _inputs_norm, "drop": _inputs_drop, "sample": _inputs_sample}


def _inputs(c, seed):
    return INPUTS[c["op"]](c, _generator(seed))


def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    s["case"] = c
    if own:                                 # the plan and its workspace, which a program makes once
        from paper_2609_37899_amd import soma
        dt = DTYPES[c["dtype"]]
        if c["op"] == "la":
            s["plan"] = soma.LinearAttention(s["q"].shape[0], c["sequences"], c["heads"], c["key_width"], c["value_width"],
                                             dt, kv_heads=c["kv_heads"], scale=s["scale"])
        elif c["op"] == "norm":
            s["plan"] = soma.RmsNorm(c["rows"], c["width"], dt, DTYPES[c["sum_dtype"]], eps=EPS, drop=c["drop"])
        elif c["op"] == "drop":
            s["plan"] = soma.Dropout(c["rows"], c["width"], dt, c["drop"])
        else:
            s["plan"] = soma.Sampler(c["rows"], c["vocab"], dt)
    return s


def run(state):
    s = state
    return {"la": _run_la, "norm": _run_norm, "drop": _run_drop, "sample": _run_sample}[s["case"]["op"]](s, s["case"])


# --------------------------------------------------------------------------
# Linear attention:  S_t = a S_{t-1} + k_t v_t^T,  o_t = scale q_t^T S_t

def _rows_of(s, lengths, T):
    """Row of every (sequence, time) and whether there is one."""
    t = torch.arange(T, device="cuda")[None, :]
    first = torch.cat([lengths.new_zeros(1), lengths.cumsum(0)[:-1]])[:, None]
    there = t < lengths[:, None]
    return torch.where(there, first + t, 0), there


def _heads_of(x, at, there, heads, of):
    """[S][heads][T][width] in 32 bits from rows of ``of`` heads, each of which several may share; zeros where there is no
    row."""
    S, T = at.shape
    y = x[at].float().view(S, T, of, -1) * there[:, :, None, None]
    return y.repeat_interleave(heads // of, dim=2).transpose(1, 2).contiguous()


def _decays(log_decay, n):
    """a^m for m = 0 .. n, [heads][n + 1]."""
    return torch.exp(log_decay[:, None] * torch.arange(n + 1, device="cuda", dtype=torch.float32))


def _within(pw, n):
    """a^(i - j) for j <= i, else 0: [heads][n][n]."""
    i = torch.arange(n, device="cuda")
    d = i[:, None] - i[None, :]
    return torch.where(d >= 0, pw[:, d.clamp(min=0)], 0.0)


def _remaining(lengths, at, n):
    """Rows that each sequence has in a chunk of n rows from time ``at`` on, [S]."""
    return (lengths - at).clamp(0, n)


def _plain_forward(q, k, v, s0, log_decay, lengths, scale):
    S, H, T, _ = q.shape
    pw = _decays(log_decay, CHUNK)
    heads = torch.arange(H, device="cuda")[None, :]
    out, state = [], s0.clone()
    for at in range(0, T, CHUNK):
        a, b, c = (x[:, :, at:at + CHUNK] for x in (q, k, v))
        n = a.shape[2]
        m = _remaining(lengths, at, n)
        A = (a @ b.transpose(2, 3)) * _within(pw, n)
        out.append(scale * (A @ c + pw[:, 1:n + 1, None] * (a @ state)))
        # rows of a chunk are as far from its end as the sequence has rows left
        left = m[:, None] - 1 - torch.arange(n, device="cuda")[None, :]
        w = torch.where((left >= 0)[:, None, :], pw[:, left.clamp(min=0)].transpose(0, 1), 0.0)
        state = pw[heads, m[:, None]][:, :, None, None] * state + (b * w[..., None]).transpose(2, 3) @ c
    return torch.cat(out, 2), state


def _plain_backward(q, k, v, do, s0, dsT, log_decay, lengths, scale):
    S, H, T, _ = q.shape
    pw = _decays(log_decay, CHUNK)
    heads = torch.arange(H, device="cuda")[None, :]
    dq, dk, dv, state = [], [], [], s0.clone()
    for at in range(0, T, CHUNK):           # states from the front
        b, c, d = (x[:, :, at:at + CHUNK] for x in (k, v, do))
        n = b.shape[2]
        m = _remaining(lengths, at, n)
        dA = (d @ c.transpose(2, 3)) * _within(pw, n)
        dq.append(scale * (dA @ b + pw[:, 1:n + 1, None] * (d @ state.transpose(2, 3))))
        left = m[:, None] - 1 - torch.arange(n, device="cuda")[None, :]
        w = torch.where((left >= 0)[:, None, :], pw[:, left.clamp(min=0)].transpose(0, 1), 0.0)
        state = pw[heads, m[:, None]][:, :, None, None] * state + (b * w[..., None]).transpose(2, 3) @ c
    back = dsT.clone()                      # the gradient of the state behind a chunk
    for at in range((T - 1) // CHUNK * CHUNK, -1, -CHUNK):
        a, b, c, d = (x[:, :, at:at + CHUNK] for x in (q, k, v, do))
        n = a.shape[2]
        m = _remaining(lengths, at, n)
        D = _within(pw, n)
        A, dA = (a @ b.transpose(2, 3)) * D, (d @ c.transpose(2, 3)) * D
        left = m[:, None] - 1 - torch.arange(n, device="cuda")[None, :]
        w = torch.where((left >= 0)[:, None, :], pw[:, left.clamp(min=0)].transpose(0, 1), 0.0)[..., None]
        dk.append(scale * (dA.transpose(2, 3) @ a) + w * (c @ back.transpose(2, 3)))
        dv.append(scale * (A.transpose(2, 3) @ d) + w * (b @ back))
        back = pw[heads, m[:, None]][:, :, None, None] * back + scale * ((a * pw[:, 1:n + 1, None]).transpose(2, 3) @ d)
    return torch.cat(dq, 2), torch.cat(dk[::-1], 2), torch.cat(dv[::-1], 2), back


def _to_rows(x, at, there, of, rows, dtype):
    """Rows again, the gradients of heads that share one summed."""
    S, H, T, w = x.shape
    x = x.transpose(1, 2).reshape(S, T, of, H // of, w).sum(3).reshape(S, T, of * w)
    out = torch.zeros((rows, of * w), device="cuda", dtype=dtype)
    out[at[there]] = x[there].to(dtype)
    return out


def _run_la(s, c):
    if own:
        plan = s["plan"]
        if c["call"] == "step":
            plan.step(s["q"], s["k"], s["v"], s["log_decay"], s["s0"], s["sT"], s["o"])
            return {"o": s["o"], "sT": s["sT"]}
        plan.forward(s["q"], s["k"], s["v"], s["log_decay"], s["o"], s["s0"], s["sT"], s["offsets"])
        if c["call"] == "forward":
            return {"o": s["o"], "sT": s["sT"]}
        plan.backward(s["q"], s["k"], s["v"], s["log_decay"], s["do"], s["dq"], s["dk"], s["dv"], s["s0"], s["dsT"],
                      s["ds0"], s["offsets"])
        return {n: s[n] for n in ("o", "sT", "dq", "dk", "dv", "ds0")}
    H, K, dt, rows = c["heads"], c["kv_heads"], DTYPES[c["dtype"]], s["q"].shape[0]
    at, there = _rows_of(s, s["lengths"], max(_lengths(c)[0]))
    q, k, v = (_heads_of(s[n], at, there, H, of) for n, of in (("q", H), ("k", K), ("v", K)))
    o, sT = _plain_forward(q, k, v, s["s0"], s["log_decay"], s["lengths"], s["scale"])
    out = {"o": _to_rows(o, at, there, H, rows, dt), "sT": sT}
    if c["call"] == "train":
        do = _heads_of(s["do"], at, there, H, H)
        dq, dk, dv, ds0 = _plain_backward(q, k, v, do, s["s0"], s["dsT"], s["log_decay"], s["lengths"], s["scale"])
        out.update(dq=_to_rows(dq, at, there, H, rows, dt), dk=_to_rows(dk, at, there, K, rows, dt),
                   dv=_to_rows(dv, at, there, K, rows, dt), ds0=ds0)
    return out


def _exact_la(s, c):
    """Every pair of rows of a sequence and head."""
    lengths, rows = _lengths(c)
    H, K, dk, dv = c["heads"], c["kv_heads"], c["key_width"], c["value_width"]
    if sum(t * t for t in lengths) * H * (dk + dv) * (3 if c["call"] == "train" else 1) > 4e12:
        return None
    f = torch.float64
    l = s["log_decay"].double()
    out = {"o": torch.zeros((rows, H, dv), dtype=f, device="cuda"), "sT": s["s0"].double().clone()}
    train = c["call"] == "train"
    if train:
        out.update(dq=torch.zeros((rows, H, dk), dtype=f, device="cuda"), dk=torch.zeros((rows, K, dk), dtype=f, device="cuda"),
                   dv=torch.zeros((rows, K, dv), dtype=f, device="cuda"), ds0=s["dsT"].double().clone())
    first = 0
    for n, T in enumerate(lengths):
        if T == 0:
            continue
        at = slice(first, first + T)
        first += T
        t = torch.arange(T, device="cuda", dtype=f)
        apart = t[:, None] - t[None, :]
        for h in range(H):
            j = h * K // H
            q, k, v = (s[x][at, i * w:(i + 1) * w].double() for x, i, w in (("q", h, dk), ("k", j, dk), ("v", j, dv)))
            s0 = s["s0"][n, h].double()
            D = torch.where(apart >= 0, torch.exp(l[h] * apart.clamp(min=0)), 0.0) * s["scale"]
            front = torch.exp(l[h] * (t + 1))[:, None] * s["scale"]      # what a row sees of s0
            tail = torch.exp(l[h] * (T - 1 - t))[:, None]                # what is left of a row in sT
            A = (q @ k.t().contiguous()) * D
            out["o"][at, h] = A @ v + front * (q @ s0)
            out["sT"][n, h] = torch.exp(l[h] * T) * s0 + (k * tail).t().contiguous() @ v
            if not train:
                continue
            do, dsT = s["do"][at, h * dv:(h + 1) * dv].double(), s["dsT"][n, h].double()
            dA = (do @ v.t().contiguous()) * D
            out["dq"][at, h] = dA @ k + front * (do @ s0.t().contiguous())
            out["dk"][at, j] += dA.t().contiguous() @ q + tail * (v @ dsT.t().contiguous())
            out["dv"][at, j] += A.t().contiguous() @ do + tail * (k @ dsT)
            out["ds0"][n, h] = torch.exp(l[h] * T) * dsT + (q * front).t().contiguous() @ do
    return {n: x if n in ("sT", "ds0") else x.reshape(rows, -1) for n, x in out.items()}


# --------------------------------------------------------------------------
# Which elements are kept: 16 bits of Philox4x32-10 each, eight elements a block
# with key (lo32(seed), hi32(seed) ^ hi32(step)) and counter (lo32(b), layer,
# lo32(step), hi32(b)); element i's are half i % 2 of word i / 2 % 4 of block i / 8.

MASK = 0xFFFFFFFF


def _times(m, x):
    """Both halves of a 32-bit product, in 64-bit integers that wrap."""
    p = m * x
    return (p >> 32) & MASK, p & MASK


def _fields(n, seed, step, layer):
    """[n] fields of 16 bits."""
    b = torch.arange((n + 7) // 8, device="cuda", dtype=torch.int64)
    x = [b & MASK, torch.full_like(b, layer), torch.full_like(b, step & MASK), b >> 32]
    k0, k1 = seed & MASK, (seed >> 32) ^ (step >> 32)
    for r in range(10):
        h0, l0 = _times(0xD2511F53, x[0])
        h1, l1 = _times(0xCD9E8D57, x[2])
        x = [h1 ^ x[1] ^ ((k0 + r * 0x9E3779B9) & MASK), l1, h0 ^ x[3] ^ ((k1 + r * 0xBB67AE85) & MASK), l0]
    words = torch.stack(x, 1)
    return torch.stack([words & 0xFFFF, words >> 16], 2).view(-1)[:n]


def _kept(s, c):
    """The factor of every element: 0, or 1 over the share that is kept."""
    cut = round(c["drop"] * 65536)
    n = c["rows"] * c["width"]
    keep = _fields(n, s["seed"], s["step"], s["layer"]) >= cut
    return torch.where(keep, 65536.0 / (65536 - cut), 0.0).view(c["rows"], c["width"])


def _kept_exact(s, c):
    """The same on the host, from products of 64-bit unsigned integers."""
    cut, n = round(c["drop"] * 65536), c["rows"] * c["width"]
    b = np.arange(-(-n // 8), dtype=np.uint64)
    u = np.uint64
    w0, w1, w2, w3 = b & u(MASK), np.full_like(b, s["layer"]), np.full_like(b, s["step"] & MASK), b >> u(32)
    k0, k1 = s["seed"] % 2 ** 32, (s["seed"] // 2 ** 32) ^ (s["step"] // 2 ** 32)
    for _ in range(10):
        a, d = w0 * u(0xD2511F53), w2 * u(0xCD9E8D57)
        w0, w1, w2, w3 = (d >> u(32)) ^ w1 ^ u(k0), d & u(MASK), (a >> u(32)) ^ w3 ^ u(k1), a & u(MASK)
        k0, k1 = (k0 + 0x9E3779B9) % 2 ** 32, (k1 + 0xBB67AE85) % 2 ** 32
    out = np.empty((b.size, 8), dtype=np.float64)
    for i, w in enumerate((w0, w1, w2, w3)):
        out[:, 2 * i] = (w % u(65536)) >= u(cut)
        out[:, 2 * i + 1] = (w // u(65536)) >= u(cut)
    keep = torch.from_numpy(out.reshape(-1)[:n]).cuda().view(c["rows"], c["width"])
    return keep / (1 - cut / 65536)


# --------------------------------------------------------------------------
# Norm:  total = residual + drop(x),  y = gain total / sqrt(mean(total^2) + eps)

def _run_norm(s, c):
    if own:
        plan, where = s["plan"], (s["seed"], s["step"], s["layer"])
        if c["call"] == "codes":
            plan.forward(s["x"], s["gain"], s["y"], s["residual"], s["total"], s["scale"], *where)
            return {"total": s["total"], "y": s["y"], "scale": s["scale"]}
        plan.forward(s["x"], s["gain"], s["y"], s["residual"], s["total"], None, *where)
        if c["call"] == "forward":
            return {"total": s["total"], "y": s["y"]}
        plan.backward(s["total"], s["gain"], s["dy"], s["dtotal"], s["dresidual"], s["dx"], s["dgain"], *where)
        return {n: s[n] for n in ("total", "y", "dresidual", "dx", "dgain")}
    factor = _kept(s, c) if c["drop"] else 1.0
    t = s["residual"].float() + factor * s["x"].float()
    y = t * torch.rsqrt((t * t).mean(1, keepdim=True) + EPS) * s["gain"]
    total = t.to(s["total"].dtype)
    if c["call"] == "codes":
        top = y.abs().amax(1, keepdim=True)
        codes = y * torch.where(top > 0, 448.0 / top, 0.0)
        return {"total": total, "y": codes.to(torch.float8_e4m3fn), "scale": top[:, 0] * (1.0 / 448.0)}
    out = {"total": total, "y": y.to(s["y"].dtype)}
    if c["call"] == "forward":
        return out
    # The backward pass starts from the sum as it is kept.
    t, dy = total.float(), s["dy"].float()
    inv = torch.rsqrt((t * t).mean(1, keepdim=True) + EPS)
    n, h = t * inv, dy * s["gain"]
    dt = s["dtotal"].float() + inv * (h - n * (h * n).mean(1, keepdim=True))
    return dict(out, dresidual=dt.to(s["dresidual"].dtype), dx=(dt * factor).to(s["dx"].dtype), dgain=(dy * n).sum(0))


def _exact_norm(s, c):
    factor = _kept_exact(s, c) if c["drop"] else 1.0
    t = s["residual"].double() + factor * s["x"].double()
    g = s["gain"].double()
    y = g * t / (t.square().mean(1, keepdim=True) + EPS).sqrt()
    if c["call"] == "codes":                # a code has no value in 64 bits, its row's scale has
        return {"total": t, "y": None, "scale": y.abs().amax(1) / 448}
    out = {"total": t, "y": y}
    if c["call"] == "forward":
        return out
    t = t.to(s["total"].dtype).double()
    r = (t.square().mean(1, keepdim=True) + EPS).sqrt()
    h = s["dy"].double() * g
    dt = s["dtotal"].double() + h / r - t * (h * t).mean(1, keepdim=True) / r ** 3
    return dict(out, dresidual=dt, dx=dt * factor, dgain=(s["dy"].double() * t / r).sum(0))


# --------------------------------------------------------------------------
# Dropout

def _run_drop(s, c):
    if own:
        s["plan"].forward(s["x"], s["y"], s["residual"], s["seed"], s["step"], s["layer"])
        return {"y": s["y"]}
    y = _kept(s, c) * s["x"].float()
    if c["residual"]:
        y = s["residual"].float() + y
    return {"y": y.to(s["y"].dtype)}


def _exact_drop(s, c):
    y = _kept_exact(s, c) * s["x"].double()
    return {"y": y + s["residual"].double() if c["residual"] else y}


# --------------------------------------------------------------------------
# The next token.  Tokens are ranked by their logits, the lower index first among
# equals; top-k keeps the first k, top-p the shortest run of those whose share of
# their probability reaches p, min-p what has at least that share of the
# likeliest one's.  Of what is left, in the order of the indices, the first whose
# cumulative probability is over u.  No temperature: the first of the ranking.

def _run_sample(s, c):
    if own:
        s["plan"].sample(s["logits"], s["u"], s["tokens"], s["logprob"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
        return {"tokens": s["tokens"], "logprob": s["logprob"]}
    x = s["logits"].float()
    R, V = x.shape
    ranked, index = torch.sort(x, dim=1, descending=True, stable=True)
    t = s["temperature"].double()[:, None]
    greedy = t <= 0
    # sums that decide between neighbours: 64 bits
    w = torch.exp((ranked - ranked[:, :1]).double() / torch.where(greedy, 1.0, t))
    rank = torch.arange(V, device="cuda")[None, :]
    keep = torch.where(greedy, rank < 1, True)
    if c["top_k"]:
        keep = keep & (rank < s["top_k"][:, None].long())
    if c["top_p"]:
        kept = w * keep
        before = kept.cumsum(1) - kept
        keep = keep & ((before < s["top_p"].double()[:, None] * kept.sum(1, keepdim=True)) | (rank < 1))
    if c["min_p"]:
        keep = keep & (w >= s["min_p"].double()[:, None])
    w = torch.zeros_like(w).scatter_(1, index, w * keep)
    cumulative = w.cumsum(1)
    whole = cumulative[:, -1:]
    token = (cumulative <= s["u"].double()[:, None] * whole).sum(1).clamp(max=V - 1)
    share = w.gather(1, token[:, None]) / whole
    return {"tokens": token.to(torch.int32), "logprob": torch.log(share)[:, 0].float()}


def _exact_sample(s, c):
    """Row by row on the host."""
    x = s["logits"].float().cpu().numpy().astype(np.float64)
    u, t = (s[n].cpu().numpy().astype(np.float64) for n in ("u", "temperature"))
    k, p, m = (s[n].cpu().numpy() if s[n] is not None else None for n in ("top_k", "top_p", "min_p"))
    tokens, logs = [], []
    for r, row in enumerate(x):
        order = np.argsort(-row, kind="stable")
        if t[r] == 0:
            tokens.append(int(order[0]))
            logs.append(0.0)
            continue
        w = np.exp((row - row.max()) / t[r])
        if k is not None:
            order = order[:k[r]]
        if p is not None:
            run = np.cumsum(w[order])
            order = order[:max(1, int(np.searchsorted(run, float(p[r]) * run[-1], side="left")) + 1)]
        if m is not None:
            order = order[w[order] >= float(m[r])]
        order = np.sort(order)
        run = np.cumsum(w[order])
        at = min(int(np.searchsorted(run, u[r] * run[-1], side="right")), order.size - 1)
        tokens.append(int(order[at]))
        logs.append(float(np.log(w[order[at]] / run[-1])))
    return {"tokens": torch.tensor(tokens, dtype=torch.int32, device="cuda"),
            "logprob": torch.tensor(logs, dtype=torch.float64, device="cuda")}


def exact(case, seed):
    s = _inputs(case, seed)
    return {"la": _exact_la, "norm": _exact_norm, "drop": _exact_drop, "sample": _exact_sample}[case["op"]](s, case)
