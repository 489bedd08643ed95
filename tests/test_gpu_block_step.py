"""A residual block's operators together, as a model uses them: a training step (norm, linear attention, dropout of the
branch, norm, cross entropy, AdamW) against 64 bits, and generation token by token against the whole prompt at once."""
import numpy as np
import pytest

import block_reference as ref
from gpu_common import require_gpu
from paper_2609_37899_amd import soma

pytestmark = pytest.mark.gpu

V, E, H, K, D, DV, P, EPS = 300, 40, 4, 2, 12, 10, 0.25, 1e-5
LENGTHS = [30, 0, 7, 90, 1]
SCALE = D ** -0.5


def weights(torch, seed=5):
    g = torch.Generator().manual_seed(seed)
    shapes = {"emb": (V, E), "qkv": (H * D + K * D + K * DV, E), "out": (E, H * DV), "head": (V, E), "g1": (E,), "g2": (E,)}
    return {n: torch.randn(s, generator=g) * 0.1 + 1 if n[0] == "g" else torch.randn(s, generator=g) * (1.0 if n == "emb" else 0.2)
            for n, s in shapes.items()}


def model64(torch, p, log_decay, ids, targets, w, factor):
    """The model in float64 on the CPU, with torch's derivatives."""
    p = {n: x.detach().double().cpu().requires_grad_() for n, x in p.items()}

    def norm(t, gain):
        return gain * t / torch.sqrt((t * t).mean(1, keepdim=True) + EPS)

    x = p["emb"][ids]
    qkv = norm(x, p["g1"]) @ p["qkv"].t()
    q, k, v = qkv.split([H * D, K * D, K * DV], dim=1)
    q, k, v = q.view(-1, H, D), k.view(-1, K, D).repeat_interleave(H // K, 1), v.view(-1, K, DV).repeat_interleave(H // K, 1)
    a, o, at = torch.exp(log_decay)[:, None, None], [], 0
    for n in LENGTHS:
        S = torch.zeros(H, D, DV, dtype=torch.float64)
        for t in range(at, at + n):
            S = a * S + k[t][:, :, None] * v[t][:, None, :]
            o.append(SCALE * (q[t][:, :, None] * S).sum(1).reshape(-1))
        at += n
    total = x + factor * (torch.stack(o) @ p["out"].t())
    logits = norm(total, p["g2"]) @ p["head"].t()
    loss = (torch.nn.functional.cross_entropy(logits, targets, reduction="none") * w).sum()
    loss.backward()
    return float(loss.detach()), {n: x.grad for n, x in p.items()}


@pytest.mark.parametrize("bits", [32, 8])
def test_training_steps(bits):
    """Three steps: losses and gradients against 64 bits from the weights that the GPU has then; the mask of each is its
    update's."""
    torch = require_gpu()
    rows, S = sum(LENGTHS), len(LENGTHS)
    p = {n: x.cuda() for n, x in weights(torch).items()}
    grads = {n: torch.zeros_like(x) for n, x in p.items()}
    g = torch.Generator().manual_seed(6)
    ids, targets = torch.randint(0, V, (rows,), generator=g), torch.randint(0, V, (rows,), generator=g)
    w = torch.full((rows,), 1.0 / rows)
    log_decay = torch.log1p(-2.0 ** -torch.linspace(1, 7, H))
    dev = {"ids": ids.cuda(), "targets": targets.to(torch.int32).cuda(), "w": w.cuda(), "l": log_decay.cuda(),
           "off": torch.tensor([0] + list(np.cumsum(LENGTHS)), dtype=torch.int32).cuda()}
    n1, n2 = soma.RmsNorm(rows, E, torch.float32, eps=EPS), soma.RmsNorm(rows, E, torch.float32, eps=EPS, drop=P)
    la = soma.LinearAttention(rows, S, H, D, DV, torch.float32, kv_heads=K)
    ce = soma.CrossEntropy(rows, V, E, torch.float32)
    names = sorted(p)
    opt = soma.AdamW([p[n] for n in names], [grads[n] for n in names], bits=bits, weight_decay=[0.0 if n[0] == "g" else 0.1 for n in names],
                     rounding="random" if bits == 8 else "nearest")

    def empty(*width):
        return torch.empty(rows, *width, device="cuda")

    y1, y2, total, dy2, dres, db, dx, o = empty(E), empty(E), empty(E), empty(E), empty(E), empty(E), empty(E), empty(H * DV)
    dq, dk, dv, loss, lse = empty(H * D), empty(K * D), empty(K * DV), empty(), empty()
    cut = [H * D, H * D + K * D]
    for t in range(1, 4):
        before = {n: x.clone() for n, x in p.items()}
        x = p["emb"][dev["ids"]]
        n1.forward(x, p["g1"], y1)
        qkv = y1 @ p["qkv"].t()
        q, k, v = qkv[:, :cut[0]], qkv[:, cut[0]:cut[1]], qkv[:, cut[1]:]
        la.forward(q, k, v, dev["l"], o, offsets=dev["off"])
        n2.forward(o @ p["out"].t(), p["g2"], y2, x, total, seed=9, step=t, layer=1)
        ce.loss(y2, p["head"], dev["targets"], loss, lse)
        ce.grad(y2, p["head"], dev["targets"], lse, dev["w"], dy2, grads["head"])
        n2.backward(total, p["g2"], dy2, None, dres, db, grads["g2"], seed=9, step=t, layer=1)
        torch.mm(db.t(), o, out=grads["out"])
        la.backward(q, k, v, dev["l"], db @ p["out"], dq, dk, dv, offsets=dev["off"])
        dqkv = torch.cat([dq, dk, dv], 1)
        torch.mm(dqkv.t(), y1, out=grads["qkv"])
        n1.backward(x, p["g1"], dqkv @ p["qkv"], dres, dx, None, grads["g1"])
        grads["emb"].zero_().index_add_(0, dev["ids"], dx)
        opt.step(t, 1e-2)
        torch.cuda.synchronize()
        factor = torch.from_numpy(ref.keep(rows, E, P, 9, t, 1))
        want_loss, want = model64(torch, before, log_decay.double(), ids, targets, w.double(), factor)
        assert abs(float((loss * dev["w"]).sum()) - want_loss) <= 1e-5 * abs(want_loss)
        for n in names:
            # sums of up to 128 rows and 300 outputs in fp32 through six operators, relative to the whole
            assert float((grads[n].double().cpu() - want[n]).norm() / want[n].norm()) <= 2e-5, n
            # AdamW's first updates move by about lr
            assert float((p[n] - before[n]).abs().max()) <= 0.05 and torch.isfinite(p[n]).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_generation_is_the_prompt_at_once(dtype):
    """Prompts in one call and the rest token by token give what all tokens in one call give; the sampler takes the
    likeliest token, or one whose share in what top-k leaves is not 0."""
    torch = require_gpu()
    S, T, more, dt = 6, 37, 4, getattr(torch, dtype)
    p = {n: x.cuda() for n, x in weights(torch, 7).items()}
    c = {n: p[n].to(dt) for n in ("qkv", "out", "head")}
    l = torch.log1p(-2.0 ** -torch.linspace(1, 7, H)).cuda()
    g = torch.Generator().manual_seed(8)
    ids = torch.randint(0, V, (S, T + more), generator=g).cuda()
    u = torch.rand(S, generator=g).cuda()

    def layer(x, attend):
        y, total = torch.empty_like(x, dtype=dt), torch.empty_like(x)
        norm = soma.RmsNorm(x.shape[0], E, dt, torch.float32, eps=EPS)
        norm.forward(x.to(dt), p["g1"], y)
        qkv = y @ c["qkv"].t()
        o = torch.empty(x.shape[0], H * DV, dtype=dt, device="cuda")
        attend(qkv[:, :H * D], qkv[:, H * D:H * D + K * D], qkv[:, H * D + K * D:], o)
        norm.forward(o @ c["out"].t(), p["g2"], y, x, total)
        return (y @ c["head"].t()).float()

    def prompt(n, sT):
        la = soma.LinearAttention(S * n, S, H, D, DV, dt, kv_heads=K, grad=False)
        return layer(p["emb"][ids[:, :n].reshape(-1)], lambda q, k, v, o: la.forward(q, k, v, l, o, None, sT))

    whole = prompt(T + more, None).view(S, T + more, V)
    state = torch.empty(S, H, D, DV, device="cuda")
    first = prompt(T, state).view(S, T, V)
    step = soma.LinearAttention(S, S, H, D, DV, dt, kv_heads=K, grad=False)
    parts = [first] + [layer(p["emb"][ids[:, t]], lambda q, k, v, o: step.step(q, k, v, l, state, state, o)).view(S, 1, V)
                       for t in range(T, T + more)]
    got = torch.cat(parts, 1)
    # two orders of sums; in bf16 o may land on the next value, half a unit of its last place either way, and so may what follows it
    assert float((got - whole).norm() / whole.norm()) <= (1e-5 if dtype == "float32" else 2.0 ** -6)
    logits = got[:, -1].contiguous()
    tokens, likely, logprob = (torch.empty(S, dtype=t, device="cuda") for t in (torch.int32, torch.int32, torch.float32))
    sampler = soma.Sampler(S, V, torch.float32)
    sampler.sample(logits, u, likely, temperature=torch.zeros(S, device="cuda"))
    sampler.sample(logits, u, tokens, logprob, top_k=torch.full((S,), 5, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(likely.long(), logits.argmax(1))
    best, at = logits.double().topk(5, dim=1)
    hit = at == tokens[:, None]
    assert hit.sum(1).eq(1).all()
    want = torch.log_softmax(best, 1)[hit]
    assert (logprob.double() - want).abs().max() <= 1e-6
