"""The draw of the next token against its definition in 64 bits, row by row."""
import numpy as np
import pytest

import block_reference as ref
from gpu_common import require_gpu
from paper_2609_37899_amd import soma

pytestmark = pytest.mark.gpu


def draw(torch, logits, u, plan=None, **settings):
    """tokens and logprob of float32 or bfloat16 logits on the GPU."""
    n, V = logits.shape
    plan = plan or soma.Sampler(n, V, logits.dtype)
    tokens, logprob = torch.full((n,), 77777777, dtype=torch.int32, device="cuda"), torch.full((n,), 7.0, device="cuda")
    dev = {k: torch.from_numpy(np.asarray(v, dtype=np.int32 if k == "top_k" else np.float32)).cuda() for k, v in settings.items()}
    plan.sample(logits, torch.from_numpy(u.astype(np.float32)).cuda(), tokens, logprob, **dev)
    torch.cuda.synchronize()
    return tokens.cpu().numpy(), logprob.double().cpu().numpy()


def check(torch, logits, u, most_near=0, **settings):
    """Tokens are the reference's, but where u or a filter's border is nearer to a cumulative weight than weights that are
    multiples of 2^-s can tell: half of one for each token, 2^-62 ceil2(vocab) vocab / 2, on either side."""
    tokens, logprob = draw(torch, logits, u, **settings)
    V = logits.shape[1]
    unit = 2.0 ** -(62 - int(np.ceil(np.log2(V))))
    l = logits.double().cpu().numpy()
    u = u.astype(np.float32).astype(np.float64)
    near = 0
    for r in range(l.shape[0]):
        kw = {k: np.float32(v[r]) if k != "top_k" else int(v[r]) for k, v in settings.items()}
        token, share, gap = ref.sample(l[r], u[r], **kw)
        if gap <= V * unit + 1e-13:
            near += 1
            continue
        assert tokens[r] == token, (r, kw, gap)
        # its weight in fp64, the sum off by V units of a sum of 1 or more, the logarithm's rounding
        assert logprob[r] == share or abs(logprob[r] - share) <= V * unit + 2 * ref.U * abs(share) + 1e-12, (r, logprob[r], share)
    assert near <= most_near, near


def make(torch, rows, vocab, dtype, seed=0, spread=2.5):
    g = np.random.default_rng(seed)
    logits = torch.from_numpy((spread * g.standard_normal((rows, vocab))).astype(np.float32)).to(getattr(torch, dtype)).cuda()
    return logits, g.random(rows), g


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocab", [1, 2, 5, 64, 256, 1000, 4096, 4097, 10007, 50257])
@pytest.mark.parametrize("filters", ["", "k", "p", "m", "kp", "kpm"])
def test_matches_reference(dtype, vocab, filters):
    torch = require_gpu()
    rows = 40 if vocab <= 10007 else 12
    logits, u, g = make(torch, rows, vocab, dtype)
    kw = {"temperature": np.where(np.arange(rows) % 7 == 3, 0.0, g.uniform(0.3, 2.0, rows))}
    if "k" in filters:
        kw["top_k"] = np.exp(g.uniform(0, np.log(vocab + 1), rows)).astype(np.int32)
    if "p" in filters:
        kw["top_p"] = g.uniform(0.05, 1.0, rows)
    if "m" in filters:
        kw["min_p"] = g.uniform(0.0, 0.3, rows)
    check(torch, logits, u, **kw)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocab", [100, 256, 257, 1000, 5000])
def test_equal_logits(dtype, vocab):
    """Ties go to the lowest index: rows of one value, of two, and of small whole numbers."""
    torch = require_gpu()
    g = np.random.default_rng(3)
    x = np.stack([np.zeros(vocab), np.where(np.arange(vocab) % 2, 1.0, -1.0)] + [g.integers(-3, 4, vocab) for _ in range(30)])
    logits = torch.from_numpy(x.astype(np.float32)).to(getattr(torch, dtype)).cuda()
    logits[0, ::3] = -0.0
    n = len(x)
    u = g.random(n)
    for kw in ({}, {"top_k": np.full(n, vocab // 3)}, {"top_p": np.full(n, 0.37)}, {"top_k": np.full(n, 7), "top_p": np.full(n, 0.61)},
               {"temperature": np.zeros(n)}):
        check(torch, logits, u, **kw)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_settings_at_the_ends_of_their_ranges(dtype):
    torch = require_gpu()
    inf, nan = np.inf, np.nan
    logits, u, g = make(torch, 14, 3000, dtype, seed=5)
    check(torch, logits, u, temperature=np.array([0.0, -1.0, nan, 1e-3, 1e-30, 1e30, inf, 1.0, 50.0, 1e-44, 0.1, 2.0, 3.0, 4.0]))
    check(torch, logits, u, top_k=np.array([0, -5, 1, 2, 2999, 3000, 3001, 2**31 - 1, -2**31, 3, 4, 5, 6, 7]))
    check(torch, logits, u, top_p=np.array([0.0, -1.0, nan, 1.0, 2.0, inf, 1e-30, 0.999999, 0.5, 1e-3, 0.1, 0.2, 0.3, 0.4]))
    check(torch, logits, u, min_p=np.array([0.0, -1.0, nan, 1.0, 2.0, inf, 1e-30, 0.999999, 0.5, 1e-3, 0.1, 0.2, 0.3, 0.4]))
    # u outside [0, 1): the first or the last of those left
    tokens, _ = draw(torch, logits[:4], np.array([-1.0, nan, 1.0, inf]), top_k=[5] * 4)
    for r in range(4):
        five = np.sort(np.argsort(-logits[r].double().cpu().numpy(), kind="stable")[:5])
        assert tokens[r] == five[0 if r < 2 else 4]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocab", [50, 6000])
def test_masked_logits(dtype, vocab):
    """Rows that a mask leaves nothing of, one token, a few; masks of -infinity, of NaN and of the type's lowest value;
    infinities."""
    torch = require_gpu()
    logits, u, g = make(torch, 9, vocab, dtype, seed=6)
    low = torch.finfo(logits.dtype).min
    logits[0] = float("-inf")
    logits[1] = float("nan")
    logits[2] = low
    logits[3], logits[3, 17] = float("-inf"), -5.0
    logits[4], logits[4, [3, 40, 41]] = low, torch.tensor([1.0, 2.0, 3.0], dtype=logits.dtype, device="cuda")
    logits[5, [9, 30]] = float("inf")
    logits[6, ::2] = float("nan")
    logits[7, 1::2] = float("-inf")
    logits[8] = torch.finfo(logits.dtype).max
    for kw in ({}, {"top_k": np.full(9, 10)}, {"top_p": np.full(9, 0.6)}, {"temperature": np.full(9, 0.2), "min_p": np.full(9, 0.1)},
               {"temperature": np.zeros(9)}, {"temperature": np.full(9, np.inf)}):
        check(torch, logits, u, **kw)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("pad,shift", [(1, 0), (3, 1), (8, 8)])
def test_strides_and_alignment(dtype, pad, shift):
    torch = require_gpu()
    logits, u, g = make(torch, 20, 5003, dtype, seed=7)
    flat = torch.full((20 * (5003 + pad) + shift + 8,), float("inf"), dtype=logits.dtype, device="cuda")
    view = flat[shift:shift + 20 * (5003 + pad)].view(20, 5003 + pad)[:, :5003]
    view.copy_(logits)
    for kw in ({}, {"top_k": np.full(20, 50), "top_p": np.full(20, 0.8)}):
        a, b = draw(torch, logits, u, **kw), draw(torch, view, u, **kw)
        assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


@pytest.mark.parametrize("dtype,vocab", [("bfloat16", 56175), ("bfloat16", 70001), ("float32", 28090), ("float32", 131072)])
def test_rows_too_long_for_lds(dtype, vocab):
    """Both sides of the length that a row is held up to, and beyond; rows of any alignment."""
    torch = require_gpu()
    logits, u, g = make(torch, 6, vocab, dtype, seed=14)
    for V in (vocab, vocab - 11):
        kw = {"temperature": g.uniform(0.5, 1.5, 6), "top_k": np.exp(g.uniform(0, np.log(V), 6)).astype(np.int32)}
        check(torch, logits[:, :V], u, **kw)
        check(torch, logits[:, vocab - V:], u, top_p=g.uniform(0.3, 1.0, 6), **kw)
        check(torch, logits[:, :V], u, most_near=1)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("spread", [1e-3, 0.05, 100.0])
def test_narrow_and_wide_logits(dtype, spread):
    """Bins of many equal logits, and logits so far apart that few count."""
    torch = require_gpu()
    logits, u, g = make(torch, 8, 20000, dtype, seed=15, spread=spread)
    logits[::2, 5] = 60.0                    # one far above the rest
    for kw in ({"top_k": np.array([1, 2, 17, 500, 3000, 9000, 19999, 20000])}, {"top_p": g.uniform(0.2, 1.0, 8)},
               {"top_k": np.full(8, 4000), "top_p": np.full(8, 0.7), "temperature": np.full(8, 1.7)}):
        check(torch, logits, u, **kw)


def test_shares():
    """Many draws of one row: every token's share within 6 deviations."""
    torch = require_gpu()
    n, V = 200000, 10
    logits, _, g = make(torch, 1, V, "float32", seed=8, spread=1.0)
    tokens, _ = draw(torch, logits.expand(n, V).contiguous(), g.random(n), temperature=np.full(n, 0.7), top_k=np.full(n, 6))
    l = logits[0].double().cpu().numpy() / np.float64(np.float32(0.7))
    w = np.where(np.argsort(np.argsort(-l)) < 6, np.exp(l), 0)
    p = w / w.sum()
    share = np.bincount(tokens, minlength=V) / n
    assert (np.abs(share - p) <= 6 * np.sqrt(p * (1 - p) / n)).all()


def test_largest_vocabulary_repeated_and_without_logprob():
    torch = require_gpu()
    logits, u, g = make(torch, 3, 2**20, "float32", seed=9)
    check(torch, logits, u, most_near=3, top_p=np.array([0.9, 0.5, 0.99]), temperature=np.full(3, 0.8))
    plan = soma.Sampler(3, 2**20, torch.float32)
    t = [torch.zeros(3, dtype=torch.int32, device="cuda") for _ in range(4)]
    for x in t:
        plan.sample(logits, torch.from_numpy(u.astype(np.float32)).cuda(), x)
    torch.cuda.synchronize()
    assert all(torch.equal(x, t[0]) for x in t)


def test_captured():
    """Replays see new logits and random numbers."""
    torch = require_gpu()
    logits, u, g = make(torch, 16, 5000, "bfloat16", seed=10)
    plan, other = soma.Sampler(16, 5000, torch.bfloat16), soma.Sampler(16, 5000, torch.bfloat16)
    ud, tokens = torch.from_numpy(u.astype(np.float32)).cuda(), torch.zeros(16, dtype=torch.int32, device="cuda")
    p = torch.full((16,), 0.9, device="cuda")
    plan.sample(logits, ud, tokens, top_p=p)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.sample(logits, ud, tokens, top_p=p)
    for seed in (11, 12, 13):
        new, u, _ = make(torch, 16, 5000, "bfloat16", seed=seed)
        logits.copy_(new)
        ud.copy_(torch.from_numpy(u.astype(np.float32)))
        graph.replay()
        want = torch.zeros_like(tokens)
        other.sample(new, ud, want, top_p=p)
        torch.cuda.synchronize()
        assert torch.equal(tokens, want)
