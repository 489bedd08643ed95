"""The gated linear recurrence at the ends of its ranges, against 64 bits."""
import numpy as np
import pytest

import train_reference as ref
from gpu_common import require_gpu
from paper_2609_37899_amd import soma
from test_gpu_scan import check, make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("offsets", [False, True])
def test_no_rows(dtype, offsets):
    """Every sequence keeps its state and passes its gradient on; nothing else is written."""
    torch = require_gpu()
    S, H, dt = 5, 70, getattr(torch, dtype)
    plan = soma.GatedScan(0, S, H, dt)
    gates, h = (torch.zeros((0, k * H), dtype=dt, device="cuda") for k in (4, 1))
    off = torch.zeros(S + 1, dtype=torch.int32, device="cuda") if offsets else None
    c0, dcT = torch.randn(S, H, device="cuda"), torch.randn(S, H, device="cuda")
    cT, dc0 = torch.zeros(S, H, device="cuda"), torch.zeros(S, H, device="cuda")
    states = plan.new_states()
    plan.forward(gates, h, c0, cT, states, off)
    plan.backward(gates, states, h, torch.zeros((0, 4 * H), dtype=dt, device="cuda"), c0, dcT, dc0, off)
    torch.cuda.synchronize()
    assert torch.equal(cT, c0) and torch.equal(dc0, dcT)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("lengths", [[70, 0, 33], [3000], [1, 1, 1]])
@pytest.mark.parametrize("scale", [0.3, 1e-3, 1e-5, 1e-7])
def test_small_states_keep_their_digits(dtype, lengths, scale):
    """Candidates and initial states near 0: h, and the gradients that are as small, to a relative bound.

    With the gates i, f, o within s(2) and everything of one sign nothing cancels but 1 - s(x).  In u = 2^-24: a sigmoid is
    off by 10 u (2 |x| + 6), a tanh by 12 u of its value (two for its polynomial; above 0.35, 4 u of 1), a product or sum
    of the recursion by 6 u.  So a term of a state is off by 30 u, and 16 u more for each row that it has passed, 8.4
    on average at the most (f <= 0.881): 165 u.  What the rows behind pass on: 150 u.  1 - s(x) >= 0.119 is off by 75 u.
    The widest, f's gradient, has a product of a state, such a factor, a sigmoid and what is passed on: 400 u.  For bf16
    gates a tanh is off by 2^-15, and every result has two at the most (the candidates', which the states hold, and
    their own)."""
    torch = require_gpu()
    rng = np.random.default_rng(11)
    S, H, n = len(lengths), 130, sum(lengths)
    dt = getattr(torch, dtype)

    def dev(x, t=torch.float32):
        return torch.from_numpy(x.astype(np.float32)).cuda().to(t)

    x = rng.uniform(-2, 2, (n, 4, H))
    x[:, 2] = scale * rng.uniform(0.1, 1, (n, H))
    gates = dev(x.reshape(n, 4 * H), dt)
    c0, dh, dcT = dev(scale * rng.uniform(0.1, 1, (S, H))), dev(rng.uniform(0.1, 1, (n, H)), dt), dev(rng.uniform(0.1, 1, (S, H)))
    off = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32, device="cuda")
    plan = soma.GatedScan(n, S, H, dt)
    h, cT, dg, dc0 = (torch.zeros(n, H, dtype=dt, device="cuda"), torch.zeros(S, H, device="cuda"),
                      torch.zeros(n, 4 * H, dtype=dt, device="cuda"), torch.zeros(S, H, device="cuda"))
    states = plan.new_states()
    plan.forward(gates, h, c0, cT, states, off)
    plan.backward(gates, states, dh, dg, c0, dcT, dc0, off)
    torch.cuda.synchronize()
    want = ref.scan(gates.double().cpu().numpy(), lengths, c0.double().cpu().numpy(), dh.double().cpu().numpy(),
                    dcT.double().cpu().numpy())
    got = {"h": h, "cT": cT, "dgates": dg, "dc0": dc0}
    if n == S:                                           # one row each: the step as well
        h1, c1 = torch.zeros_like(h), torch.zeros_like(cT)
        plan.step(gates, c0, c1, h1)
        torch.cuda.synchronize()
        got.update(h_step=h1, cT_step=c1)
    for name, y in got.items():
        exact = want[name.split("_")[0]]
        tol = 400 * ref.U + (2 * 2.0**-15 if dtype == "bfloat16" else 0)
        tol = tol * (1 + 2.0**-8) + (ref.half_step(dtype) if y.dtype != torch.float32 else 0)
        rel = np.abs(y.double().cpu().numpy() - exact) / np.abs(exact)
        assert rel.max() <= tol, (name, rel.max(), tol)


@pytest.mark.parametrize("behind", [0, 9])
def test_many_ragged_sequences_two_channels_a_lane(behind):
    """600 sequences in one launch: enough blocks for two bf16 channels a lane without pieces."""
    torch = require_gpu()
    H = 130
    lengths = [int(k) for k in np.random.default_rng(7).integers(0, 70, 600)]
    x, want = make(torch, "bfloat16", H, lengths, behind=behind)
    plan = soma.GatedScan(x["gates"].shape[0], len(lengths), H, torch.bfloat16)
    y = run(torch, plan, x, "bfloat16")
    torch.cuda.synchronize()
    check(y, want, "bfloat16")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("off", [[0, 500, 4000, 1 << 30], [-5, 600, 200, 2000], [0, 0, 0, -1], [1900, 100, 50, 2000],
                                 [0, 1500, 700, 1000]])
def test_offsets_that_break_the_rules_in_pieces_stay_inside(dtype, off):
    """Rows enough for pieces: both walks over a piece's sequences go on at every step whatever the offsets say, and rows
    behind the arrays stay as they were."""
    torch = require_gpu()
    H, rows, dt = 64, 2000, getattr(torch, dtype)
    plan = soma.GatedScan(rows, 3, H, dt)
    assert plan._bytes > 0                                # pieces
    gates = torch.randn(rows, 4 * H, device="cuda").to(dt)
    guard = torch.full((rows + 64, H), 7.0, device="cuda", dtype=dt)
    dguard = torch.full((rows + 64, 4 * H), 7.0, device="cuda", dtype=dt)
    o = torch.tensor(off, dtype=torch.int32, device="cuda")
    states = torch.zeros_like(plan.new_states())
    plan.forward(gates, guard[:rows], None, None, states, o)
    plan.backward(gates, states, guard[:rows].clone(), dguard[:rows], None, None, None, o)
    torch.cuda.synchronize()
    assert (guard[rows:] == 7).all() and (dguard[rows:] == 7).all()
