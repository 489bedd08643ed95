"""The gated linear recurrence against a 64-bit loop over time: widths, lengths, types, strides, initial and final
states, gradients, captured and repeated calls."""
import numpy as np
import pytest

import train_reference as ref
from gpu_common import require_gpu
from paper_2609_37899_amd import soma

pytestmark = pytest.mark.gpu

LENGTHS = {
    "one": [1], "empty": [0, 1, 0, 2, 0], "tile": [64], "around": [63, 65, 1, 64], "ragged": [200, 0, 7, 129, 0, 1, 90],
    "long": [2500], "long_pair": [1300, 0, 700], "many": [5] * 150, "all_empty": [0, 0],
}


def make(torch, dtype, width, lengths, behind=3, pad=0, seed=0):
    """Gates (in rows `pad` elements longer than needed), states and gradients, on the GPU and as float64."""
    g = np.random.default_rng(seed)
    dt = getattr(torch, dtype)
    rows = sum(lengths) + behind

    def both(x, t):
        y = torch.from_numpy(x.astype(np.float32)).to(t).cuda()
        return y, y.double().cpu().numpy()

    gates, gates64 = both(g.standard_normal((rows, 4 * width + pad)) * 1.5, dt)
    dh, dh64 = both(g.standard_normal((rows, width)), dt)
    c0, c064 = both(g.standard_normal((len(lengths), width)), torch.float32)
    dcT, dcT64 = both(g.standard_normal((len(lengths), width)), torch.float32)
    off = torch.tensor([0] + list(np.cumsum(lengths)), dtype=torch.int32).cuda()
    x = {"gates": gates[:, :4 * width], "dh": dh, "c0": c0, "dcT": dcT, "offsets": off}
    return x, ref.scan(gates64[:, :4 * width], lengths, c064, dh64, dcT64)


def run(torch, plan, x, dtype, stream=None, offsets=True):
    rows, S, H = x["gates"].shape[0], plan.sequences, plan.width
    dt = getattr(torch, dtype)
    y = {"h": torch.full((rows, H), 7.0, dtype=dt, device="cuda"), "cT": torch.full((S, H), 7.0, device="cuda"),
         "dgates": torch.full((rows, 4 * H), 7.0, dtype=dt, device="cuda"), "dc0": torch.full((S, H), 7.0, device="cuda"),
         "states": plan.new_states()}
    off = x["offsets"] if offsets else None
    plan.forward(x["gates"], y["h"], x["c0"], y["cT"], y["states"], off, stream=stream)
    plan.backward(x["gates"], y["states"], x["dh"], y["dgates"], x["c0"], x["dcT"], y["dc0"], off, stream=stream)
    return y


def check(y, want, dtype):
    for name in ("h", "cT", "dgates", "dc0"):
        got, exact = y[name].double().cpu().numpy(), want[name]
        step = ref.half_step(dtype if name in ("h", "dgates") else "float32")
        outside = np.isnan(exact)
        assert np.all(got[outside] == 7.0), f"{name}: rows behind the last sequence were written"
        # the type's smallest steps as well
        tol = want[name + "_err"] * (1 + step) + step * np.abs(np.nan_to_num(exact)) + 1e-37
        bad = ~(np.abs(got - exact) <= tol)            # NaN counts as wrong
        bad[outside] = False
        assert not bad.any(), (f"{name}: {bad.sum()} of {bad.size}, worst {np.nanmax(np.abs(got - exact) / tol):.2f} "
                               f"of the bound")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("lengths", sorted(LENGTHS))
@pytest.mark.parametrize("width", [1, 64, 130, 361])
def test_matches_reference(dtype, lengths, width):
    torch = require_gpu()
    x, want = make(torch, dtype, width, LENGTHS[lengths])
    plan = soma.GatedScan(x["gates"].shape[0], len(LENGTHS[lengths]), width, getattr(torch, dtype))
    y = run(torch, plan, x, dtype)
    torch.cuda.synchronize()
    check(y, want, dtype)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("pad,shift", [(1, 0), (2, 1), (64, 3)])
def test_strides_and_alignment(dtype, pad, shift):
    """Rows further apart than their length, starting at any element."""
    torch = require_gpu()
    lengths, H = [70, 3, 40], 66
    x, want = make(torch, dtype, H, lengths)
    rows = x["gates"].shape[0]
    wide = torch.full((rows * (4 * H + pad) + shift + 8,), float("nan"), dtype=getattr(torch, dtype), device="cuda")
    view = wide[shift:shift + rows * (4 * H + pad)].view(rows, 4 * H + pad)[:, :4 * H]
    view.copy_(x["gates"])
    x["gates"] = view
    y = run(torch, soma.GatedScan(rows, 3, H, getattr(torch, dtype)), x, dtype)
    torch.cuda.synchronize()
    check(y, want, dtype)


@pytest.mark.parametrize("sequences,length", [(1, 1), (4, 100), (600, 3), (1, 1500), (300, 1)])
def test_equal_lengths_without_offsets(sequences, length):
    """The same bits as with offsets."""
    torch = require_gpu()
    lengths = [length] * sequences
    x, want = make(torch, "float32", 65, lengths, behind=0)
    plan = soma.GatedScan(sequences * length, sequences, 65, torch.float32)
    y, z = run(torch, plan, x, "float32", offsets=False), run(torch, plan, x, "float32")
    torch.cuda.synchronize()
    check(y, want, "float32")
    for k in ("h", "cT", "dgates", "dc0"):
        assert torch.equal(y[k], z[k]), k


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("lengths", [[20000], [9000, 0, 11003]])
def test_repeated_calls_give_the_same_bits(dtype, lengths):
    """Few long sequences: what the blocks pass on does not depend on which of them is done first."""
    torch = require_gpu()
    x, want = make(torch, dtype, 96, lengths)
    plan = soma.GatedScan(x["gates"].shape[0], len(lengths), 96, getattr(torch, dtype))
    y = run(torch, plan, x, dtype)
    torch.cuda.synchronize()
    check(y, want, dtype)
    for _ in range(5):
        z = run(torch, plan, x, dtype)
        torch.cuda.synchronize()
        for k in ("h", "cT", "dgates", "dc0"):
            assert torch.equal(y[k], z[k]), k


@pytest.mark.parametrize("lengths", ["ragged", "long", "long_pair", "many"])
def test_states_in_place_and_left_out(lengths):
    """cT over c0 and dc0 over dcT; without them the states are zeros and nothing else changes."""
    torch = require_gpu()
    L, H = LENGTHS[lengths], 96
    x, want = make(torch, "float32", H, L)
    plan = soma.GatedScan(x["gates"].shape[0], len(L), H, torch.float32)
    y = run(torch, plan, x, "float32")
    c, d = x["c0"].clone(), x["dcT"].clone()
    h, dg = torch.full_like(y["h"], 7.0), torch.full_like(y["dgates"], 7.0)
    states = plan.new_states()
    plan.forward(x["gates"], h, c, c, states, x["offsets"])
    plan.backward(x["gates"], states, x["dh"], dg, x["c0"], d, d, x["offsets"])
    torch.cuda.synchronize()
    assert torch.equal(c, y["cT"]) and torch.equal(h, y["h"]) and torch.equal(dg, y["dgates"]) and torch.equal(d, y["dc0"])
    plan.forward(x["gates"], h, None, None, states, x["offsets"])
    plan.backward(x["gates"], states, x["dh"], dg, None, None, None, x["offsets"])
    zero = torch.zeros_like(x["c0"])
    z = run(torch, plan, dict(x, c0=zero, dcT=zero), "float32")
    torch.cuda.synchronize()
    assert torch.equal(h, z["h"]) and torch.equal(dg, z["dgates"])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("sequences,width", [(1, 1), (3, 361), (64, 512), (300, 40)])
def test_step(dtype, sequences, width):
    """One row for every sequence, the state in place."""
    torch = require_gpu()
    x, want = make(torch, dtype, width, [1] * sequences, behind=0, pad=5)
    plan = soma.GatedScan(sequences, sequences, width, getattr(torch, dtype))
    c, h = x["c0"].clone(), torch.empty((sequences, width), dtype=getattr(torch, dtype), device="cuda")
    plan.step(x["gates"], c, c, h)
    torch.cuda.synchronize()
    for got, name in ((h, "h"), (c, "cT")):
        step = ref.half_step(dtype if name == "h" else "float32")
        tol = want[name + "_err"] * (1 + step) + step * np.abs(want[name])
        assert np.all(np.abs(got.double().cpu().numpy() - want[name]) <= tol), name


@pytest.mark.parametrize("lengths", [[64, 30, 80], [100, 900, 500]])
def test_lowest_values_and_nan(lengths):
    """Gates of a type's lowest and largest value saturate; a sequence's NaN stays its own."""
    torch = require_gpu()
    H = 64
    x, _ = make(torch, "float32", H, lengths, behind=0)
    big = torch.finfo(torch.float32).max
    x["gates"][3, :] = -big
    x["gates"][5, :] = big
    x["gates"][lengths[0] + 2, :] = float("nan")          # the second sequence
    plan = soma.GatedScan(sum(lengths), 3, H, torch.float32)
    y = run(torch, plan, x, "float32")
    torch.cuda.synchronize()
    own = slice(lengths[0], lengths[0] + lengths[1])
    assert torch.isnan(y["h"][own][2:]).all() and torch.isnan(y["cT"][1]).all()
    for k in ("h", "dgates"):
        rest = torch.cat([y[k][:own.start], y[k][own.stop:]])
        assert torch.isfinite(rest).all(), k
    assert torch.isfinite(y["cT"][[0, 2]]).all() and torch.isfinite(y["dc0"][[0, 2]]).all()
    # everything shut: the state is gone and nothing comes in; everything open: c = 1 c + 1
    assert (y["h"][3] == 0).all() and (y["dgates"][3] == 0).all()
    x["gates"][lengths[0] + 2, :] = 0.0
    want = ref.scan(x["gates"].double().cpu().numpy(), lengths, *(x[k].double().cpu().numpy() for k in ("c0", "dh", "dcT")))
    y = run(torch, plan, x, "float32")
    torch.cuda.synchronize()
    far = np.abs(x["gates"].double().cpu().numpy()).max(1) > 1e30
    for name, rows in (("h", ~far), ("dgates", ~far)):      # the bounds' |x| terms do not apply to the saturated rows
        got, exact = y[name].double().cpu().numpy(), want[name]
        assert np.all(np.abs(got - exact)[rows] <= 1e-5 * (1 + np.abs(exact[rows]))), name


def test_gradient_against_differences():
    """dgates and dc0 against central differences of the loss sum(dh h) + sum(dcT cT), formed in 64 bits from the
    reference; a sample of coordinates, both ways of splitting the work."""
    torch = require_gpu()
    for lengths in ([9, 0, 20], [300]):
        H = 5
        x, _ = make(torch, "float32", H, lengths, behind=0)
        plan = soma.GatedScan(sum(lengths), len(lengths), H, torch.float32)
        y = run(torch, plan, x, "float32")
        torch.cuda.synchronize()
        gates, c0, dh, dcT = (x[k].double().cpu().numpy() for k in ("gates", "c0", "dh", "dcT"))

        def loss(gates, c0):
            o = ref.scan(gates, lengths, c0)
            return np.sum(dh * o["h"]) + np.sum(dcT * o["cT"])

        rng = np.random.default_rng(1)
        eps = 1e-5
        for _ in range(12):
            r, k = rng.integers(gates.shape[0]), rng.integers(4 * H)
            d = np.zeros_like(gates)
            d[r, k] = eps
            num = (loss(gates + d, c0) - loss(gates - d, c0)) / (2 * eps)
            # eps^2 of the third derivative and fp64 cancellation / eps
            assert abs(num - float(y["dgates"][r, k])) < 1e-5 * (1 + abs(num))
        d = np.zeros_like(c0)
        d[0, 2] = eps
        num = (loss(gates, c0 + d) - loss(gates, c0 - d)) / (2 * eps)
        assert abs(num - float(y["dc0"][0, 2])) < 1e-5 * (1 + abs(num))


@pytest.mark.parametrize("lengths", ["ragged", "long_pair"])
def test_captured_on_another_stream_and_repeated(lengths):
    """A captured forward and backward, replayed on changing inputs with eager work between, gives the eager bits."""
    torch = require_gpu()
    L, H = LENGTHS[lengths], 100
    x, _ = make(torch, "bfloat16", H, L)
    rows = x["gates"].shape[0]
    plan, eager = (soma.GatedScan(rows, len(L), H, torch.bfloat16) for _ in range(2))
    st = torch.cuda.Stream()
    y = run(torch, plan, x, "bfloat16", stream=st)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.forward(x["gates"], y["h"], x["c0"], y["cT"], y["states"], x["offsets"])
        plan.backward(x["gates"], y["states"], x["dh"], y["dgates"], x["c0"], x["dcT"], y["dc0"], x["offsets"])
    for k in range(3):
        z, _ = make(torch, "bfloat16", H, L, seed=10 + k)
        for name in ("gates", "dh", "c0", "dcT"):
            x[name].copy_(z[name])
        graph.replay()
        torch.cuda.synchronize()
        e = run(torch, eager, z, "bfloat16")
        torch.cuda.synchronize()
        for name in ("h", "cT", "dgates", "dc0"):
            assert torch.equal(y[name], e[name]), (k, name)


def test_offsets_that_break_the_rules_stay_inside():
    """Offsets beyond the rows or out of order: results are unspecified, memory outside the arrays is not touched
    (every row and offset is clamped); a guard of rows behind stays as it was."""
    torch = require_gpu()
    H, rows = 64, 200
    plan = soma.GatedScan(rows, 3, H, torch.float32)
    gates = torch.randn(rows, 4 * H, device="cuda")
    guard = torch.full((rows + 64, H), 7.0, device="cuda")
    dguard = torch.full((rows + 64, 4 * H), 7.0, device="cuda")
    for off in ([0, 50, 400, 1 << 30], [-5, 60, 20, 200], [0, 0, 0, -1]):
        o = torch.tensor(off, dtype=torch.int32, device="cuda")
        states = torch.zeros_like(plan.new_states())
        plan.forward(gates, guard[:rows], None, None, states, o)
        plan.backward(gates, states, guard[:rows].clone(), dguard[:rows], None, None, None, o)
        torch.cuda.synchronize()
        assert (guard[rows:] == 7).all() and (dguard[rows:] == 7).all()
