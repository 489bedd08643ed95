"""How many launches a call of linear attention enqueues: the nodes of a graph that captures it."""
import ctypes

import pytest

from gpu_common import require_gpu
from paper_2609_37899_amd import soma

pytestmark = pytest.mark.gpu


def nodes(torch, call):
    """Of a call on a captured stream."""
    hip = ctypes.CDLL(soma.LIB_PATH)           # and the runtime that it is linked to
    stream, graph, n = torch.cuda.Stream(), ctypes.c_void_p(), ctypes.c_size_t()
    torch.cuda.synchronize()
    assert hip.hipStreamBeginCapture(ctypes.c_void_p(stream.cuda_stream), 2) == 0
    try:
        call(stream)
    finally:
        assert hip.hipStreamEndCapture(ctypes.c_void_p(stream.cuda_stream), ctypes.byref(graph)) == 0
    assert hip.hipGraphGetNodes(graph, None, ctypes.byref(n)) == 0
    assert hip.hipGraphDestroy(graph) == 0
    return n.value


@pytest.mark.parametrize("sequences,heads,widths,launches", [
    (32, 8, (64, 64), 2), (64, 8, (64, 64), 2), (32, 8, (64, 40), 2), (2, 2, (64, 64), 7), (32, 8, (64, 128), 5)])
def test_gradient_of_states_in_place_copies_only_what_goes_in_pieces(sequences, heads, widths, launches):
    """ds0 over dsT is two walks (dk and dq, dv).  A walk in pieces is three launches, and dv's then needs a copy of its
    states: 3 + 1 + 3.  32 sequences of 8 heads go in pieces in walks of their own only: not where dv's goes like the
    others, and where it does not (64 x 128), it does, with its copy, beside the others in one launch."""
    torch = require_gpu()
    dk, dv = widths
    rows = 1024 * sequences
    plan = soma.LinearAttention(rows, sequences, heads, dk, dv, torch.bfloat16)
    q, k = (torch.zeros(rows, heads * dk, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    v, do = (torch.zeros(rows, heads * dv, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    l = torch.full((heads,), -0.1, device="cuda")
    s = torch.zeros(sequences, heads, dk, dv, device="cuda")
    out = [torch.empty_like(t) for t in (q, k, v)]
    assert nodes(torch, lambda st: plan.backward(q, k, v, l, do, *out, None, s, s, stream=st)) == launches
