"""Dropout and the norm in rows narrower than a group of eight, contiguous and apart, against their formulas in 64 bits."""
import numpy as np
import pytest

import block_reference as ref
from gpu_common import require_gpu
from paper_2609_37899_amd import soma
from test_gpu_norm_dropout import LAYER, SEED, STEP, TYPES, both, make, near

pytestmark = pytest.mark.gpu

WIDTHS = [1, 2, 3, 4, 5, 6, 7, 8, 9]
# elements between rows: none, so that groups reach over several rows; 8 and 11, so that fp32 rows of 4 and 5 and bf16
# rows of any of these widths are aligned or not
PADS = [0, 4, 8, 11]


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("rows", [2, 20])
@pytest.mark.parametrize("pad", PADS)
def test_norm_of_narrow_rows(types, width, rows, pad):
    torch = require_gpu()
    T, S = types
    p, where = 0.2, (SEED, STEP, LAYER)
    x, w = make(torch, types, rows, width, p, pad=pad)
    plan = soma.RmsNorm(rows, width, getattr(torch, T), getattr(torch, S), eps=1e-5, drop=p)
    total, y = torch.full_like(x["dtotal"], 7.0), torch.full_like(x["dy"], 7.0)
    plan.forward(x["x"], x["gain"], y, x["residual"], total, None, *where)
    torch.cuda.synchronize()
    eps = np.float64(np.float32(1e-5))
    want = ref.norm(w["x"], w["residual"], w["gain"], eps, w["factor"])
    near(total, want["total"], want["total_err"], S, "total")
    near(y, want["y"], want["y_err"], T, "y")
    dr, dx, dg = torch.full_like(total, 7.0), torch.full_like(y, 7.0), torch.full_like(x["gain"], 7.0)
    plan.backward(total, x["gain"], x["dy"], x["dtotal"], dr, dx, dg, *where)
    torch.cuda.synchronize()
    back = ref.norm_backward(total.double().cpu().numpy(), w["gain"], w["dy"], w["dtotal"], eps, w["factor"])
    near(dr, back["dresidual"], back["dresidual_err"], S, "dresidual")
    near(dx, back["dx"], back["dx_err"], T, "dx")
    near(dg, back["dgain"], back["dgain_err"], "float32", "dgain")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("rows", [2, 20])
@pytest.mark.parametrize("pad", PADS)
def test_dropout_of_narrow_rows(dtype, width, rows, pad):
    """Strided rows added to contiguous ones, and into these."""
    torch = require_gpu()
    g = np.random.default_rng(5)
    x, x64 = both(torch, g.standard_normal((rows, width)), dtype, pad=pad)
    r, r64 = both(torch, g.standard_normal((rows, width)), dtype)
    plan = soma.Dropout(rows, width, x.dtype, 0.3)
    y, z = torch.full_like(r, 7.0), r.clone()
    plan.forward(x, y, r, SEED, STEP, LAYER)
    plan.forward(x, z, z, SEED, STEP, LAYER)
    torch.cuda.synchronize()
    exact = ref.drop(x64, ref.keep(rows, width, 0.3, SEED, STEP, LAYER))
    near(y, exact + r64, ref.U * (2 * np.abs(exact) + np.abs(exact + r64)), dtype, "y")
    assert torch.equal(y, z)
