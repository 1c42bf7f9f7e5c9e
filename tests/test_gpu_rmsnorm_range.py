"""moe_add_rmsnorm over all of bf16's range, with no or nearly no epsilon: squares that underflow or overflow fp32, and rows
whose mean does neither, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2607_12696_amd as moe
from oracle import attention as ref
from synth import attention as draw

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

DEV = torch.device("cuda:0")


@pytest.mark.parametrize("eps", [0.0, 1e-36])
@pytest.mark.parametrize("d", [32, 512, 2880, 7168, 16384])
@pytest.mark.parametrize("residual", [False, True])
def test_size_of_a_row(d, eps, residual):
    """Rows of 1e-38 to 1e38: the sum of squares of half of them is past fp32, at either end.  The norm's error is that of an
    fp32 sum of d squares, its root and two products, then one bf16 rounding."""
    print(f"range d={d} eps={eps} residual={residual}", flush=True)
    sizes = [1e-38, 1e-33, 1e-24, 1e-21, 1e-18, 1e-13, 1e-12, 1e-11, 1.0, 1e17, 1e19, 1e20, 1e25, 3e37]
    x = (draw.normal(d, "x", len(sizes), d).double() * torch.tensor(sizes, dtype=torch.float64)[:, None]).to(torch.bfloat16)
    r = (draw.normal(d, "r", len(sizes), d).double() * torch.tensor(sizes, dtype=torch.float64)[:, None]).to(torch.bfloat16)
    w = (1 + 0.3 * draw.normal(d, "w", d).float()).to(torch.bfloat16)
    r = r if residual else None
    v, u = ref.rmsnorm(x.double().numpy(), None if r is None else r.double().numpy(), w.double().numpy(), eps)
    assert np.all(np.abs(v) < 3.3e38)
    total, y, q, s = moe.moe_add_rmsnorm(x.to(DEV), w.to(DEV), eps, residual=None if r is None else r.to(DEV),
                                         qfmt=moe.MOE_Q_FP8_ROW)
    rel = (d / 2 + 12) * 2.0 ** -24
    assert np.all(np.abs(total.cpu().double().numpy() - v) <= (2.0 ** -8 + 2.0 ** -23) * np.abs(v) + 2.0 ** -133)
    assert np.all(np.abs(y.cpu().double().numpy() - u) <= (2.0 ** -8 + rel) * np.abs(u) + 1e-38)
    top = np.abs(u).max(1, keepdims=True)
    assert np.all(np.abs(s.cpu().double().numpy() - top / 448) <= (rel + 2.0 ** -22) * top / 448)
    # A code's value is within half a step of three bits, or of the smallest codes' spacing 2^-9.
    wide = s.cpu().double().numpy()
    assert np.all(np.abs(ref.E4M3[q.cpu().numpy()] * wide - u) <= (2.0 ** -4 + 4 * rel) * np.abs(u) + 2.0 ** -10 * wide)


@pytest.mark.parametrize("fmt", [moe.MOE_Q_FP8_GROUP, moe.MOE_Q_MXFP8, moe.MOE_Q_FP8_ROW])
def test_rows_beside_each_other_and_specials(fmt):
    """Tiny, huge, infinite and NaN rows leave each other alone; a row of zeros without epsilon is 0 / 0."""
    x = draw.normal(5, "x", 7, 4096)
    x[1] *= 2.0 ** -100
    x[2] *= 2.0 ** 100
    x[3] = 0
    x[4, 9], x[5, 9] = float("inf"), float("nan")
    w = (1 + 0.3 * draw.normal(5, "w", 4096).float()).to(torch.bfloat16)
    _, y, q, _ = (t if t is None else t.cpu() for t in moe.moe_add_rmsnorm(x.to(DEV), w.to(DEV), 0.0, qfmt=fmt))
    keep = [0, 1, 2, 6]
    _, u = ref.rmsnorm(x[keep].double().numpy(), None, w.double().numpy(), 0.0)
    assert np.all(np.abs(y[keep].double().numpy() - u) <= (2.0 ** -8 + 2060 * 2.0 ** -24) * np.abs(u) + 1e-38)
    assert torch.isnan(y[3]).all() and torch.isnan(y[5]).all()
    assert torch.isnan(y[4, 9]) and (y[4, :9] == 0).all() and (y[4, 10:] == 0).all()
    assert (q[[3, 5]] & 0x7F).eq(0x7F).all()
    # A power of two through the whole row changes nothing.
    _, z, _, _ = moe.moe_add_rmsnorm(draw.normal(5, "x", 7, 4096).to(DEV), w.to(DEV), 0.0)
    assert torch.equal(y[1:3], z.cpu()[1:3])
