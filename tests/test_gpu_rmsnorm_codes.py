"""The 8-bit codes of moe_add_rmsnorm where the norm is known to the bit: rows of +-1 without epsilon have it at +-weight, so
scales and codes follow from fp32 divisions alone, and quotients lie on ties between two codes."""
import numpy as np
import pytest
import torch

import paper_2607_12696_amd as moe
from oracle import attention as ref

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

DEV = torch.device("cuda:0")


def weights(top):
    """[2048] bf16 weights, `top` first in every 128: of all 1024 bf16 numbers from 2^-7 to 2, those up to `top`, mixed."""
    w = torch.arange(0x3C00, 0x4000, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    w = w[w <= top]
    order = torch.randperm(len(w), generator=torch.Generator().manual_seed(1))
    out = w[order.repeat(4)[:2048]].clone()
    out[::128] = top
    return out


@pytest.mark.parametrize("fmt", [moe.MOE_Q_FP8_GROUP, moe.MOE_Q_FP8_ROW, moe.MOE_Q_MXFP8])
@pytest.mark.parametrize("top", [1.0, 1.078125, 1.1875, 1.296875, 1.53125, 1.59375, 1.625, 1.75, 1.9375])
def test_codes_are_those_of_the_quotient(top, fmt):
    w = weights(top)
    x = torch.where(torch.rand(3, 2048, generator=torch.Generator().manual_seed(2)) < 0.5, -1.0, 1.0).to(torch.bfloat16)
    _, y, q, s = (t.cpu() for t in moe.moe_add_rmsnorm(x.to(DEV), w.to(DEV), 0.0, qfmt=fmt))
    u = x.float() * w.float()
    assert torch.equal(y.float(), u)
    if fmt == moe.MOE_Q_MXFP8:
        wide = np.repeat(np.exp2(s.numpy().astype(np.float32) - 127), 32, 1)
    else:
        assert np.array_equal(s.numpy(), np.full(s.shape, np.float32(top) / np.float32(448)))
        wide = np.repeat(s.numpy(), 2048 // s.shape[1], 1)
    want = ref.e4m3(u.numpy() / wide)
    got = q.numpy()
    bad = np.argwhere(got != want)
    assert not len(bad), (top, [(float(u[i, j]), hex(got[i, j]), hex(want[i, j])) for i, j in bad[:5]])


@pytest.mark.parametrize("fmt", [moe.MOE_Q_FP8_GROUP, moe.MOE_Q_FP8_ROW, moe.MOE_Q_MXFP8])
def test_zeros_and_infinities(fmt):
    """Zeros keep their sign.  An infinite norm (a weight too large for it) saturates in MX, whose scale stays finite; the
    other formats' scale is infinite then, and the quotients are zeros and a NaN."""
    x = torch.ones(2, 256).to(torch.bfloat16)
    x[:, 3], x[:, 4], x[1, 7] = 0.0, -0.0, -255.0  # row 1: 7 has 15.6 times the root mean square
    w = torch.ones(256, dtype=torch.bfloat16)
    w[7] = 3.2e38
    _, y, q, s = (t.cpu() for t in moe.moe_add_rmsnorm(x.to(DEV), w.to(DEV), 0.0, qfmt=fmt))
    assert y[1, 7] == -float("inf") and torch.isfinite(y[0]).all()
    assert (q[:, 3] == 0).all() and (q[:, 4] == 0x80).all()
    if fmt == moe.MOE_Q_MXFP8:
        assert s[1, 0] == 247 and q[1, 7] == 0xFE  # 2^120, -448
        assert (q[1, 32:] != 0).all()
    else:
        assert s[1, 0] == float("inf") and q[1, 7] & 0x7F == 0x7F
        assert (q[1, 8:128] & 0x7F == 0).all()
