"""moe_add_rmsnorm against the definition in 64 bits: every output format, widths that end inside a group and inside a
workgroup's vectors, aliased outputs, one row to many, and rows of zeros, large and non-finite values."""
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
FMT = {"none": moe.MOE_Q_NONE, "group": moe.MOE_Q_FP8_GROUP, "mx": moe.MOE_Q_MXFP8, "row": moe.MOE_Q_FP8_ROW}


def check(x, residual, w, eps, fmt, total, y, q, scales):
    v, u = ref.rmsnorm(x.double().numpy(), None if residual is None else residual.double().numpy(), w.double().numpy(), eps)
    d = x.shape[1]
    # v is one fp32 addition; the mean is an fp32 sum of d squares, its root and quotient a few roundings more.
    if total is not None:
        assert np.all(np.abs(total.cpu().double().numpy() - v) <= (2.0 ** -8 + 2.0 ** -23) * np.abs(v))
    rel = (d / 2 + 12) * 2.0 ** -24
    if y is not None:
        assert np.all(np.abs(y.cpu().double().numpy() - u) <= (2.0 ** -8 + rel) * np.abs(u) + 1e-38)
    if fmt == "none":
        return
    s, width = ref.group_scales(u, fmt)
    if fmt == "mx":
        got_s = 2.0 ** (scales.cpu().numpy().astype(np.float64) - 127)
        # A group whose maximum lies on a power of two may take either scale.
        near = np.stack([np.abs(u[:, i:i + 32]).max(1) for i in range(0, d, 32)], 1)
        edge = np.abs(near / 2.0 ** np.round(np.log2(np.maximum(near, 1e-300))) - 1) <= 4 * rel
        assert np.all((got_s == s) | edge)
    else:
        got_s = scales.cpu().double().numpy()
        assert np.all(np.abs(got_s - s) <= (rel + 2.0 ** -22) * s)
    wide = np.repeat(got_s, width, 1)[:, :d]
    value = ref.E4M3[q.cpu().numpy()]
    # The nearest code to u / scale, but for quotients within the fp32 error of a tie.
    exact = np.clip(u / wide, -448, 448)
    lo, hi = ref.E4M3[ref.e4m3(exact * (1 - 4 * rel))], ref.E4M3[ref.e4m3(exact * (1 + 4 * rel))]
    assert np.all((value >= np.minimum(lo, hi)) & (value <= np.maximum(lo, hi)))


@pytest.mark.parametrize("fmt", list(FMT))
@pytest.mark.parametrize("T,d", [(1, 32), (3, 160), (2, 512), (5, 2048), (4, 2080), (7, 2880), (64, 4096), (4, 7168), (3, 8192),
                                 (2, 8224), (3, 16384), (700, 320)])
def test_against_definition(T, d, fmt):
    print(f"rmsnorm T={T} d={d} fmt={fmt}", flush=True)
    x, r = draw.normal(d, "x", T, d), draw.normal(d, "r", T, d, std=3.0)
    r[:, ::41] *= 30
    w = (1 + 0.3 * draw.normal(d, "w", d).float()).to(torch.bfloat16)
    out = moe.moe_add_rmsnorm(x.to(DEV), w.to(DEV), 1e-6, residual=r.to(DEV), qfmt=FMT[fmt])
    check(x, r, w, 1e-6, fmt, *out)


@pytest.mark.parametrize("fmt", ["none", "group"])
def test_in_place_and_without_residual(fmt):
    T, d = 6, 1536
    x, r = draw.normal(1, "x", T, d), draw.normal(1, "r", T, d)
    w = draw.normal(1, "w", d)
    xd, rd, wd = x.to(DEV), r.to(DEV), w.to(DEV)
    out = moe.moe_add_rmsnorm(xd, wd, 1e-5, residual=rd, qfmt=FMT[fmt], sum=rd, y=xd)
    assert out[0] is rd and out[1] is xd
    check(x, r, w, 1e-5, fmt, *out)
    total, y, q, s = moe.moe_add_rmsnorm(x.to(DEV), wd, 1e-5, qfmt=FMT[fmt], want_sum=False, want_y=fmt == "none")
    assert total is None and (y is None) == (fmt != "none")
    check(x, None, w, 1e-5, fmt, None, y, q, s)


@pytest.mark.parametrize("fmt", list(FMT))
def test_special_rows(fmt):
    T, d = 6, 480
    x = draw.normal(2, "x", T, d)
    x[1] = 0
    x[2, 7] = float("inf")
    x[3, 100] = float("nan")
    x[4] = 1e18  # the mean of its squares fits fp32, their sum does not; the row after it must not notice
    w = torch.ones(d, dtype=torch.bfloat16)
    total, y, q, s = (None if t is None else t.cpu() for t in moe.moe_add_rmsnorm(x.to(DEV), w.to(DEV), 1e-6, qfmt=FMT[fmt]))
    keep = [0, 1, 4, 5]
    check(x[keep], None, w, 1e-6, fmt, total[keep], y[keep], None if q is None else q[keep], None if s is None else s[keep])
    assert torch.isnan(y[2, 7]) and (y[2, :7] == 0).all()
    assert torch.isnan(y[3]).all()
    if q is not None:
        assert (q[1] & 0x7F).eq(0).all() and q[3].eq(0x7F).logical_or(q[3].eq(0xFF)).all()


def test_other_stream_and_repeatability():
    x, w = draw.normal(3, "x", 33, 2880).to(DEV), draw.normal(3, "w", 2880).to(DEV)
    first = moe.moe_add_rmsnorm(x, w, 1e-6, qfmt=moe.MOE_Q_MXFP8)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        again = moe.moe_add_rmsnorm(x, w, 1e-6, qfmt=moe.MOE_Q_MXFP8)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))
