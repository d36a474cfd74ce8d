"""Norms with an 8-bit output and their backward pass where fp32 alone would lose the result: rows whose mean is far larger than their spread, rows at either
end of fp32's range.  Against the definitions in 64 bits."""
import pytest
import torch

import paper_2401_09135_amd as A
from fp8_reference import DEV, LEAST, STEP, expand, norm_backward, norm_forward, quantise, wide

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24          # half a step of fp32
LEAST32 = 2.0 ** -150   # half of its smallest step
MOST32 = torch.finfo(torch.float32).max


def backward(dy, total, rstd, gain, norm):
    rows, d = total.shape
    ds, dgain = torch.full((rows, d), 7.0, device=DEV), torch.full((d,), 7.0, device=DEV)
    ws = torch.full((A.k_norm_bwd_ws_bytes(rows, d),), 0xFF, dtype=torch.uint8, device=DEV)
    A.k_norm_bwd(dy.to(DEV), total.to(DEV), rstd.to(DEV), gain.to(DEV), ds, dgain, ws, norm=norm)
    return ds.cpu().double(), dgain.cpu().double()


def check_backward(dy, total, gain, norm):
    """Every term with the roundings of the sums behind it; the row's mean costs nothing but what 64 bits leave of it."""
    rows, d = total.shape
    rstd = norm_forward(total, gain, 1e-5, norm)[1].float()
    want, want_g = norm_backward(dy, total, rstd, gain, norm)
    ds, dgain = backward(dy, total, rstd, gain, norm)
    r64, t64, h64 = rstd.double()[:, None], total.double(), (dy.double() * gain.double()).abs()
    n = 32 + d / 64
    off = t64.abs().amax(1, keepdim=True) * r64 * n * 2.0 ** -52 * (norm == "layer")
    xh = (t64 - t64.mean(1, keepdim=True) if norm == "layer" else t64).abs() * r64 + off
    err = r64 * n * U * (h64 + h64.mean(1, keepdim=True) + xh * (h64 * xh).mean(1, keepdim=True)) + 2 * LEAST32
    err = err + r64 * off * ((h64 * xh).mean(1, keepdim=True) + xh * h64.mean(1, keepdim=True)) * 2
    assert ((ds - want).abs() <= err).all()
    assert ((dgain - want_g).abs() <= (dy.double().abs() * (xh * (n + rows / 512 + 600) * U + 2 * off)).sum(0)).all()


@pytest.mark.parametrize("rows,d", [(40, 896), (700, 100), (9, 1023), (12, 2048), (5, 4104), (6, 9999), (3, 16384)])
@pytest.mark.parametrize("ratio", [1e3, 1e5])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layer_backward_of_rows_far_from_zero(rows, d, ratio, dtype):
    g = torch.Generator().manual_seed(rows + d)
    total = (ratio * torch.randn(rows, 1, generator=g).sign() + torch.randn(rows, d, generator=g)) * torch.exp(torch.randn(rows, 1, generator=g))
    dy = (0.1 * torch.randn(rows, d, generator=g)).to(TYPES[dtype])
    check_backward(dy, total, 1 + 0.2 * torch.randn(d, generator=g), "layer")


@pytest.mark.parametrize("rows,d", [(40, 896), (12, 2048), (6, 9999)])
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_backward_of_the_largest_rows(rows, d, norm):
    """Sums of a row, and the distance of an element from the mean, beyond fp32's range; rstd is below its normal numbers."""
    g = torch.Generator().manual_seed(d)
    total = (0.9 + 0.1 * torch.rand(rows, d, generator=g)) * 3.3e38
    total[:, ::7] *= -1
    check_backward(0.1 * torch.randn(rows, d, generator=g), total, 1 + 0.2 * torch.randn(d, generator=g), norm)


def check_forward(x, gain, eps, norm, fmt, resid=None):
    rows, d = x.shape
    y, rstd, q = torch.empty(rows, d, dtype=torch.bfloat16, device=DEV), torch.empty(rows, device=DEV), A.Fp8.empty(rows, d, fmt)
    total = torch.empty(rows, d, device=DEV) if resid is not None else None
    A.k_norm_fwd(x.to(DEV), gain.to(DEV), resid=resid.to(DEV) if resid is not None else None, total=total, y=y, q=q, rstd=rstd, norm=norm, eps=eps)
    t = x.float() if resid is None else x.float() + resid
    want, want_r = norm_forward(t, gain, eps, norm)
    fits = want_r <= MOST32
    got_r = rstd.cpu().double()
    assert ((got_r - want_r).abs() <= want_r * 1.01 * U + LEAST32)[fits].all() and torch.isinf(got_r[~fits]).all()
    # in double but for one rounding: what is left of the mean's, and that rounding
    err = t.double().abs().amax(1, keepdim=True) * want_r[:, None] * gain.double().abs() * (24 + d / 64) * 2.0 ** -52 * (norm == "layer") + want.abs() * 1.01 * U + LEAST32
    assert torch.isfinite(want).all() and ((y.cpu().double() - want).abs() <= err + (want.abs() + err) * 2.0 ** -8 + 2.0 ** -134).all()
    got_s = q.scale.cpu().view(torch.uint8).int()
    low, high = quantise((want.abs() - err).clamp(min=0), 1, fmt)[1].int(), quantise(want.abs() + err, 1, fmt)[1].int()
    # A block of zeros has the scale 1, byte 127, although one of `err` has the least: the two bounds, 127 and 0, then hold nothing between them.
    assert (((got_s >= low) & (got_s <= high)) | (got_s == quantise(want, 1, fmt)[1].int())).all()
    step = torch.maximum((want.abs() + err) * STEP[fmt], LEAST[fmt] * expand(torch.pow(2.0, got_s.double() - 127), 1, rows, d))
    assert ((wide(q) - want).abs() <= err + step).all()


@pytest.mark.parametrize("rows,d", [(5, 3), (40, 896), (9, 1023), (12, 2048), (5, 4104), (6, 9999)])
@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gain", [1.0, 100.0, 1e-30])
def test_forward_of_the_largest_rows(rows, d, norm, dtype, gain):
    g = torch.Generator().manual_seed(d)
    x = (0.9 + 0.1 * torch.rand(rows, d, generator=g)) * 3.3e38
    x[:, ::3] *= -1
    x[0, 1:], x[0, 0] = -3.3e38, 3.3e38
    check_forward(x.to(TYPES[dtype]), gain * (1 + 0.2 * torch.rand(d, generator=g)), 1e-5, norm, "e4m3" if d % 2 else "e5m2")


@pytest.mark.parametrize("rows,d", [(5, 3), (40, 896), (9, 1023), (12, 2048)])
@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("size,gain", [(1e-20, 1.0), (1e-30, 1e-9), (1e-37, 1e-3), (1e-41, 1.0), (1e-41, 1e-20)])
def test_forward_of_the_smallest_rows(rows, d, norm, size, gain):
    """Without eps: the result has the size of the gain, whatever the row's; rstd is infinite where it leaves fp32's range."""
    g = torch.Generator().manual_seed(d)
    x = torch.randn(rows, d, generator=g) * size
    x[:, 0] = 2 * size
    check_forward(x, gain * (1 + 0.2 * torch.rand(d, generator=g)), 0.0, norm, "e4m3")


def test_forward_with_an_eps_below_fp32():
    """A row of zeros stays one."""
    x = torch.zeros(4, 200)
    x[2] = torch.randn(200, generator=torch.Generator().manual_seed(0))
    check_forward(x, torch.ones(200), 1e-50, "rms", "e4m3", resid=torch.zeros(4, 200))
