"""The norms' backward pass where fp32 alone would lose the result: rows whose mean is far larger than their spread, rows at the end of fp32's range.  Against the definitions in 64 bits."""
import pytest
import torch

import paper_2401_09135_amd as A
from fp8_reference import DEV, norm_backward, norm_forward

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24          # half a step of fp32
LEAST32 = 2.0 ** -150   # half of its smallest step


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
