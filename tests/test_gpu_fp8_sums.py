"""What the 8-bit instruction loses of sums of products that differ widely, and that fp32 results do not take it."""
import pytest
import torch

import paper_2401_09135_amd as A
from fp8_reference import DEV, wide

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def values(kind, rows, cols, g):
    x = torch.randn(rows, cols, generator=g)
    if kind == "one sign":
        return x.abs()
    if kind == "wide, one sign":
        return (x * torch.exp(2 * torch.randn(rows, cols, generator=g))).abs()
    if kind == "wide":
        return x * torch.exp(2 * torch.randn(rows, cols, generator=g))
    x[:, ::16] *= 100
    return x


@pytest.mark.parametrize("kind", ["one sign", "wide, one sign", "wide", "outliers"])
@pytest.mark.parametrize("fa,fb", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("tile", [64, 128, 256])
def test_sums_of_products_that_differ_widely(kind, fa, fb, tile):
    M, N, K = 80, 72, 1000
    g = torch.Generator().manual_seed(K)
    a, b = A.Fp8.empty(M, K, fa), A.Fp8.empty(N, K, fb)
    A.k_quant_fp8(values(kind, M, K, g).to(DEV), a)
    A.k_quant_fp8(values(kind, N, K, g).to(DEV), b)
    wa, wb = wide(a), wide(b)
    want, size = wa @ wb.t(), wa.abs() @ wb.abs().t()
    h, c = torch.empty(M, N, dtype=torch.bfloat16, device=DEV), torch.empty(M, N, device=DEV)
    A.set_gemm_fp8(tile)
    try:
        A.k_gemm_fp8(a, b, h)
        A.k_gemm_fp8(a, b, c)
    finally:
        A.set_gemm_fp8(0)
    # fp32 results: each of K additions rounds or cuts at most one step of the sum of magnitudes
    sums = (K + 8) * 2 * U * size
    assert ((c.cpu().double() - want).abs() <= sums).all()
    # bf16 results: of 8 neighbours in K, 7 lose less than 2^-13 of the largest product each, and then half a step of bf16
    p = (wa[:, None, :] * wb[None, :, :]).abs().view(M, N, K // 8, 8).amax(3).sum(2)
    lost = 7 * 2.0 ** -13 * p + sums
    assert ((h.cpu().double() - want).abs() <= lost + (want.abs() + lost) * 2.0 ** -8).all()
