"""Operators of 8-bit layers and clipping on batches without rows, on matrices without columns, and on more rows than the products' tiles are numbered for."""
import pytest
import torch

import paper_2401_09135_amd as A
from fp8_reference import DEV

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def new(*shape, dtype=F32):
    return torch.full(shape, 7.0, dtype=dtype, device=DEV)


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("outs", ["y", "q", "yq"])
@pytest.mark.parametrize("d", [1, 896, 5000])
def test_norm_of_no_rows(add, outs, d):
    r = new(0, d) if add else None
    A.k_norm_fwd(new(0, d), new(d), resid=r, total=r, y=new(0, d, dtype=BF16) if "y" in outs else None, q=A.Fp8.empty(0, d) if "q" in outs else None, rstd=new(0))
    dg = new(d)
    A.k_norm_bwd(new(0, d, dtype=BF16), new(0, d), new(0), new(d), new(0, d), dg, None, ds_in=r, ds_lp=new(0, d, dtype=BF16))
    assert (dg == 0).all()


@pytest.mark.parametrize("rows,cols", [(0, 128), (0, 5), (7, 0), (0, 0)])
def test_quantiser_of_nothing(rows, cols):
    q, qt = A.Fp8.empty(rows, cols), A.Fp8.empty(cols, rows, "e5m2", 128)
    for pair in ((q, None), (None, qt), (q, qt)):
        A.k_quant_fp8(new(rows, cols), *pair)


@pytest.mark.parametrize("M,N,K", [(0, 5, 128), (5, 0, 128), (0, 0, 0), (0, 5, 0), (300, 200, 0)])
@pytest.mark.parametrize("out", [F32, BF16])
def test_products_of_nothing(M, N, K, out):
    a, b, c = A.Fp8.empty(M, K), A.Fp8.empty(N, K, block_rows=128), new(M, N, dtype=out)
    A.k_gemm_fp8(a, b, c)
    assert (c == 0).all()
    r = torch.randn(M, N, device=DEV)
    A.k_gemm_fp8(a, b, c, resid=r, ws=torch.empty(256, dtype=torch.uint8, device=DEV))
    assert torch.equal(c, r.to(out))


def test_adamw_of_nothing():
    e = new(0)
    A.k_adamw_clip(e, e, e, e, None, 0, 1, 1e-3, new(1), 1.0)


@pytest.mark.parametrize("tile", [64, 128, 256])
def test_more_rows_than_a_launch_numbers(tile):
    """N = 3: a launch takes 2^22 rows.  Whole numbers, so that every element is exact."""
    M, N, K = (1 << 22) + 300, 3, 130
    g = torch.Generator(DEV).manual_seed(1)
    a, b = A.Fp8.empty(M, K, block_rows=128), A.Fp8.empty(N, K)
    va, vb = (torch.randint(-4, 5, (n, K), generator=g, device=DEV).float() for n in (M, N))
    for f, v in ((a, va), (b, vb)):
        f.data.copy_(v.to(torch.float8_e4m3fn))
        f.scale.view(torch.uint8).fill_(127)
    half = a.scale.view(torch.uint8)
    half[-2:] = 128                                     # the last 172 rows under a scale of 2
    c = new(M, N)
    A.set_gemm_fp8(tile)
    try:
        A.k_gemm_fp8(a, b, c)
    finally:
        A.set_gemm_fp8(0)
    want = va @ vb.t().contiguous()                     # |sums| <= 130 * 16: exact in fp32
    want[(len(half) - 2) * 128:] *= 2
    assert torch.equal(c, want)
