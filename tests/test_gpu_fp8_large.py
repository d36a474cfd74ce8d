"""The operators of 8-bit layers and clipping where offsets pass 32 bits: the last rows of large matrices against calls on those rows alone."""
import pytest
import torch

import paper_2401_09135_amd as A

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def rows_of(f, at, n):
    """n rows of an Fp8 from row at on, with a scale for each row, as an Fp8 of its own."""
    return A.Fp8(f.data[at:at + n], f.scale[at:at + n], 1)


def test_quantiser_and_products_beyond_32_bits():
    rows, cols, tail = 70000, 65536, 512
    at = rows - tail - 3
    x = torch.zeros(rows, cols, dtype=BF16, device=DEV)
    x[at:] = torch.randn(rows - at, cols, device=DEV, generator=torch.Generator(DEV).manual_seed(1))
    q, qt = A.Fp8.empty(rows, cols), A.Fp8.empty(cols, rows)
    A.k_quant_fp8(x, q, qt)
    few = A.Fp8.empty(rows - at, cols)
    A.k_quant_fp8(x[at:], few)
    assert torch.equal(q.data[at:].view(torch.uint8), few.data.view(torch.uint8)) and torch.equal(q.scale[at:].view(torch.uint8), few.scale.view(torch.uint8))
    assert not q.data[:at].view(torch.uint8).any()
    last = A.Fp8.empty(130, rows)
    A.k_quant_fp8(x[:, cols - 130:], qt=last)            # blocks along the rows: the same whatever columns there are
    assert torch.equal(qt.data[cols - 130:].view(torch.uint8), last.data.view(torch.uint8)) and torch.equal(qt.scale[cols - 130:].view(torch.uint8), last.scale.view(torch.uint8))
    del x, qt, last
    b = A.Fp8.empty(192, cols)
    A.k_quant_fp8(torch.randn(192, cols, device=DEV, generator=torch.Generator(DEV).manual_seed(2)), b)
    for tile in (64, 128, 256):
        A.set_gemm_fp8(tile)
        try:
            c, d = torch.empty(rows, 192, device=DEV), torch.empty(tail, 192, device=DEV)
            A.k_gemm_fp8(q, b, c)
            A.k_gemm_fp8(rows_of(q, rows - tail, tail), b, d)
        finally:
            A.set_gemm_fp8(0)
        assert torch.equal(c[rows - tail:], d) and d.any() and not c[:at].any()


def product(a, b, out, tile):
    c = torch.empty(a.shape[0], b.shape[0], dtype=out, device=DEV)
    A.set_gemm_fp8(tile)
    try:
        A.k_gemm_fp8(a, b, c, resid=torch.zeros_like(c, dtype=torch.float32))
    finally:
        A.set_gemm_fp8(0)
    return c


@pytest.mark.parametrize("out", [torch.float32, BF16])
def test_results_beyond_32_bits(out):
    M, N, K, tail = 70000, 40000, 128, 700
    g = torch.Generator(DEV).manual_seed(3)
    a, b = A.Fp8.empty(M, K), A.Fp8.empty(N, K)
    A.k_quant_fp8(torch.randn(M, K, device=DEV, generator=g), a)
    A.k_quant_fp8(torch.randn(N, K, device=DEV, generator=g), b)
    r = torch.zeros(M, N, device=DEV)
    r[M - tail:] = torch.randn(tail, N, device=DEV, generator=g)
    for tile in (64, 256):
        A.set_gemm_fp8(tile)
        try:
            c, d = torch.empty(M, N, dtype=out, device=DEV), torch.empty(tail, N, dtype=out, device=DEV)
            A.k_gemm_fp8(a, b, c, resid=r)
            A.k_gemm_fp8(rows_of(a, M - tail, tail), b, d, resid=r[M - tail:])
        finally:
            A.set_gemm_fp8(0)
        assert torch.equal(c[M - tail:], d)
        assert torch.equal(c[:128], product(rows_of(a, 0, 128), b, out, tile))   # the same kernel: another adds in another order


def test_norms_beyond_32_bits():
    rows, d, tail = 300000, 16384, 40
    x = torch.zeros(rows, d, dtype=BF16, device=DEV)
    x[rows - tail:] = torch.randn(tail, d, device=DEV, generator=torch.Generator(DEV).manual_seed(4))
    gain = torch.rand(d, device=DEV) + 0.5

    def forward(x):
        n = len(x)
        y, rstd, q = torch.empty(n, d, dtype=BF16, device=DEV), torch.empty(n, device=DEV), A.Fp8.empty(n, d)
        A.k_norm_fwd(x, gain, y=y, q=q, rstd=rstd)
        return y, rstd, q.data.view(torch.uint8), q.scale.view(torch.uint8)

    every, few = forward(x), forward(x[rows - tail:].clone())
    for a, b in zip(every, few):
        assert torch.equal(a[rows - tail:], b)
    assert not every[0][:rows - tail].any()
    total, rstd = x.float(), every[1]
    del every
    ws, ws2 = (torch.empty(A.k_norm_bwd_ws_bytes(n, d), dtype=torch.uint8, device=DEV) for n in (rows, tail))
    ds, ds2 = torch.empty(rows, d, device=DEV), torch.empty(tail, d, device=DEV)
    dg, dg2 = torch.empty(d, device=DEV), torch.empty(d, device=DEV)
    A.k_norm_bwd(x, total, rstd, gain, ds, dg, ws)
    A.k_norm_bwd(x[rows - tail:].clone(), total[rows - tail:].clone(), rstd[rows - tail:].clone(), gain, ds2, dg2, ws2)
    assert torch.equal(ds[rows - tail:], ds2) and not ds[:rows - tail].any()
    # the gain's gradient adds the same 40 rows, the others are zero, in another order
    assert ((dg - dg2).abs() <= 2 * 40 * 2.0 ** -24 * (x[rows - tail:].float().abs() * (total[rows - tail:] * rstd[rows - tail:, None]).abs()).sum(0)).all()


def test_gradients_beyond_32_bits():
    n = (1 << 32) + 5
    g = torch.zeros(n, dtype=BF16, device=DEV)
    g[0], g[-1], g[1 << 31] = 3.0, 4.0, 12.0
    norm, ws = torch.empty(1, device=DEV), torch.empty(A.k_grad_norm_ws_bytes([g]), dtype=torch.uint8, device=DEV)
    A.k_grad_norm([g], norm, ws)
    assert norm.item() == 13.0
    A.k_grad_clip([g], [g], 6.5, norm, ws)
    assert (g[0].item(), g[1 << 31].item(), g[-1].item()) == (1.5, 6.0, 2.0) and not g[1:1 << 31].any() and not g[(1 << 31) + 1:-1].any()
    del g
    P = (1 << 30) + 3                                           # 4 GiB a vector
    theta, grad, m, v = (torch.zeros(P, device=DEV) for _ in range(4))
    grad[-1], grad[-5] = 3.0, -4.0
    A.k_grad_norm([grad], norm, torch.empty(A.k_grad_norm_ws_bytes([grad]), dtype=torch.uint8, device=DEV))
    A.k_adamw_clip(theta, grad, m, v, None, P, 1, 0.5, norm, 2.5)
    # clipped to half: m = 0.1 g / 2; the first step of AdamW is lr times the sign (eps aside)
    assert abs(m[-1].item() - 0.15) < 1e-7 and abs(m[-5].item() + 0.2) < 1e-7
    assert abs(theta[-1].item() + 0.5) < 1e-6 and abs(theta[-5].item() - 0.5) < 1e-6 and not theta[:-5].any()
