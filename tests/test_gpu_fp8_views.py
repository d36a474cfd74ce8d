"""Operators of 8-bit layers on views, and in place wherever the interface allows it."""
import pytest
import torch

import paper_2401_09135_amd as A
from fp8_reference import DEV, DT, quantise, wide

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def rand(*shape, seed=0, dtype=F32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


@pytest.mark.parametrize("rows,d", [(1, 1), (3, 7), (9, 896), (5, 1023), (4, 2049), (3, 5001), (2, 16383)])
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_norm_adds_in_place_of_its_input(rows, d, norm):
    """total may be x in fp32."""
    x, r, gain = rand(rows, d), rand(rows, d, seed=1), rand(d, seed=2)

    def run(x, total):
        y, rstd, q = torch.zeros(rows, d, dtype=BF16, device=DEV), torch.zeros(rows, device=DEV), A.Fp8.empty(rows, d)
        A.k_norm_fwd(x, gain, resid=r, total=total, y=y, q=q, rstd=rstd, norm=norm)
        return [total, y, rstd, q.data.view(torch.uint8), q.scale.view(torch.uint8)]

    want = run(x, torch.empty_like(x))
    for a, b in zip(run(x, x), want):
        assert torch.equal(a, b)


def whole(rows, cols, fmt, seed):
    """Whole numbers up to 4 in the middle of a larger matrix of 8 bits, which holds NaN elsewhere."""
    g = torch.Generator().manual_seed(seed)
    up = lambda n, m: -(-n // m) * m
    kb = -(-cols // 128)
    data = torch.full((rows + 3, up(cols, 16) + 1024), 0x7F, dtype=torch.uint8, device=DEV)
    scale = torch.full((rows + 3, up(kb, 4) + 8), 0xFF, dtype=torch.uint8, device=DEV)
    f = A.Fp8(data.view(DT[fmt])[1:rows + 1, 512:512 + cols], scale.view(torch.float8_e8m0fnu)[1:rows + 1, 4:4 + kb])
    f.data.copy_(torch.randint(-4, 5, (rows, cols), generator=g).float().to(DT[fmt]).to(DEV))
    f.scale.view(torch.uint8).copy_(torch.randint(126, 129, (rows, kb), generator=g).to(torch.uint8).to(DEV))
    return f


@pytest.mark.parametrize("M,N,K,shares", [(1, 5, 40, 1), (70, 130, 300, 1), (70, 130, 300, 2), (300, 260, 700, 1), (300, 260, 700, 3), (256, 256, 512, 1), (384, 192, 256, 2)])
@pytest.mark.parametrize("tile", [64, 128, 256])
@pytest.mark.parametrize("out", [F32, BF16])
def test_product_of_views_with_a_view_added(M, N, K, shares, tile, out):
    """Operands inside larger ones, R and C inside larger matrices of different widths, aligned for 16 bytes or not: exact, and nothing else written."""
    a, b = whole(M, K, "e4m3", 1), whole(N, K, "e5m2", 2)
    want = wide(a) @ wide(b).t()
    ws = torch.full((shares * M * (N + 3) * 4 + 256,), 0xFF, dtype=torch.uint8, device=DEV)
    r64 = torch.randint(-100, 100, (M, N), generator=torch.Generator().manual_seed(3)).double() / 4
    A.set_gemm_fp8(tile, shares)
    try:
        for rpad, rat in ((16 - N % 16, 0), (16 - N % 16 + 16, 4), (5, 1)):
            for cpad, cat in ((16 - N % 16, 0), (16 - N % 16 + 16, 8), (3, 2)):
                rbig = torch.full((M + 1, N + rpad), float("nan"), device=DEV)
                r = rbig[:M, rat:rat + N]
                r.copy_(r64.float())
                big = torch.full((M + 2, N + cpad), 7.0, dtype=out, device=DEV)
                c = big[1:M + 1, cat:cat + N]
                A.k_gemm_fp8(a, b, c, resid=r, ws=ws)
                assert torch.equal(c.cpu(), (want + r64).float().to(out)), (rpad, rat, cpad, cat)
                c.fill_(7.0)
                assert (big == 7.0).all()
                if out is F32:
                    A.k_gemm_fp8(a, b, r, resid=r, ws=ws)          # C is R, inside a larger matrix
                    assert torch.equal(r.cpu().double(), want + r64)
                    r.fill_(float("nan"))
                    assert torch.isnan(rbig).all()
    finally:
        A.set_gemm_fp8(0)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_quantiser_from_and_into_views(dtype):
    """Columns of a larger matrix into the middle of larger ones in both orientations."""
    rows, cols = 261, 390
    big = rand(rows + 2, cols + 37, dtype=dtype)
    x = big[1:rows + 1, 5:5 + cols]
    q, qt = whole(rows, cols, "e4m3", 1), whole(cols, rows, "e4m3", 2)
    A.k_quant_fp8(x, q, qt)
    for f, m in ((q, x), (qt, x.t())):
        want, scale = quantise(m.contiguous(), 1, "e4m3")
        assert torch.equal(f.data.cpu().view(torch.uint8), want.view(torch.uint8)) and torch.equal(f.scale.cpu().view(torch.uint8), scale)
        base = f.data._base if f.data._base is not None else f.data
        assert int((base.view(torch.uint8) != 0x7F).sum()) <= f.data.numel()


def test_clipping_an_empty_list_and_lists_without_elements():
    norm = torch.full((1,), 5.0, device=DEV)
    A.k_grad_clip([], [], 1.0, norm, None)
    assert norm.item() == 0.0
    norm.fill_(5.0)
    e = [torch.empty(0, device=DEV)] * 120
    A.k_grad_clip(e, e, 1.0, norm, torch.empty(16, dtype=torch.uint8, device=DEV))
    assert norm.item() == 0.0
