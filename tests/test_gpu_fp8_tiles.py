"""Products in 8 bits of more tiles than the chip has CUs, where a workgroup goes from one tile to the next: whole numbers, so that every element has to be exact."""
import pytest
import torch

import paper_2401_09135_amd as A
from fp8_reference import DEV, DT, expand

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def operand(rows, cols, fmt, block_rows, seed):
    """Whole numbers up to 4 under scales of 1/2, 1 or 2; NaN in what lies behind the columns.  (Fp8, the values in float64)"""
    g = torch.Generator(DEV).manual_seed(seed)
    up = lambda n, m: -(-n // m) * m
    kb, rb = -(-cols // 128), -(-rows // block_rows)
    data = torch.full((rows, up(cols, 16) + 16), 0x7F, dtype=torch.uint8, device=DEV)
    scale = torch.full((rb, up(kb, 4) + 4), 0xFF, dtype=torch.uint8, device=DEV)
    f = A.Fp8(data.view(DT[fmt])[:, :cols], scale.view(torch.float8_e8m0fnu)[:, :kb], block_rows)
    v = torch.randint(-4, 5, (rows, cols), generator=g, device=DEV).float()
    e = torch.randint(-1, 2, (rb, kb), generator=g, device=DEV)
    f.data.copy_(v.to(DT[fmt]))
    f.scale.view(torch.uint8).copy_((e + 127).to(torch.uint8))
    return f, v.double() * expand(torch.ldexp(torch.ones_like(e, dtype=torch.float64), e), block_rows, rows, cols)


# (M, N, shares): 340, 396 and 660 tiles of 256 x 256, the last row and column of them partly or (by 128) half outside; whole ones
SIZES = [(5000, 4200, 1), (2950, 2600, 3), (2950, 2600, 5), (4992, 4160, 1)]


@pytest.mark.parametrize("M,N,shares", SIZES)
@pytest.mark.parametrize("K", [15, 128, 130, 385, 640, 897, 1500])
@pytest.mark.parametrize("out", [F32, BF16])
def test_every_element_of_many_tiles(M, N, shares, K, out):
    """Sums of multiples of 1/4 below 2^24 / 4, in any order."""
    fa, fb, ra, rb = [("e4m3", "e4m3", 1, 128), ("e5m2", "e4m3", 1, 1), ("e4m3", "e5m2", 128, 1), ("e5m2", "e5m2", 1, 128)][(K + shares) % 4]
    (a, wa), (b, wb) = operand(M, K, fa, ra, K), operand(N, K, fb, rb, K + 1)
    want = wa @ wb.t().contiguous()
    r = torch.randint(-100, 100, (M, N), device=DEV, generator=torch.Generator(DEV).manual_seed(3)).float() / 4
    ws = torch.full((shares * M * (N + 3) * 4 + 256,), 0xFF, dtype=torch.uint8, device=DEV) if shares > 1 else None
    A.set_gemm_fp8(256, shares)
    try:
        for pad in (-N % 16 + 16, 1):
            for add in (None, r):
                big = torch.full((M + 2, N + pad), 7.0, dtype=out, device=DEV)
                c = big[1:M + 1, :N]
                A.k_gemm_fp8(a, b, c, resid=add, ws=ws)
                assert torch.equal(c, (want + add if add is not None else want).float().to(out)), (pad, add is None)
                big[1:M + 1, :N] = 7.0
                assert (big == 7.0).all()
    finally:
        A.set_gemm_fp8(0)


@pytest.mark.parametrize("M,N,K", [(130, 140, 200), (600, 520, 450)])
@pytest.mark.parametrize("tile", [64, 128, 256])
@pytest.mark.parametrize("out", [F32, BF16])
def test_what_is_not_finite_shows_in_every_kernel(M, N, K, tile, out):
    (a, wa), (b, wb) = operand(M, K, "e5m2", 1, 5), operand(N, K, "e4m3", 1, 6)
    a.data.view(torch.uint8)[3, K - 1] = 0x7C        # infinity
    a.data.view(torch.uint8)[M - 1, 130] = 0x7E      # NaN
    b.data.view(torch.uint8)[5, 0] = 0x7F            # NaN
    wa, wb = wa.cpu(), wb.cpu()
    wa[3, K - 1], wa[M - 1, 130], wb[5, 0] = float("inf"), float("nan"), float("nan")
    want = wa @ wb.t()
    c = torch.empty(M, N, dtype=out, device=DEV)
    A.set_gemm_fp8(tile)
    try:
        A.k_gemm_fp8(a, b, c)
    finally:
        A.set_gemm_fp8(0)
    got, want, ok = c.cpu().double(), want.float().to(out).double(), ~torch.isnan(want)
    assert torch.equal(torch.isnan(got), ~ok) and torch.equal(got[ok], want[ok])
