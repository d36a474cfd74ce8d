"""Operators for linear layers in 8 bits on the GPU, against their definitions in 64 bits (fp8_reference)."""
import math

import pytest
import torch

import paper_2401_09135_amd as A
from fp8_reference import DEV, DT, LEAST, STEP, TOP, block_amax, expand, norm_backward, norm_forward, quantise, wide

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24      # half a step of fp32


def fp8_in_canvas(rows, cols, fmt, block_rows, extra=0):
    """An Fp8 inside buffers that are wider and longer than it and hold 0xAA: (Fp8, data canvas, scale canvas)."""
    up = lambda n, m: -(-n // m) * m
    kb, rb = -(-cols // 128), -(-rows // block_rows)
    data = torch.full((rows + 2, up(cols, 16) + 16 * extra), 0xAA, dtype=torch.uint8, device=DEV)
    scale = torch.full((rb + 2, up(kb, 4) + 4 * extra), 0xAA, dtype=torch.uint8, device=DEV)
    f = A.Fp8(data.view(DT[fmt])[1:rows + 1, :cols], scale.view(torch.float8_e8m0fnu)[1:rb + 1, :kb], block_rows)
    return f, data, scale


def untouched(canvas, rows, cols):
    c = canvas.cpu().clone()
    c[1:rows + 1, :cols] = 0xAA
    return bool((c == 0xAA).all())


def special_values(rows, cols, seed, dtype):
    """Blocks of ordinary values, with rows of zeros, of the smallest and the largest numbers, of ties and of what is not finite."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(3 * torch.randn(rows, 1, generator=g))
    kinds = torch.arange(rows) % 11
    x[kinds == 3] = 0.0
    x[kinds == 4] *= 1e-38 / 3
    x[kinds == 5] = x[kinds == 5].sign() * 3.0e38
    x[kinds == 6] = torch.round(x[kinds == 6].clamp(-3, 3) * 16) / 16      # many ties
    x[kinds == 7, ::3] = float("inf")
    x[kinds == 7, 1::5] = float("-inf")
    x[kinds == 8, ::4] = float("nan")
    x[kinds == 9] = float("nan")
    x[kinds == 10, ::2] = 448.0 * 2.0 ** -7      # the border of a scale, and one step above it
    x[kinds == 10, 1::2] = 448.0 * 2.0 ** -7 * (1 + 2.0 ** -7 * (cols % 2))
    return x.to(dtype)


def bytes_of(t):
    return t.cpu().view(torch.uint8)


def same_values(got, want):
    """Bit for bit, all NaNs being one."""
    g, w = got.cpu().float(), want.float()
    return torch.equal(torch.isnan(g), torch.isnan(w)) and torch.equal(bytes_of(got)[~torch.isnan(g)], bytes_of(want)[~torch.isnan(w)])


SIZES = [(1, 1), (3, 5), (1, 4096), (2777, 1), (16, 128), (128, 128), (129, 257), (300, 1000), (37, 2048), (255, 127)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantiser_is_exact(rows, cols, block_rows, fmt, dtype):
    x = special_values(rows, cols, rows + cols, TYPES[dtype])
    q, dq, sq = fp8_in_canvas(rows, cols, fmt, block_rows)
    qt, dt, st = fp8_in_canvas(cols, rows, fmt, block_rows, extra=1)
    want, want_s = quantise(x, block_rows, fmt)
    want_t, want_st = quantise(x.t().contiguous(), block_rows, fmt)
    for outs in ((q, None), (None, qt), (q, qt)):
        for canvas in (dq, sq, dt, st):
            canvas.fill_(0xAA)
        A.k_quant_fp8(x.to(DEV), *outs)
        if outs[0]:
            assert torch.equal(bytes_of(q.scale), want_s) and same_values(q.data, want)
            assert untouched(dq, rows, cols) and untouched(sq, *want_s.shape)
        if outs[1]:
            assert torch.equal(bytes_of(qt.scale), want_st) and same_values(qt.data, want_t)
            assert untouched(dt, cols, rows) and untouched(st, *want_st.shape)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("off,pad", [(0, 0), (1, 0), (0, 3), (3, 5), (8, 8)])
def test_quantiser_takes_strided_and_unaligned_input(dtype, off, pad):
    rows, cols = 140, 200
    buf = special_values(rows + 1, cols + pad + 8, 7, TYPES[dtype]).to(DEV).view(-1)
    x = buf[off:off + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    q, qt = A.Fp8.empty(rows, cols, "e4m3", 1), A.Fp8.empty(cols, rows, "e5m2", 128)     # different forms for either
    A.k_quant_fp8(x, q, qt)
    for f, want in ((q, quantise(x, 1, "e4m3")), (qt, quantise(x.t().contiguous(), 128, "e5m2"))):
        assert torch.equal(bytes_of(f.scale), want[1]) and same_values(f.data, want[0])


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_quantiser_rounds_every_fp32_near_every_8_bit_value(fmt):
    """All 8-bit values, the midpoints between neighbours and the fp32 numbers next to both, under a scale of 1."""
    v = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(DT[fmt]).float()
    v = v[torch.isfinite(v)].sort().values
    mid = (v[1:] + v[:-1]) / 2
    base = torch.cat([v, mid])
    x = torch.cat([base, torch.nextafter(base, torch.full_like(base, math.inf)), torch.nextafter(base, torch.full_like(base, -math.inf))])
    x = x[x.abs() <= TOP[fmt]]
    rows = -(-x.numel() // 127)
    m = torch.full((rows, 128), TOP[fmt])
    m[:, 1:] = torch.cat([x, torch.zeros(rows * 127 - x.numel())]).view(rows, 127)
    q = A.Fp8.empty(rows, 128, fmt)
    A.k_quant_fp8(m.to(DEV), q)
    assert (bytes_of(q.scale) == 127).all()
    assert torch.equal(bytes_of(q.data), bytes_of(m.to(DT[fmt])))


# ---- norm ------------------------------------------------------------------------------------------
NORM_SIZES = [(1, 1), (1, 4096), (3, 7), (5, 128), (9, 896), (33, 1000), (4, 1024), (2, 1032), (17, 4104), (3, 9999), (2, 16384), (600, 64)]


def norm_case(rows, d, dtype, seed, zeros=True):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, d, generator=g) * torch.exp(torch.randn(rows, 1, generator=g))).to(TYPES[dtype])
    r = torch.randn(rows, d, generator=g)
    gain = 1 + 0.2 * torch.randn(d, generator=g)
    if zeros and rows > 2:
        x[1] = 0
        r[1] = 0
    return x, r, gain


# on either side of where the kernels change, and rows that end in each place of a run
NORM_BORDERS = [(5, d) for d in (2, 4, 5, 6, 511, 512, 513, 1022, 1025, 2047, 2048, 2049, 4095, 4098, 8191, 8192, 8193, 12289, 16381, 16383)]


@pytest.mark.parametrize("rows,d", NORM_SIZES + NORM_BORDERS)
@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("dtype,add", [("f32", True), ("bf16", True), ("bf16", False), ("f32", False)])
def test_norm_forward(rows, d, norm, dtype, add):
    fmt = "e4m3" if (rows + d) % 2 else "e5m2"
    x, r, gain = norm_case(rows, d, dtype, rows * d)
    eps = 1e-5
    total = torch.empty(rows, d, device=DEV) if add else None
    y, rstd = torch.empty(rows, d, dtype=torch.bfloat16, device=DEV), torch.empty(rows, device=DEV)
    q, dq, sq = fp8_in_canvas(rows, d, fmt, 1)
    A.k_norm_fwd(x.to(DEV), gain.to(DEV), resid=r.to(DEV) if add else None, total=total, y=y, q=q, rstd=rstd, norm=norm, eps=eps)
    t = x.float() + r if add else x.float()
    if add:
        assert torch.equal(total.cpu(), t)
    want, want_r = norm_forward(t, gain, eps, norm)
    # A sum of d terms takes at most log2(64) + d / 64 + 16 roundings on its way to the total, each of half a step of at most the sum of magnitudes; the mean's
    # error enters a centred element absolutely.  Then four products and a root.
    n = 24 + d / 64
    size = t.double().abs().amax(1) * want_r * n * U if norm == "layer" else torch.zeros(rows, dtype=torch.float64)
    err = (want.abs() * (n + 8) * U) + (size[:, None] * gain.double().abs() * 2)
    # the mean's error against the spread of the row, as it enters rstd
    assert ((rstd.cpu().double() - want_r).abs() <= want_r * ((n + 8) * U + 2 * size)).all()
    err = err + want.abs() * 2 * size[:, None]
    assert ((y.cpu().double() - want).abs() <= err + (want.abs() + err) * 2.0 ** -8).all()
    # 8 bits: the block's scale is that of its largest magnitude, unless that is within the error of a border; then the element is off by half a step of it
    want_s = quantise(want, 1, fmt)[1].int()
    got_s = bytes_of(q.scale).int()
    low, high = quantise((want.abs() - err).clamp(min=0), 1, fmt)[1].int(), quantise(want.abs() + err, 1, fmt)[1].int()
    assert (((got_s >= low) & (got_s <= high)) | (got_s == want_s)).all()
    step = torch.maximum((want.abs() + err) * STEP[fmt], LEAST[fmt] * expand(torch.pow(2.0, got_s.double() - 127), 1, rows, d))
    assert ((wide(q) - want).abs() <= err + step).all()
    assert untouched(dq, rows, d) and untouched(sq, *want_s.shape)
    # each output alone, the sum in place of what was added, gives the same bits
    y2, rstd2, r2 = torch.empty_like(y), torch.empty_like(rstd), r.to(DEV)
    A.k_norm_fwd(x.to(DEV), gain.to(DEV), resid=r2 if add else None, total=r2 if add else None, y=y2, rstd=rstd2, norm=norm, eps=eps)
    q2 = A.Fp8.empty(rows, d, fmt)
    A.k_norm_fwd(x.to(DEV), gain.to(DEV), resid=r.to(DEV) if add else None, total=total, q=q2, rstd=rstd2, norm=norm, eps=eps)
    assert torch.equal(y2, y) and torch.equal(rstd2, rstd) and torch.equal(bytes_of(q2.data), bytes_of(q.data)) and torch.equal(bytes_of(q2.scale), bytes_of(q.scale))
    if add:
        assert torch.equal(r2, total)


@pytest.mark.parametrize("rows,d", NORM_SIZES + NORM_BORDERS + [(2500, 48), (0, 100), (1200, 9001)])
@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("dtype,add", [("f32", True), ("bf16", True), ("bf16", False)])
def test_norm_backward(rows, d, norm, dtype, add):
    total, ds_in, gain = norm_case(rows, d, "f32", rows * d + 1)
    dy = (torch.randn(rows, d, generator=torch.Generator().manual_seed(5)) * 0.1).to(TYPES[dtype])
    rstd = norm_forward(total, gain, 1e-5, norm)[1].float()
    ds, lp = torch.full((rows, d), 7.0, device=DEV), torch.empty(rows, d, dtype=torch.bfloat16, device=DEV)
    dgain = torch.full((d,), 7.0, device=DEV)
    ws = torch.full((max(A.k_norm_bwd_ws_bytes(rows, d), 16),), 0xFF, dtype=torch.uint8, device=DEV)
    A.k_norm_bwd(dy.to(DEV), total.to(DEV), rstd.to(DEV), gain.to(DEV), ds, dgain, ws, ds_in=ds_in.to(DEV) if add else None, ds_lp=lp, norm=norm)
    if rows == 0:
        assert (dgain == 0).all()
        return
    want, want_g = norm_backward(dy, total, rstd, gain, norm)
    r64, t64, h64 = rstd.double()[:, None], total.double(), (dy.double() * gain.double()).abs()
    # every term of a row's ds, with the roundings of the sums behind it (d / 64 + 24 of them) and of the products
    n = 32 + d / 64
    off = t64.abs().amax(1, keepdim=True) * r64 * n * U * (norm == "layer")     # of xh, by the mean
    xh = (t64 - t64.mean(1, keepdim=True) if norm == "layer" else t64).abs() * r64 + off
    err = r64 * n * U * (h64 + h64.mean(1, keepdim=True) + xh * (h64 * xh).mean(1, keepdim=True))
    err = err + r64 * off * ((h64 * xh).mean(1, keepdim=True) + xh * h64.mean(1, keepdim=True)) * 2
    if add:
        want, err = want + ds_in.double(), err + (want.abs() + ds_in.double().abs()) * U
    assert ((ds.cpu().double() - want).abs() <= err).all()
    assert torch.equal(lp, ds.bfloat16())
    # rows are added in at most rows / 512 + 600 steps
    assert ((dgain.cpu().double() - want_g).abs() <= ((dy.double().abs() * (xh * (n + rows / 512 + 600) * U + 2 * off)).sum(0))).all()
    again, ds2 = torch.empty_like(dgain), ds_in.to(DEV)
    A.k_norm_bwd(dy.to(DEV), total.to(DEV), rstd.to(DEV), gain.to(DEV), ds2, again, ws, ds_in=ds2 if add else None, norm=norm)      # in place
    assert torch.equal(again, dgain) and torch.equal(ds2, ds)


@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_norm_gradient_against_differences(norm):
    """d/dt sum(w y(total + t v, gain + t u)) by central differences in 64 bits."""
    rows, d, eps = 6, 200, 1e-5
    total, w, gain = norm_case(rows, d, "f32", 3, zeros=False)
    w = w * 0.1
    rstd = norm_forward(total, gain, eps, norm)[1].float()
    ds, dgain = torch.empty(rows, d, device=DEV), torch.empty(d, device=DEV)
    ws = torch.empty(A.k_norm_bwd_ws_bytes(rows, d), dtype=torch.uint8, device=DEV)
    A.k_norm_bwd(w.to(DEV), total.to(DEV), rstd.to(DEV), gain.to(DEV), ds, dgain, ws, norm=norm)
    g = torch.Generator().manual_seed(1)
    for _ in range(5):
        v, u = torch.randn(rows, d, generator=g).double(), torch.randn(d, generator=g).double()
        f = lambda t: float((w.double() * norm_forward(total.double() + t * v, gain.double() + t * u, eps, norm)[0]).sum())  # noqa: E731
        t = 1e-4
        num = (8 * (f(t) - f(-t)) - (f(2 * t) - f(-2 * t))) / (12 * t)     # error of the order t^4
        got = float((ds.cpu().double() * v).sum() + (dgain.cpu().double() * u).sum())
        size = float((ds.cpu().double() * v).abs().sum() + (dgain.cpu().double() * u).abs().sum())
        assert abs(num - got) <= 40 * U * size + 1e-9 * size


def test_norm_of_more_rows_than_a_launch_has():
    """The last rows, which a second launch has, and the first: as in a call of their own."""
    rows, d = (1 << 21) + 37, 24
    x = torch.randn(rows, d, device=DEV, generator=torch.Generator(DEV).manual_seed(1)).bfloat16()
    r, gain = torch.randn(rows, d, device=DEV, generator=torch.Generator(DEV).manual_seed(2)), torch.rand(d, device=DEV)

    def run(x, r):
        n = len(x)
        out = dict(total=torch.empty(n, d, device=DEV), y=torch.empty(n, d, dtype=torch.bfloat16, device=DEV), rstd=torch.empty(n, device=DEV))
        q = A.Fp8.empty(n, d)
        A.k_norm_fwd(x, gain, resid=r, q=q, norm="layer", **out)
        return [out["total"], out["y"], out["rstd"], q.data.view(torch.uint8), q.scale.view(torch.uint8)]

    every = run(x, r)
    for at in (0, (1 << 21) - 100, rows - 300):
        for a, b in zip(every, run(x[at:at + 300].contiguous(), r[at:at + 300].contiguous())):
            assert torch.equal(a[at:at + 300], b)


def test_norm_passes_on_what_is_not_finite():
    x, r, gain = norm_case(8, 300, "f32", 0)
    x[2, 5], x[4, 7] = float("inf"), float("nan")
    total, y, rstd = torch.empty(8, 300, device=DEV), torch.empty(8, 300, dtype=torch.bfloat16, device=DEV), torch.empty(8, device=DEV)
    q = A.Fp8.empty(8, 300, "e4m3")
    A.k_norm_fwd(x.to(DEV), gain.to(DEV), resid=r.to(DEV), total=total, y=y, q=q, rstd=rstd)
    v = wide(q)
    ok = torch.tensor([i not in (2, 4) for i in range(8)])
    assert torch.isfinite(v[ok]).all() and torch.isnan(v[2, 5]) and torch.isnan(v[4]).all() and (v[2, :5] == 0).all()


# ---- products --------------------------------------------------------------------------------------
def int_operand(rows, cols, fmt, block_rows, seed, most):
    """Whole numbers up to `most` under scales of 1/2, 1 or 2, in a canvas of NaN bytes."""
    g = torch.Generator().manual_seed(seed)
    f, data, scale = fp8_in_canvas(rows, cols, fmt, block_rows, extra=seed % 2)
    data.fill_(0x7F)       # NaN in both formats
    scale.fill_(0xFF)      # NaN
    v = torch.randint(-most, most + 1, (rows, cols), generator=g).float()
    f.data.copy_(v.to(DT[fmt]).to(DEV))
    f.scale.view(torch.uint8).copy_(torch.randint(126, 129, tuple(f.scale.shape), generator=g).to(torch.uint8).to(DEV))
    return f


GEMM_SIZES = [(1, 1, 1), (1, 64, 128), (5, 300, 896), (64, 64, 64), (65, 63, 130), (128, 128, 128), (100, 257, 15), (33, 129, 1000), (256, 256, 512), (257, 511, 385),
              (513, 100, 2049), (300, 1000, 48), (1024, 512, 256), (640, 896, 640), (16, 4096, 1024), (31, 2000, 4097), (4, 8, 20000), (1500, 40, 3000)]


@pytest.mark.parametrize("M,N,K", GEMM_SIZES)
@pytest.mark.parametrize("fa,fb,ra,rb", [("e4m3", "e4m3", 1, 128), ("e5m2", "e4m3", 1, 128), ("e4m3", "e5m2", 1, 1), ("e5m2", "e5m2", 128, 1)])
@pytest.mark.parametrize("with_ws", [False, True])
def test_product_of_whole_numbers_is_exact(M, N, K, fa, fb, ra, rb, with_ws):
    """Multiples of 1/4 up to 4 * 4 * 4 = 64, K of them: exact in fp32 while K * 64 * 4 < 2^24, so every order of sums gives the same."""
    assert K * 64 * 4 < 2 ** 24
    a, b = int_operand(M, K, fa, ra, 1, 4), int_operand(N, K, fb, rb, 2, 4)
    ws = torch.full((max(A.k_gemm_fp8_ws_bytes(M, N, K), 256),), 0xFF, dtype=torch.uint8, device=DEV) if with_ws else None
    want = wide(a) @ wide(b).t()
    big = torch.full((M + 2, N + 3), 7.0, device=DEV)
    c = big[1:M + 1, 1:N + 1]
    A.k_gemm_fp8(a, b, c, ws=ws)
    assert torch.equal(c.cpu().double(), want)
    outside = big.cpu().clone()
    outside[1:M + 1, 1:N + 1] = 7.0
    assert (outside == 7.0).all()
    # bf16 is that, rounded once; with something added (multiples of 1/4 too), also in place
    cb = torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
    A.k_gemm_fp8(a, b, cb, ws=ws)
    assert torch.equal(cb.cpu(), want.float().bfloat16())
    r = torch.randint(-100, 100, (M, N), generator=torch.Generator().manual_seed(3)).float() / 4
    rc = r.to(DEV)
    A.k_gemm_fp8(a, b, cb, resid=rc, ws=ws)
    assert torch.equal(cb.cpu(), (want + r.double()).float().bfloat16())
    A.k_gemm_fp8(a, b, rc, resid=rc, ws=ws)
    assert torch.equal(rc.cpu().double(), want + r.double())


VARIANT_SIZES = [(1, 1, 1), (65, 63, 130), (100, 257, 15), (257, 511, 385), (513, 100, 2049), (300, 1000, 48), (31, 2000, 4097), (1500, 40, 3000), (640, 896, 640), (1100, 2100, 1500), (128, 64, 128), (384, 320, 256), (896, 448, 100), (129, 64, 300), (256, 65, 300)]


@pytest.mark.parametrize("tile", [256, 128, 64])
@pytest.mark.parametrize("shares", [1, 2, 3, 5])
def test_every_kernel_takes_every_size(tile, shares):
    try:
        for i, (M, N, K) in enumerate(VARIANT_SIZES):
            fa, fb, ra, rb = [("e4m3", "e4m3", 1, 128), ("e5m2", "e4m3", 1, 1), ("e4m3", "e5m2", 128, 1)][(i + shares) % 3]
            a, b = int_operand(M, K, fa, ra, 1, 4), int_operand(N, K, fb, rb, 2, 4)
            want = wide(a) @ wide(b).t()
            r = torch.randint(-100, 100, (M, N), generator=torch.Generator().manual_seed(3)).float() / 4
            A.set_gemm_fp8(tile, shares)
            ws = torch.full((shares * M * (N + 3) * 4 + 256,), 0xFF, dtype=torch.uint8, device=DEV)
            # aligned rows, and rows at odd addresses, inside a larger matrix; with and without something added
            for pad in (-N % 16 + 16, 1):
                for dt in (torch.float32, torch.bfloat16):
                    for add in (None, r):
                        big = torch.full((M + 2, N + pad), 7.0, dtype=dt, device=DEV)
                        c = big[1:M + 1, :N]
                        A.k_gemm_fp8(a, b, c, resid=add.to(DEV) if add is not None else None, ws=ws)
                        assert torch.equal(c.cpu(), (want + (add.double() if add is not None else 0)).float().to(dt)), (M, N, K, pad, dt, add is None)
                        big[1:M + 1, :N] = 7.0
                        assert (big == 7.0).all()
    finally:
        A.set_gemm_fp8(0)


def test_a_small_workspace_means_fewer_shares():
    M, N, K = 64, 512, 8192
    tile, shares = A.gemm_fp8_route(M, N, K)
    assert shares > 1 and A.gemm_fp8_route(M, N, K, ws_bytes=0)[1] == 1
    a, b = int_operand(M, K, "e4m3", 1, 1, 4), int_operand(N, K, "e4m3", 128, 2, 4)
    want = wide(a) @ wide(b).t()
    c = torch.empty(M, N, device=DEV)
    for size in (0, 256, M * N * 4 * 2, A.k_gemm_fp8_ws_bytes(M, N, K)):
        ws = torch.full((size + 512,), 0x55, dtype=torch.uint8, device=DEV)
        c.zero_()
        A.k_gemm_fp8(a, b, c, ws=ws[:size] if size else None)
        assert torch.equal(c.cpu().double(), want) and (ws[size:] == 0x55).all()


@pytest.mark.parametrize("M,N,K", [(70, 80, 300), (300, 257, 300)])
def test_product_with_the_least_scale(M, N, K):
    """2^-127, which is no normal fp32 number: the elements of A are 2^-125 to 2^-124 there."""
    a, b = int_operand(M, K, "e4m3", 1, 5, 4), int_operand(N, K, "e4m3", 1, 6, 4)
    a.data.copy_((4 + 4 * (torch.arange(K) % 2)).float().to(DT["e4m3"]).to(DEV).expand(M, K))
    a.scale.view(torch.uint8).fill_(0)
    b.scale.view(torch.uint8).fill_(127 + 100)
    want = wide(a) @ wide(b).t()
    c, h = torch.empty(M, N, device=DEV), torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
    A.k_gemm_fp8(a, b, c)
    assert torch.equal(c.cpu().double(), want)
    A.k_gemm_fp8(a, b, h)
    assert torch.equal(h.cpu(), want.float().bfloat16())


@pytest.mark.parametrize("M,N,K", [(200, 300, 1000), (256, 512, 4096), (3, 700, 15315), (1000, 900, 129)])
@pytest.mark.parametrize("fa,fb", [("e4m3", "e4m3"), ("e5m2", "e4m3")])
def test_product_of_quantised_values(M, N, K, fa, fb):
    g = torch.Generator().manual_seed(M)
    x = torch.randn(M, K, generator=g) * torch.exp(2 * torch.randn(M, 1, generator=g))
    w = torch.randn(N, K, generator=g) * 0.02
    a, b = A.Fp8.empty(M, K, fa), A.Fp8.empty(N, K, fb, 128)
    A.k_quant_fp8(x.to(DEV), a)
    A.k_quant_fp8(w.to(DEV), b)
    ws = torch.empty(max(A.k_gemm_fp8_ws_bytes(M, N, K), 256), dtype=torch.uint8, device=DEV)
    c = torch.empty(M, N, device=DEV)
    A.k_gemm_fp8(a, b, c, ws=ws)
    wa, wb = wide(a), wide(b)
    # every one of K additions rounds or cuts at most one step of the sum of magnitudes
    assert ((c.cpu().double() - wa @ wb.t()).abs() <= (K + 8) * 2 * U * (wa.abs() @ wb.abs().t())).all()
    # and far nearer than that in the mean: sums of random sign
    want = wa @ wb.t()
    assert float((c.cpu().double() - want).norm() / want.norm()) < 1e-5
    again = torch.empty_like(c)
    A.k_gemm_fp8(a, b, again, ws=ws)
    assert torch.equal(again, c)
    # bf16: half a step of it, and of each product up to 2^-13 of the largest of its 8 neighbours: at most 7 of 8 of them, so 7 2^-13 of the sum of magnitudes
    h = torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
    A.k_gemm_fp8(a, b, h, ws=ws)
    assert ((h.cpu().double() - want).abs() <= want.abs() * 2.0 ** -8 + 7 * 2.0 ** -13 * (wa.abs() @ wb.abs().t()) * 1.01).all()
    assert float((h.cpu().double() - want).norm() / want.norm()) < 2.0 ** -9


def test_product_with_extreme_scales():
    """Scales from 2^-120 to 2^120 whose products are in range."""
    M, N, K = 70, 80, 300
    a, b = int_operand(M, K, "e4m3", 1, 5, 4), int_operand(N, K, "e4m3", 1, 6, 4)
    a.scale.view(torch.uint8).copy_((torch.arange(M) % 2 * 200 + 20).to(torch.uint8)[:, None].expand(M, 3).to(DEV))
    b.scale.view(torch.uint8).fill_(130)
    c = torch.empty(M, N, device=DEV)
    A.k_gemm_fp8(a, b, c)
    assert torch.equal(c.cpu().double(), wide(a) @ wide(b).t())


def test_product_passes_on_what_is_not_finite():
    M, N, K = 130, 140, 200
    a, b = int_operand(M, K, "e5m2", 1, 5, 4), int_operand(N, K, "e4m3", 1, 6, 4)
    a.data.view(torch.uint8)[3, 199] = 0x7C        # inf
    b.data.view(torch.uint8)[5, 0] = 0x7F          # NaN
    c = torch.empty(M, N, device=DEV)
    A.k_gemm_fp8(a, b, c)
    got, want = c.cpu().double(), wide(a) @ wide(b).t()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~torch.isnan(want)], want[~torch.isnan(want)])


def test_product_over_nothing():
    r = torch.randn(5, 9, device=DEV)
    a, b = A.Fp8.empty(5, 0), A.Fp8.empty(9, 0)
    c = torch.full((5, 9), 7.0, device=DEV)
    A.k_gemm_fp8(a, b, c)
    assert (c == 0).all()
    A.k_gemm_fp8(a, b, c, resid=r)
    assert torch.equal(c, r)


# ---- together ---------------------------------------------------------------------------------------
def layer_step(s):
    """One training step of y = norm(x + r) W^T in 8 bits, from the gradient dz of its output to the updated weights."""
    A.k_norm_fwd(s["x"], s["gain"], resid=s["r"], total=s["total"], y=s["y"], q=s["q"], rstd=s["rstd"], stream=s["stream"])
    A.k_quant_fp8(s["w"], s["wq"], s["wqt"], stream=s["stream"])
    A.k_gemm_fp8(s["q"], s["wq"], s["z"], ws=s["ws"], stream=s["stream"])
    A.k_quant_fp8(s["dz"], s["dq"], s["dqt"], stream=s["stream"])
    A.k_gemm_fp8(s["dq"], s["wqt"], s["dy"], ws=s["ws"], stream=s["stream"])
    A.k_quant_fp8(s["y"], None, s["yt"], stream=s["stream"])
    A.k_gemm_fp8(s["dqt"], s["yt"], s["dw"], ws=s["ws"], stream=s["stream"])
    A.k_norm_bwd(s["dy"], s["total"], s["rstd"], s["gain"], s["ds"], s["dgain"], s["ws"], ds_in=s["r"], ds_lp=s["lp"], stream=s["stream"])
    A.k_grad_norm([s["dw"], s["dgain"]], s["norm"], s["ws"], stream=s["stream"])
    A.k_adamw_clip(s["w"], s["dw"], s["m"], s["v"], s["w16"], s["w"].numel(), 1, 1e-3, s["norm"], 0.5, stream=s["stream"])


def layer_state(T, d, n, seed, stream=None):
    g = torch.Generator().manual_seed(seed)
    f = lambda *shape: torch.zeros(*shape, device=DEV)  # noqa: E731
    h = lambda *shape: torch.zeros(*shape, dtype=torch.bfloat16, device=DEV)  # noqa: E731
    F = A.Fp8.empty
    s = dict(x=torch.randn(T, d, generator=g).bfloat16().to(DEV), r=torch.randn(T, d, generator=g).to(DEV), gain=(1 + 0.1 * torch.randn(d, generator=g)).to(DEV), total=f(T, d), y=h(T, d),
             q=F(T, d), rstd=f(T), w=(0.02 * torch.randn(n, d, generator=g)).to(DEV), wq=F(n, d, "e4m3", 128), wqt=F(d, n, "e4m3", 128), z=h(T, n),
             dz=(0.1 * torch.randn(T, n, generator=g)).bfloat16().to(DEV), dq=F(T, n, "e5m2"), dqt=F(n, T, "e5m2"), dy=f(T, d), yt=F(d, T), dw=f(n, d), ds=f(T, d), dgain=f(d), lp=h(T, d),
             norm=f(1), m=f(n, d), v=f(n, d), w16=h(n, d), stream=stream)
    need = max(A.k_norm_bwd_ws_bytes(T, d), A.k_grad_norm_ws_bytes([s["dw"], s["dgain"]]), *(A.k_gemm_fp8_ws_bytes(*mnk) for mnk in ((T, n, d), (T, d, n), (n, d, T))))
    s["ws"] = torch.empty(need + 256, dtype=torch.uint8, device=DEV)
    return s


@pytest.mark.parametrize("T,d,n", [(96, 128, 256), (333, 200, 520), (1, 64, 64)])
def test_layer_step_against_its_formulas(T, d, n):
    s = layer_state(T, d, n, 11)
    w0 = s["w"].cpu().double()
    layer_step(s)
    c = {k: v.cpu() for k, v in s.items() if isinstance(v, torch.Tensor)}
    y64, rstd64 = norm_forward(c["x"].float() + c["r"], c["gain"], 1e-5, "rms")
    # what 8 bits leave of a value is within half a step of it; a product of two is off by the sum, and a sum of K of them in the mean by that over its terms' 2-norm
    z64 = y64 @ w0.t()
    terms = lambda p, q: torch.sqrt((p * p) @ (q * q).t())  # noqa: E731
    near = lambda got, want, size, e: float(((got.double() - want).abs() / (6 * e * size + 1e-9)).max()) < 1  # noqa: E731
    assert near(c["z"], z64, terms(y64, w0) + z64.abs() * 2.0 ** -4, 2.0 ** -4 * 1.5)
    dz = c["dz"].double()
    assert near(c["dy"], dz @ w0, terms(dz, w0.t()), 2.0 ** -3 * 1.2)
    dw64 = dz.t() @ y64
    assert near(c["dw"], dw64, terms(dz.t(), y64.t()), 2.0 ** -3 * 1.2)
    # from here on from what the products left, in fp32
    ds, dgain = norm_backward(c["dy"], c["total"], c["rstd"], c["gain"], "rms")
    assert float((c["ds"].double() - ds - c["r"].double()).norm() / ds.norm()) < 1e-5 and float((c["dgain"].double() - dgain).norm() / dgain.norm()) < 1e-5
    norm = torch.sqrt((c["dw"].double() ** 2).sum() + (c["dgain"].double() ** 2).sum())
    assert abs(float(c["norm"]) - float(norm)) <= U * 1.01 * float(norm)
    g = c["dw"].double() * min(1.0, 0.5 / float(norm))
    m, v = 0.1 * g, 0.001 * g * g
    w = w0 - 1e-3 * ((m / 0.1) / (torch.sqrt(v / 0.001) + 1e-8) + 0.1 * w0)
    assert float((c["m"].double() - m).norm() / m.norm()) < 1e-6 and float((c["w"].double() - w).norm() / (w - w0).norm()) < 1e-5
    assert torch.equal(c["w16"], c["w"].bfloat16())


def test_layer_step_on_a_stream_and_replayed():
    """Launched on a stream of its own and as a graph, beside another step on another stream: the same bits, replay after replay."""
    T, d, n = 200, 256, 300
    want = layer_state(T, d, n, 3)
    want2 = layer_state(T, d, n, 4)
    weights = []
    for _ in range(4):
        layer_step(want)
        layer_step(want2)
        weights.append((want["w"].clone(), want2["w"].clone(), want["z"].clone(), want["norm"].clone()))
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    a, b = layer_state(T, d, n, 3, one), layer_state(T, d, n, 4, two)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=one):
        layer_step(a)
    for w1, w2, z, norm in weights:
        with torch.cuda.stream(one):
            graph.replay()
        layer_step(b)
        torch.cuda.synchronize()
        assert torch.equal(a["w"], w1) and torch.equal(b["w"], w2) and torch.equal(a["z"], z) and torch.equal(a["norm"], norm)
        (torch.randn(1000, device=DEV) @ torch.randn(1000, device=DEV)).item()
