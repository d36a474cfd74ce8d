"""What the operators for 8-bit layers and clipping refuse: checked before any work reaches the GPU, so these run without one."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2401_09135_amd as A
from paper_2401_09135_amd.binding import _Fp8Struct

lib = A.lib
P16 = 4096          # stands for an aligned device address; a refused call reads none
INVALID = -1


def f8(rows, cols, data=P16, scale=P16, ld=None, ld_scale=None, fmt=0, block_rows=1):
    up = lambda n, m: -(-n // m) * m
    return _Fp8Struct(data, scale, up(cols, 16) if ld is None else ld, up(-(-cols // 128), 4) if ld_scale is None else ld_scale, fmt, block_rows)


BAD_FP8 = [dict(ld=100), dict(ld=120), dict(ld_scale=0), dict(ld_scale=3), dict(data=0), dict(scale=0), dict(data=P16 + 8), dict(scale=P16 + 2), dict(fmt=2),
           dict(fmt=-1), dict(block_rows=64), dict(block_rows=0)]


def quant(x=P16, dtype=0, rows=10, cols=128, ldx=128, q=True, qt=False, **bad):
    a = C.byref(f8(rows, cols, **bad)) if q else None
    b = C.byref(f8(cols, rows, **bad)) if qt else None
    return lib.als_k_quant_fp8(x, dtype, rows, cols, ldx, a, b, None)


@pytest.mark.parametrize("bad", BAD_FP8)
@pytest.mark.parametrize("qt", [False, True])
def test_quant_refuses_bad_matrices(bad, qt):
    if qt and "ld" in bad:
        bad = dict(ld=bad["ld"] - 98)     # rows are 10 long there
    assert quant(q=not qt, qt=qt, **bad) == INVALID


@pytest.mark.parametrize("bad", [dict(x=None), dict(x=P16 + 2), dict(x=P16 + 1, dtype=1), dict(dtype=2), dict(rows=-1), dict(cols=-1, ldx=1), dict(ldx=127),
                                 dict(q=False)])
def test_quant_refuses_bad_arguments(bad):
    assert quant(**bad) == INVALID


@pytest.mark.parametrize("rows,cols", [(0, 128), (10, 0), (0, 0)])
def test_nothing_to_do_is_no_error(rows, cols):
    assert lib.als_k_quant_fp8(None, 0, rows, cols, cols, C.byref(f8(rows, cols, data=0, scale=0)), None, None) == 0
    assert lib.als_k_gemm_fp8(C.byref(f8(rows, 64, data=P16)), C.byref(f8(cols, 64)), None, cols, 0, None, 0, rows, cols, 64, None, 0, None) == 0


def norm_fwd(x=P16, dtype=0, resid=P16, gain=P16, total=P16, y=P16, q=None, rstd=P16, rows=4, d=256, eps=1e-5, kind=0):
    return lib.als_k_norm_fwd(x, dtype, resid, gain, total, y, q, rstd, rows, d, eps, kind, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(gain=None), dict(rstd=None), dict(total=None), dict(resid=None), dict(y=None), dict(dtype=3), dict(rows=-1),
                                 dict(d=0), dict(d=16385), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(kind=2), dict(x=P16 + 2), dict(y=P16 + 1),
                                 dict(q=C.byref(f8(4, 256, block_rows=128))), dict(q=C.byref(f8(4, 256, ld=128)))])
def test_norm_fwd_refuses(bad):
    assert norm_fwd(**bad) == INVALID


def norm_bwd(dy=P16, dtype=0, total=P16, rstd=P16, gain=P16, ds_in=None, ds=P16, lp=None, dgain=P16, rows=4, d=256, kind=0, ws=P16, ws_bytes=1 << 20):
    return lib.als_k_norm_bwd(dy, dtype, total, rstd, gain, ds_in, ds, lp, dgain, rows, d, kind, ws, ws_bytes, None)


@pytest.mark.parametrize("bad", [dict(dy=None), dict(total=None), dict(rstd=None), dict(gain=None), dict(ds=None), dict(dgain=None), dict(ws=None), dict(ws=P16 + 8),
                                 dict(ws_bytes=0), dict(dtype=2), dict(d=16385), dict(kind=7), dict(ds_in=P16 + 2), dict(lp=P16 + 1)])
def test_norm_bwd_refuses(bad):
    assert norm_bwd(**bad) == INVALID
    assert lib.als_k_norm_bwd_ws_bytes(4, 0) == 0


def gemm(a={}, b={}, c=P16, ldc=192, out=0, r=None, ldr=0, M=64, N=192, K=256, ws=None, ws_bytes=0):
    return lib.als_k_gemm_fp8(C.byref(f8(M, K, **a)), C.byref(f8(N, K, **b)), c, ldc, out, r, ldr, M, N, K, ws, ws_bytes, None)


@pytest.mark.parametrize("bad", BAD_FP8)
@pytest.mark.parametrize("side", ["a", "b"])
def test_gemm_refuses_bad_matrices(bad, side):
    assert gemm(**{side: bad}) == INVALID


@pytest.mark.parametrize("bad", [dict(c=None), dict(c=P16 + 2), dict(ldc=191), dict(out=2), dict(r=P16 + 64, ldr=191), dict(r=P16 + 2, ldr=192), dict(M=-1), dict(N=-1), dict(K=-1),
                                 dict(r=P16, ldr=192, out=1), dict(r=P16, ldr=256), dict(ws=P16 + 16, ws_bytes=1 << 20), dict(K=(1 << 30) + 1)])
def test_gemm_refuses_bad_arguments(bad):
    assert gemm(**bad) == INVALID


def clip(n=3, grads=(P16, 1 << 20, 1 << 21), outs=None, numel=(10, 20, 30), dtypes=(0, 1, 0), max_norm=1.0, norm=P16, ws=P16, ws_bytes=1 << 16, only_norm=False):
    outs = grads if outs is None else outs
    g, o = (C.c_void_p * 3)(*grads), (C.c_void_p * 3)(*outs)
    nu, dt = (C.c_int64 * 3)(*numel), (C.c_int32 * 3)(*dtypes)
    if only_norm:
        return lib.als_k_grad_norm(n, g, nu, dt, norm, ws, ws_bytes, None)
    return lib.als_k_grad_clip(n, g, o, nu, dt, max_norm, norm, ws, ws_bytes, None)


@pytest.mark.parametrize("bad", [dict(n=-1), dict(norm=None), dict(norm=P16 + 2), dict(numel=(10, -1, 30)), dict(dtypes=(0, 2, 0)), dict(grads=(None, 1 << 20, 1 << 21)),
                                 dict(grads=(P16 + 2, 1 << 20, 1 << 21)), dict(grads=(P16, (1 << 20) + 1, 1 << 21)), dict(ws=None), dict(ws=P16 + 8), dict(ws_bytes=8)])
@pytest.mark.parametrize("only_norm", [False, True])
def test_gradient_lists_are_checked(bad, only_norm):
    assert clip(only_norm=only_norm, **bad) == INVALID


@pytest.mark.parametrize("bad", [dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(max_norm=float("inf")), dict(max_norm=1e-60),
                                 dict(outs=(P16, 1 << 20, None)), dict(outs=(P16, 1 << 20, (1 << 21) + 2)),
                                 dict(outs=(P16, 1 << 20, 1 << 20)),                       # two outputs in one place
                                 dict(outs=(P16 + 4, 1 << 20, 1 << 21)),                   # an output over its own input, one element on
                                 dict(outs=(1 << 21, 1 << 20, 1 << 22)),                   # an output over another's input
                                 dict(grads=(P16, 1 << 20, P16))])                         # a tensor listed twice, in place
def test_clip_refuses(bad):
    assert clip(**bad) == INVALID


def test_clip_overlap_check_takes_what_is_apart():
    """Outputs that touch but do not overlap pass the check: the workspace, checked behind it, is what is refused here."""
    ok = dict(grads=(P16, P16 + 40, P16 + 80), outs=(1 << 20, (1 << 20) + 40, (1 << 20) + 80))
    assert clip(ws_bytes=0, **ok) == INVALID and b"workspace" in lib.als_last_error()


@pytest.mark.parametrize("bad", [dict(max_norm=0.0), dict(norm=None), dict(theta=P16 + 4), dict(grad=P16 + 8), dict(lp=P16 + 4), dict(step=0), dict(P=-1), dict(P_decay=-1)])
def test_adamw_clip_refuses(bad):
    a = dict(theta=P16, grad=P16, m=P16, v=P16, lp=P16, P=100, P_decay=50, step=1, norm=P16, max_norm=1.0)
    a.update(bad)
    assert lib.als_k_adamw_clip(a["theta"], a["grad"], a["m"], a["v"], a["lp"], a["P"], a["P_decay"], a["step"], 1e-3, 0.9, 0.999, 1e-8, 0.1, a["norm"],
                                a["max_norm"], None) == INVALID


def test_binding_refuses_tensors_of_the_host_and_of_other_types():
    x = torch.zeros(4, 128)
    q = torch.zeros(4, 128, dtype=torch.float8_e4m3fn)
    s = torch.zeros(4, 4, dtype=torch.uint8).view(torch.float8_e8m0fnu)[:, :1]
    with pytest.raises(A.AlsError, match="GPU"):
        A.Fp8(q, s)
    with pytest.raises(A.AlsError, match="scale"):
        A.Fp8(q, torch.zeros(4, 1))
    with pytest.raises(A.AlsError, match="block_rows"):
        A.Fp8(q, s, 2)
    with pytest.raises(A.AlsError, match="scale must be"):
        A.Fp8(q, s, 128)
    with pytest.raises(A.AlsError, match="GPU"):
        A.k_quant_fp8(x)
    with pytest.raises(A.AlsError, match="unit column stride"):
        A.k_quant_fp8(x.t())
    with pytest.raises(A.AlsError, match="GPU"):
        A.k_grad_norm([x], x[0, :1], x)


def test_product_kernels_by_size():
    """The choices that the rule's comment gives figures for, and what it asks for as a workspace."""
    for (M, N, K), want in {(896, 3584, 15315): (128, 1), (1024, 896, 3584): (64, 1), (2048, 2048, 2048): (128, 1), (16384, 3584, 896): (256, 1), (16384, 896, 896): (256, 1),
                            (5, 3584, 896): (64, 1), (1, 1, 1): (64, 1), (8192, 8192, 8192): (256, 1)}.items():
        assert A.gemm_fp8_route(M, N, K) == want, (M, N, K)
        # without a workspace nothing is split, whatever the size
        assert A.gemm_fp8_route(M, N, K, ws_bytes=0)[1] == 1
    assert A.gemm_fp8_route(896, 3584, 15315, 0) == (256, 4)
    tile, shares = A.gemm_fp8_route(1, 8192, 8192)
    assert tile == 64 and shares > 1
    rng = __import__("random").Random(0)
    for _ in range(300):
        M, N, K = (int(2 ** rng.uniform(0, b)) for b in (17, 15, 17))
        need = A.k_gemm_fp8_ws_bytes(M, N, K)
        for dt in (0, 1):
            tile, shares = A.gemm_fp8_route(M, N, K, dt)
            slices = -(-K // 128)
            assert tile in (64, 128, 256) and 1 <= shares <= max(1, slices // 2) and (shares == 1 or shares * M * (-(-N // 4) * 4) * 4 <= need <= 256 << 20)
            some = need // 2
            t2, s2 = A.gemm_fp8_route(M, N, K, dt, ws_bytes=some)
            assert s2 == 1 or s2 * M * (-(-N // 4) * 4) * 4 <= some
    assert A.k_gemm_fp8_ws_bytes(0, 5, 5) == 0 and A.k_gemm_fp8_ws_bytes(5, 5, 0) == 0


@pytest.mark.parametrize("tile,shares", [(32, 1), (256, 0), (64, 65), (0, -1)])
def test_product_hook_refuses(tile, shares):
    assert lib.als_k_set_gemm_fp8(tile, shares) == INVALID


@pytest.mark.parametrize("bad", [dict(ldc=(1 << 26) + 1), dict(r=P16 + 64, ldr=(1 << 26) + 1), dict(N=(1 << 20) + 1, ldc=1 << 21), dict(a=dict(ld=(1 << 23) + 16)), dict(b=dict(ld_scale=(1 << 23) + 4))])
def test_gemm_refuses_what_its_addresses_do_not_reach(bad):
    assert gemm(**bad) == INVALID


def test_clipping_of_local_steps_needs_a_context():
    out = np.zeros(1, dtype=np.float32)
    assert A.lib.als_set_grad_clip(None, 1.0) != 0 and b"null" in A.lib.als_last_error()
    assert A.lib.als_get_grad_norms(None, 0, out.ctypes.data, 1) != 0 and b"null" in A.lib.als_last_error()


def test_shares_of_many_tiles_are_numbered_or_not_taken():
    """A tile of a share has a number below 2^32 / tiles: forced shares beyond that are one."""
    A.set_gemm_fp8(64, 24)
    try:
        assert A.gemm_fp8_route(1 << 22, 64, 8192, ws_bytes=1 << 40) == (64, 1)
        assert A.gemm_fp8_route(1 << 16, 64, 8192, ws_bytes=1 << 40) == (64, 24)
    finally:
        A.set_gemm_fp8(0)
    with pytest.raises(A.AlsError):
        A.gemm_fp8_route((1 << 30) + 1, 64, 128, ws_bytes=0)


@pytest.mark.parametrize("rows,cols", [(1 << 30, 129), (129 << 12, 1 << 20)])
def test_quant_refuses_more_tiles_than_a_launch_has(rows, cols):
    f = _Fp8Struct(P16, P16, -(-cols // 16) * 16, -(-cols // 512) * 4, 0, 128)
    assert lib.als_k_quant_fp8(P16, 1, rows, cols, cols, C.byref(f), None, None) == INVALID


def test_norm_refuses_more_rows_and_other_shapes():
    assert norm_fwd(rows=(1 << 30) + 1) == INVALID and norm_bwd(rows=(1 << 30) + 1, ws_bytes=1 << 40) == INVALID
    assert lib.als_k_norm_bwd_ws_bytes((1 << 30) + 1, 8) == 0
    x, g = torch.zeros(2, 3, 4), torch.zeros(4)
    for call in (lambda: A.k_norm_fwd(x, g), lambda: A.k_norm_fwd(x[0], g, norm="batch"), lambda: A.k_norm_bwd(x, x, g, g, x, g, None),
                 lambda: A.k_norm_bwd(x[0], x, g, g, x, g, None, norm="batch")):
        with pytest.raises(A.AlsError):
            call()


def test_one_row_of_any_stride_is_a_matrix():
    """A single row's stride is never used, so that views of any are taken if the row may be read in pieces of 16 bytes."""
    buf = torch.zeros(4096, dtype=torch.uint8)
    ld, data = 100, buf[:1024].view(torch.float8_e4m3fn)
    one = torch.as_strided(data, (1, 40), (ld, 1))
    from paper_2401_09135_amd.binding import _rows_of
    assert _rows_of("x", one, 1, 40, 16)[1] == 48
    with pytest.raises(A.AlsError):
        _rows_of("x", torch.as_strided(data, (2, 40), (ld, 1)), 2, 40, 16)
    with pytest.raises(A.AlsError):
        _rows_of("x", torch.as_strided(data, (1, 40), (ld, 1), 4096 - 40), 1, 40, 16)
