"""An Fp8 stands for the memory it was made of: what of that can be changed, and what is refused."""
import pytest
import torch

import paper_2401_09135_amd as A


@pytest.mark.parametrize("name", ["data", "scale", "block_rows"])
def test_parts_cannot_be_replaced(name):
    f = A.Fp8.__new__(A.Fp8)
    with pytest.raises(AttributeError):
        setattr(f, name, torch.zeros(4, 128, dtype=torch.uint8))


@pytest.mark.parametrize("bad", [dict(format="e3m4"), dict(format=None), dict(block_rows=0), dict(block_rows=64), dict(block_rows=-1), dict(rows=-1), dict(cols=-1)])
def test_empty_refuses(bad):
    with pytest.raises(A.AlsError, match="Fp8"):
        A.Fp8.empty(**{"rows": 4, "cols": 128, "device": "cpu", **bad})


def test_empty_on_the_host_is_refused():
    with pytest.raises(A.AlsError, match="GPU"):
        A.Fp8.empty(4, 128, device="cpu")


@pytest.mark.gpu
def test_memory_that_moved_is_refused():
    """Its own calls, each of which would write or read what the tensors were: refused before a launch."""
    x = torch.randn(8, 256, device="cuda:0")
    q, w, c = A.Fp8.empty(8, 256), A.Fp8.empty(16, 256), torch.zeros(8, 16, device="cuda:0")
    A.k_quant_fp8(x, q)
    A.k_quant_fp8(torch.randn(16, 256, device="cuda:0"), w)
    A.k_gemm_fp8(q, w, c)
    for part in ("data", "scale"):
        f = A.Fp8.empty(8, 256)
        A.k_quant_fp8(x, f)
        t = getattr(f, part)
        t.set_(torch.empty_like(t))
        y, rstd = torch.zeros(8, 256, dtype=torch.bfloat16, device="cuda:0"), torch.zeros(8, device="cuda:0")
        for call in (lambda: A.k_quant_fp8(x, f), lambda: A.k_gemm_fp8(f, w, c), lambda: A.k_gemm_fp8(w, f, torch.zeros(16, 8, device="cuda:0")),
                     lambda: A.k_norm_fwd(x, x[0].contiguous(), y=y, q=f, rstd=rstd)):
            with pytest.raises(A.AlsError, match="memory"):
                call()
    e = A.Fp8.empty(0, 256)      # nothing to move, nothing to do
    A.k_quant_fp8(torch.empty(0, 256, device="cuda:0"), e)
