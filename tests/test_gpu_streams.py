"""Calls without a stream run on torch's current one, behind what that stream still has to do; and on the tensors' own GPU."""
from types import SimpleNamespace

import pytest
import torch

import paper_2401_09135_amd as A

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rand(*shape, dtype=torch.float32, seed=0):
    return torch.randn(*shape, device=DEV, generator=torch.Generator(DEV).manual_seed(seed)).to(dtype)


def empty(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype, device=DEV)


def workspace(n):
    return torch.zeros(max(n, 256), dtype=torch.uint8, device=DEV)


def quant():
    x, q = rand(300, 500), A.Fp8.empty(300, 500)
    return [x], [q.data.view(torch.uint8), q.scale.view(torch.uint8)], lambda **k: A.k_quant_fp8(x, q, **k)


def norm_fwd():
    x, gain, y, rstd = rand(300, 500), rand(500, seed=1), empty(300, 500, dtype=torch.bfloat16), empty(300)
    return [x], [y, rstd], lambda **k: A.k_norm_fwd(x, gain, y=y, rstd=rstd, **k)


def norm_bwd():
    dy, total, gain, rstd, ds, dg = rand(300, 500), rand(300, 500, seed=1), rand(500, seed=2), empty(300) + 1, empty(300, 500), empty(500)
    ws = workspace(A.k_norm_bwd_ws_bytes(300, 500))
    return [dy, total], [ds, dg], lambda **k: A.k_norm_bwd(dy, total, rstd, gain, ds, dg, ws, **k)


def gemm_fp8():
    a, b, c, ws = A.Fp8.empty(64, 8192), A.Fp8.empty(512, 8192), empty(64, 512), workspace(A.k_gemm_fp8_ws_bytes(64, 512, 8192))
    A.k_quant_fp8(rand(64, 8192), a)
    A.k_quant_fp8(rand(512, 8192, seed=1), b)
    r = rand(64, 512)
    return [r], [c], lambda **k: A.k_gemm_fp8(a, b, c, resid=r, ws=ws, **k)


def grad_norm():
    g, n = [rand(3000), rand(77, dtype=torch.bfloat16)], empty(1)
    ws = workspace(A.k_grad_norm_ws_bytes(g))
    return g, [n], lambda **k: A.k_grad_norm(g, n, ws, **k)


def grad_clip():
    g, n, o = [rand(3000), rand(77, dtype=torch.bfloat16)], empty(1), [empty(3000), empty(77, dtype=torch.bfloat16)]
    ws = workspace(A.k_grad_norm_ws_bytes(g))
    return g, [n, *o], lambda **k: A.k_grad_clip(g, o, 0.5, n, ws, **k)


def adamw_clip():
    g, n = rand(4000), empty(1) + 5
    th, m, v = empty(4000), empty(4000), empty(4000)

    def call(**k):
        th.zero_(), m.zero_(), v.zero_()
        A.k_adamw_clip(th, g, m, v, None, 100, 1, 1e-3, n, 1.0, **k)
    return [g], [th, m, v], call


def adamw():
    g = rand(4000)
    th, m, v = empty(4000), empty(4000), empty(4000)

    def call(**k):
        th.zero_(), m.zero_(), v.zero_()
        A.k_adamw(th, g, m, v, None, 100, 1, 1e-3, **k)
    return [g], [th, m, v], call


def gemm():
    a, b, c = rand(200, 300), rand(300, 100, seed=1), empty(200, 100)
    return [a], [c], lambda **k: A.k_gemm(a, b, c, 200, 100, 300, **k)


def attention():
    qkv, o, lse = rand(2, 64, 3 * 128), empty(2, 64, 128), empty(2, 2, 64)
    return [qkv], [o, lse], lambda **k: A.k_attention_fwd(qkv, o, lse, 2, 64, 2, 64, **k)


OURS = [quant, norm_fwd, norm_bwd, gemm_fp8, grad_norm, grad_clip, adamw_clip]
CASES = OURS + [adamw, gemm, attention]


@pytest.mark.parametrize("case", CASES)
def test_a_call_waits_for_what_its_stream_does_before(case):
    inputs, outs, call = case()
    call()
    torch.cuda.synchronize()
    old = [t.clone() for t in outs]
    before = [t.clone() for t in inputs]
    fresh = [t * 1.75 for t in inputs]
    for s in (torch.cuda.Stream(), torch.cuda.Stream()):     # one of two is in another hardware queue than the null stream
        for t, f in zip(inputs, before):
            t.copy_(f)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            torch.cuda._sleep(20_000_000)
            for t, f in zip(inputs, fresh):
                t.copy_(f)
            call()
            got = [t.clone() for t in outs]
        s.synchronize()
        torch.cuda.synchronize()
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs)) and not all(torch.equal(a, b) for a, b in zip(got, old))


@pytest.mark.parametrize("case", CASES)
def test_a_call_is_captured_without_naming_the_stream(case):
    inputs, outs, call = case()
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in range(3):
        for t in inputs:
            t.mul_(1.25)
        for t in outs:
            t.fill_(0)
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for t in outs:
            t.fill_(0)
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs))


@pytest.mark.parametrize("case", OURS)
def test_a_stream_of_another_gpu_is_refused(case):
    _, outs, call = case()
    torch.cuda.synchronize()
    old = [t.clone() for t in outs]
    with pytest.raises(A.AlsError, match="stream"):
        call(stream=SimpleNamespace(cuda_stream=0, device_index=1))
    torch.cuda.synchronize()
    assert case is adamw_clip or all(torch.equal(a, b) for a, b in zip(outs, old))
