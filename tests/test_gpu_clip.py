"""The global gradient norm, clipping and AdamW behind it on the GPU, against their definitions in 64 bits."""
import math

import pytest
import torch

import paper_2401_09135_amd as A

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


def tensors(sizes, dtypes, seed, spread=1.0, gap=0):
    """Views of one buffer a type, one behind the other, so that most start at odd addresses."""
    g = torch.Generator().manual_seed(seed)
    out = []
    flat = {t: torch.empty(sum(s for s, k in zip(sizes, dtypes) if k is t) + gap * len(sizes) + 8, dtype=t, device=DEV) for t in set(dtypes)}
    at = {t: gap for t in flat}
    for s, t in zip(sizes, dtypes):
        v = flat[t][at[t]:at[t] + s]
        v.copy_((torch.randn(s, generator=g) * spread * math.exp(float(torch.randn(1, generator=g)))).to(t))
        out.append(v)
        at[t] += s + gap
    return out


def workspace(grads):
    return torch.full((max(A.k_grad_norm_ws_bytes(grads), 16),), 0xFF, dtype=torch.uint8, device=DEV)


def norm64(grads):
    return math.sqrt(sum(float((t.cpu().double() ** 2).sum()) for t in grads))


F, B = torch.float32, torch.bfloat16
LISTS = [([1], [F]), ([1], [B]), ([7], [F]), ([4096], [F]), ([4097], [B]), ([3, 0, 5, 1], [F, F, B, F]), ([0, 0], [F, B]), ([1000003], [F]), ([1 << 22, 17, 1 << 20], [F, B, B]),
         ([64] * 95 + [300], [F] * 96), ([5] * 97, [F] * 97), ([11, 900, 0] * 100, [F, B, F] * 100), ([200000] * 250, [B, F] * 125)]


@pytest.mark.parametrize("sizes,dtypes", LISTS)
@pytest.mark.parametrize("gap", [0, 1])
def test_norm_and_clipping(sizes, dtypes, gap):
    grads = tensors(sizes, dtypes, len(sizes), 0.1, gap)
    ws, norm = workspace(grads), torch.full((1,), -1.0, device=DEV)
    want = norm64(grads)
    A.k_grad_norm(grads, norm, ws)
    assert abs(norm.item() - want) <= U * 1.001 * want       # the only rounding is the last one
    kept = [t.clone() for t in grads]
    for max_norm in (0.37 * want + 1e-6, 2 * want + 1):
        outs = tensors(sizes, dtypes, 1, 1.0, 1 - gap)
        A.k_grad_clip(grads, outs, max_norm, norm, ws)
        assert abs(norm.item() - want) <= U * 1.001 * want and all(torch.equal(a, b) for a, b in zip(grads, kept))
        k = min(1.0, max_norm / want) if want else 1.0
        for o, t in zip(outs, kept):
            # the coefficient is one division of two rounded numbers, then a product and the type's rounding
            ref = t.cpu().double() * k
            assert ((o.cpu().double() - ref).abs() <= ref.abs() * (4 * U + HALF[t.dtype] * 1.01)).all()
            if k == 1.0:
                assert torch.equal(o, t)
        where = [t.clone() for t in grads]      # in place, among its neighbours
        A.k_grad_clip(where, where, max_norm, norm, ws)
        assert all(torch.equal(a, b) for a, b in zip(where, outs))
    if sum(sizes):
        A.k_grad_clip(grads, grads, 0.5 * want, norm, ws)       # views of one buffer in place
        ref = [t.cpu().double() * 0.5 for t in kept]
        assert all(((a.cpu().double() - b).abs() <= b.abs() * (4 * U + HALF[a.dtype] * 1.01)).all() for a, b in zip(grads, ref))


def test_norm_of_no_tensors_is_zero():
    norm = torch.full((1,), 5.0, device=DEV)
    A.k_grad_norm([], norm, workspace([]))
    assert norm.item() == 0.0


@pytest.mark.parametrize("value,count", [(1e30, 5000), (3e38, 1), (1e-30, 70000), (1e-44, 3000)])
def test_norm_of_extreme_values(value, count):
    """Squares that leave the range of fp32, at either end."""
    t = torch.full((count,), value, device=DEV)
    ws, norm = workspace([t]), torch.empty(1, device=DEV)
    out = torch.empty_like(t)
    want = float(t[0].cpu().double()) * math.sqrt(count)
    A.k_grad_clip([t], [out], want / 2, norm, ws)
    least = 2.0 ** -149
    assert abs(norm.item() - want) <= 1.01 * U * want + least
    assert abs(float(out[0].cpu().double()) - want / 2 / math.sqrt(count)) <= 4 * U * value + 2 * least * (1 + value / max(norm.item(), least))


def test_a_norm_that_is_not_finite_shows():
    for bad, coefficient in ((float("inf"), 0.0), (float("nan"), float("nan"))):
        t = torch.ones(100, device=DEV)
        t[50] = bad
        norm, out = torch.empty(1, device=DEV), torch.empty(100, device=DEV)
        A.k_grad_clip([t], [out], 1.0, norm, workspace([t]))
        assert not math.isfinite(norm.item()) and math.isnan(out[50].item())
        assert out[0].item() == coefficient or (math.isnan(coefficient) and torch.isnan(out).all())


@pytest.mark.parametrize("P", [1, 3, 4, 1000, 4099, 1 << 20])
@pytest.mark.parametrize("part", [0.0, 0.5, 1.0])
@pytest.mark.parametrize("factor", [0.25, 4.0])
def test_adamw_behind_clipping(P, part, factor):
    g = torch.Generator().manual_seed(P)
    r = lambda s: torch.randn(P, generator=g) * s  # noqa: E731
    th, gr, m, v = r(0.02), r(1e-3), r(1e-4), r(1e-4) ** 2
    decay, step = int(P * part), 3
    d = [t.to(DEV) for t in (th, gr, m, v)]
    lp, norm = torch.empty(P, dtype=torch.bfloat16, device=DEV), torch.empty(1, device=DEV)
    A.k_grad_norm([d[1]], norm, workspace([d[1]]))
    limit = factor * float((gr.double() ** 2).sum().sqrt())
    A.k_adamw_clip(d[0], d[1], d[2], d[3], lp, decay, step, 1e-3, norm, limit)
    x = gr.double() * min(factor, 1.0)
    m64, v64 = 0.9 * m.double() + 0.1 * x, 0.999 * v.double() + 0.001 * x * x
    upd = (m64 / (1 - 0.9 ** step)) / (torch.sqrt(v64 / (1 - 0.999 ** step)) + 1e-8)
    upd[:decay] += 0.1 * th.double()[:decay]
    want = th.double() - 1e-3 * upd
    # constants rounded to fp32 and a few roundings each
    assert ((d[2].cpu().double() - m64).abs() <= 8 * U * (m.double().abs() + x.abs())).all()
    assert ((d[3].cpu().double() - v64).abs() <= 8 * U * (v.double() + 0.001 * x * x)).all()
    assert ((d[0].cpu().double() - want).abs() <= 4 * U * th.double().abs() + 40 * U * 1e-3 * (upd.abs() + m.double().abs() / (torch.sqrt(v64 / (1 - 0.999 ** step)) + 1e-8) / 0.2)).all()
    assert torch.equal(lp, d[0].bfloat16()) and torch.equal(d[1].cpu(), gr)


def test_clipping_on_a_stream_and_replayed():
    grads = tensors([1000, 3, 70001], [F, B, F], 5)
    outs = [torch.empty_like(t) for t in grads]
    s = torch.cuda.Stream()
    ws, norm = workspace(grads), torch.empty(1, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        A.k_grad_clip(grads, outs, 1.0, norm, ws, stream=s)
    for i in range(3):
        for t in grads:
            t.mul_(1.5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        norm2, outs2 = torch.empty(1, device=DEV), [torch.empty_like(t) for t in grads]
        A.k_grad_clip(grads, outs2, 1.0, norm2, workspace(grads))
        torch.cuda.synchronize()
        assert torch.equal(norm, norm2) and all(torch.equal(a, b) for a, b in zip(outs, outs2))
