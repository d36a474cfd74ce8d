"""Clipping by a norm that fp32 does not hold, and how near the clipped gradients come."""
import math

import pytest
import torch

import paper_2401_09135_amd as A

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
F, B = torch.float32, torch.bfloat16
# lists that are clipped in two launches, by more partial sums than those take, and in more than one launch of each kernel
LISTS = [([5], [F]), ([3000, 7, 0, 129], [F, B, F, B]), ([3000001, 5], [F, B]), ([4000001], [B]), ([40] * 200, [F, B] * 100)]


def workspace(grads):
    return torch.full((max(A.k_grad_norm_ws_bytes(grads), 16),), 0xFF, dtype=torch.uint8, device=DEV)


def clip(grads, outs, max_norm):
    norm = torch.full((1,), -1.0, device=DEV)
    A.k_grad_clip(grads, outs, max_norm, norm, workspace(grads))
    return norm.item()


def check(outs, grads, k):
    """One rounding of the product, the type's own, and 64 bits before."""
    for o, t in zip(outs, grads):
        ref = t.cpu().double() * k
        half = U if t.dtype is F else U + 2.0 ** -8
        assert ((o.cpu().double() - ref).abs() <= ref.abs() * 1.01 * half + (2.0 ** -150 if t.dtype is F else 2.0 ** -134)).all()


@pytest.mark.parametrize("sizes,dtypes", LISTS)
@pytest.mark.parametrize("max_norm", [1.0, 1e38, 3e38])
def test_norm_beyond_fp32_of_finite_gradients(sizes, dtypes, max_norm):
    """3e38 each: the norm is infinite in fp32, and the gradients are clipped by what it is."""
    g = torch.Generator().manual_seed(1)
    grads = [(3e38 * (0.9 + 0.1 * torch.rand(s, generator=g)) * (torch.rand(s, generator=g) - 0.5).sign()).to(t).to(DEV) for s, t in zip(sizes, dtypes)]
    want = math.sqrt(sum(float((t.cpu().double() ** 2).sum()) for t in grads))
    assert want > 3.5e38
    outs = [torch.full_like(t, 7.0) for t in grads]
    assert clip(grads, outs, max_norm) == math.inf
    check(outs, grads, max_norm / want)
    assert clip(grads, grads, max_norm) == math.inf
    assert all(torch.equal(a, b) for a, b in zip(grads, outs))


@pytest.mark.parametrize("sizes,dtypes", LISTS)
def test_clipped_gradients_are_rounded_once(sizes, dtypes):
    g = torch.Generator().manual_seed(2)
    grads = [(torch.randn(s, generator=g) * 1e-3).to(t).to(DEV) for s, t in zip(sizes, dtypes)]
    want = math.sqrt(sum(float((t.cpu().double() ** 2).sum()) for t in grads))
    for factor in (0.37, 0.999999, 1e-9):
        outs = [torch.empty_like(t) for t in grads]
        assert abs(clip(grads, outs, factor * want) - want) <= 1.001 * U * want
        check(outs, grads, factor)
    # a norm that is the limit to the last bit, or below it, changes nothing
    outs = [torch.full_like(t, 7.0) for t in grads]
    clip(grads, outs, want * (1 + 1e-12))
    assert all(torch.equal(a, b) for a, b in zip(outs, grads))


@pytest.mark.parametrize("P", [4, 4099, 100000])
def test_a_limit_that_does_not_bind_changes_adamw_by_its_constants_alone(P):
    """1 - beta rounded from double behind a norm, and formed in fp32 without: of the gradient's share of v 1.3e-5, of m 2.4e-7."""
    g = torch.Generator().manual_seed(P)
    th, gr, m, v = torch.randn(P, generator=g), torch.randn(P, generator=g), 0.1 * torch.randn(P, generator=g), torch.rand(P, generator=g) * 1e-4
    plain, clipped = ([t.to(DEV) for t in (th, gr, m, v)] for _ in range(2))
    A.k_adamw(*plain, None, P // 2, 3, 1e-3)
    A.k_adamw_clip(*clipped, None, P // 2, 3, 1e-3, torch.ones(1, device=DEV), 2.0)
    f = lambda x: float(torch.tensor(x, dtype=F))  # noqa: E731
    more = [f(1 - b) - float(torch.tensor(1.0) - torch.tensor(b, dtype=F)) for b in (0.9, 0.999)]
    # 0.1 itself is rounded by 1.5e-9, 1.5e-8 of it, and the figure by 2e-9 of it
    assert abs(more[0] / 0.1 + 2.4e-7) < 1.5e-8 + 2e-9 and abs(more[1] / 0.001 - 1.29e-5) < 1e-7
    x = gr.double()
    for i, old, share, by in ((2, m.double().abs(), x.abs(), more[0] * x), (3, v.double(), 0.001 * x * x, more[1] * x * x)):
        # five roundings a side: two products of the gradient, one of what was there, the sum
        assert (clipped[i].cpu().double() - plain[i].cpu().double() - by).abs().le(10 * U * (old + share)).all()
    # m / sqrt(v) moves by at most the first and half of the second, and by some roundings
    moved = 1e-3 * (clipped[2].cpu().double().abs() / 0.271) / torch.sqrt(clipped[3].cpu().double() / 0.002997)
    assert (clipped[0].cpu().double() - plain[0].cpu().double()).abs().le(moved * (0.7e-5 + 30 * U) + 4 * U * (th.double().abs() + 1e-3)).all()
