"""Local steps that clip their gradient: each against the definition in 64 bits, whole runs against the oracle with a clipping AdamW."""
import numpy as np
import pytest
import torch

import als_inputs as I
import paper_2401_09135_amd as A
from oracle import lm, run
from oracle.optim import AdamW

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _stream(w):
    return lambda i: I.TokenStream(w["seed"], i, w["B"], w["S"], w["V"])


def _context(w, k=None, streams=None, steps=8):
    cfg = A.Config.from_workload(w, max_local_steps=steps)
    cfg.n_workers = w["k"] if k is None else k
    return A.Context(cfg, I.theta0(lm.param_layout(w), w["seed"]), n_streams=streams or cfg.n_workers)


def _tokens(w, i, n):
    return torch.from_numpy(np.ascontiguousarray(_stream(w)(i).take(n))).to("cuda:0")


def _rel(a, b):
    a, b = np.asarray(a, np.float64), np.asarray(b, np.float64)
    return float(np.linalg.norm(a - b) / max(np.linalg.norm(b), 1e-30))


@pytest.mark.parametrize("name,k", [("tiny", 1), ("tiny", 4), ("mini_f32", 3), ("mini_bf16", 1), ("mini_bf16", 4), ("ragged_bf16", 2), ("tiny_ln", 4)])
def test_a_clipped_step_is_its_definition(name, k):
    """From the state and the gradient that the library gives: the norm, and the update of every element.  Steps are launched or replayed."""
    w = I.workload(name)
    ctx = _context(w, k)
    tok = _tokens(w, 0, 4)
    lr, b1, b2, eps, wd = w["lr"], w["beta1"], w["beta2"], w["adam_eps"], w["wd"]
    decay = lm.n_decayed(w)
    worker = k - 1
    ctx.worker_local_steps(worker, tok[:1], lr)
    first = float(np.linalg.norm(ctx.get_vector("grad", worker).astype(np.float64)))
    for s, limit in ((1, 0.3 * first), (2, 0.01 * first), (3, 50 * first)):
        ctx.set_grad_clip(limit)
        old = {v: ctx.get_vector(v, worker).astype(np.float64) for v in ("worker_theta", "adam_m", "adam_v")}
        ctx.worker_local_steps(worker, tok[s:s + 1], lr)
        norm = float(ctx.get_grad_norms(worker, 1)[0])
        th, m, v, g = (ctx.get_vector(x, worker).astype(np.float64) for x in ("worker_theta", "adam_m", "adam_v", "grad"))
        want = float(np.linalg.norm(g))
        assert abs(norm - want) <= 1.001 * U * want + 1e-13 * want      # one rounding, and the sum's own in double
        x = g * min(1.0, limit / want)
        m64, v64, n = b1 * old["adam_m"] + (1 - b1) * x, b2 * old["adam_v"] + (1 - b2) * x * x, s + 1
        root = np.sqrt(v64 / (1 - b2 ** n)) + eps
        upd = m64 / (1 - b1 ** n) / root
        upd[:decay] += wd * old["worker_theta"][:decay]
        # the coefficient is off by 3 U (norm, limit, quotient), constants by U, every operation by U
        assert (np.abs(m - m64) <= 8 * U * (np.abs(old["adam_m"]) + np.abs(x))).all()
        assert (np.abs(v - v64) <= 12 * U * (old["adam_v"] + (1 - b2) * x * x) + 1e-44).all()
        size = (np.abs(old["adam_m"]) + np.abs(x)) / (1 - b1 ** n) / root + np.abs(upd)
        assert (np.abs(th - (old["worker_theta"] - lr * upd)) <= 4 * U * np.abs(old["worker_theta"]) + 40 * U * lr * size).all()
    ctx.close()


@pytest.mark.parametrize("name,k", [("tiny", 4), ("mini_bf16", 4)])
def test_replayed_clipped_steps_equal_launched_ones(name, k):
    """The setting changes between rounds, from off to on, to another norm, and off again: the same bits, norms among them, and more steps in a call than a state holds."""
    w = I.workload(name)
    out = []
    for launched in (False, True):
        ctx = _context(w, k, steps=70)
        seen = []
        assert A.replay_info(ctx) == (k, 0, "")
        for rnd, limit in enumerate((0.0, 0.5, 0.05, 0.0, 1e9)):
            ctx.set_grad_clip(limit)
            A.prof_enable(launched)
            try:
                for i in range(k):
                    n = 70 if rnd == 2 and i == 1 else 2 + (i + rnd) % 2
                    seen.append(ctx.worker_local_steps(i, _tokens(w, i, n), [1e-3 * (1 + rnd + s) for s in range(n)], want_losses=i == 0))
                    if limit:
                        seen.append(ctx.get_grad_norms(i, n))
                        assert (seen[-1] > 0).all()
                    else:
                        with pytest.raises(A.AlsError, match="norms are taken"):
                            ctx.get_grad_norms(i, n)
                    seen.append(ctx.worker_loss_grad(i, _tokens(w, i, 1)[0])[1])
                    if limit:
                        assert np.array_equal(ctx.get_grad_norms(i, n), seen[-2])     # a gradient alone takes no norm
                torch.cuda.synchronize()
            finally:
                A.prof_enable(False)
                A.prof_collect()
            ctx.outer_apply_dn(list(range(k)), restart=True)
        graphs, steps, why = A.replay_info(ctx)
        assert graphs == k and why == "" and (steps == 0) == launched
        seen += [ctx.get_vector(v) for v in ("theta", "momentum", "delta")]
        seen += [ctx.get_vector(v, i) for i in range(k) for v in ("worker_theta", "adam_m", "adam_v", "grad")]
        ctx.close()
        out.append(seen)
    for a, b in zip(*out):
        assert (a is None and b is None) or np.array_equal(a, b)


def test_without_clipping_nothing_changes():
    """A context where clipping was on and off again before its first step gives the bits of one that never heard of it."""
    w = I.workload("mini_bf16")
    out = []
    for touched in (False, True):
        ctx = _context(w)
        if touched:
            ctx.set_grad_clip(0.25)
            ctx.set_grad_clip(0)
        ctx.worker_local_steps(2, _tokens(w, 2, 5), w["lr"])
        out.append([ctx.get_vector(v, 2) for v in ("worker_theta", "adam_m", "adam_v", "grad")] + [ctx.get_losses(2, 5)])
        ctx.close()
    for a, b in zip(*out):
        assert np.array_equal(a, b)


@pytest.mark.parametrize("name,limit", [("tiny", 1.9), ("tiny_k1", 3.6), ("mini_bf16", 2.0), ("tiny_grace_c", 0.4)])
def test_clipped_run_matches_oracle(name, limit, monkeypatch):
    """Whole asynchronous runs with clipped local steps.  The bounds are those of runs without: a coefficient that is off by 3 U moves nothing that they see."""
    norms = []

    class Clipping(AdamW):
        def step(self, theta, grad, lr):
            norm = float(np.linalg.norm(grad.astype(np.float64)))
            norms.append(norm)
            return super().step(theta, grad if norm <= limit else grad * grad.dtype.type(limit / norm), lr)

    w = I.workload(name)
    theta0 = I.theta0(lm.param_layout(w), w["seed"])
    monkeypatch.setattr(run, "AdamW", Clipping)
    ref = run.run_async(w, theta0, _stream(w))
    got = A.run_async(w, theta0, _stream(w), grad_clip=limit)
    got["ctx"].close()
    bf = w["dtype"] == "bf16"
    assert got["steps"].tolist() == ref["steps"].tolist()
    for lg, lr_ in zip(got["losses"], ref["losses"]):
        np.testing.assert_allclose(lg, lr_, rtol=2e-3 if bf else 1e-5)
    seen = [x for n in got["grad_norms"] for x in n]
    assert len(seen) == len(norms) == sum(len(x) for x in ref["losses"]) and max(norms) > limit
    np.testing.assert_allclose(sorted(seen), sorted(norms), rtol=2e-2 if bf else 1e-4)
    assert _rel(got["theta"], ref["theta"]) < (5e-3 if bf else 1e-5)
    assert _rel(got["theta"] - theta0, ref["theta"] - theta0) < (0.1 if bf else 1e-4)


@pytest.mark.parametrize("k", [1, 4])
def test_refusals(k):
    w = I.workload("tiny")
    ctx = _context(w, k)
    for bad in (-1.0, float("nan"), float("inf"), 1e39, 1e-60):
        with pytest.raises(A.AlsError, match="max_norm"):
            ctx.set_grad_clip(bad)
    tok = _tokens(w, 0, 2)
    ctx.set_grad_clip(0.5)
    with pytest.raises(A.AlsError):
        ctx.get_grad_norms(0, 1)
    ctx.worker_local_steps(0, tok, w["lr"])
    assert ctx.get_grad_norms(0, 2).shape == (2,)
    for worker, n in ((0, 3), (k, 0), (-1, 0)):
        with pytest.raises(A.AlsError):
            ctx.get_grad_norms(worker, n)
    y = torch.zeros(4, device="cuda:0")
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(ctx.streams[0]):
        g.capture_begin(capture_error_mode="relaxed")
        with pytest.raises(A.AlsError, match="captured"):
            ctx.set_grad_clip(0.25)
        y += 1
        g.capture_end()
    g.replay()
    if k == 4:
        A.prof_enable(True)
        try:
            with pytest.raises(A.AlsError, match="measured"):
                ctx.set_grad_clip(0.25)
        finally:
            A.prof_enable(False)
            A.prof_collect()
    ctx.worker_local_steps(0, tok, w["lr"])
    assert (ctx.get_grad_norms(0, 2) > 0).all() and ctx.adam_steps(0) == 4
    ctx.close()
