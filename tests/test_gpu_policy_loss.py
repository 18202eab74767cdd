"""echo_policy_loss against the formulas in 64 bits: both sides of every clip, caps, absent terms, rows that take no part, types and strides; the
gradient against differences of the loss."""
import numpy as np
import pytest
import torch

import learner_plain as plain
from test_gpu_token_logprobs import DT, ROUND, f64, make

pytestmark = pytest.mark.gpu

COEF = dict(clip_low=0.2, clip_high=0.3, ratio_cap=4.0, sampler_cap=2.0, kl_coef=0.05, entropy_coef=0.02)


@pytest.fixture(scope="module")
def learner():
    from paper_2602_02192_amd import learner as l
    return l


def inputs(x, targets, r, T):
    """Ratios well inside and outside every bound (never at one, where the slope jumps), advantages of both signs and zero."""
    want = plain.rows(f64(x), targets.cpu().numpy(), T)
    R = x.shape[0]
    lp = np.where(np.isfinite(want["logprobs"]), want["logprobs"], -3.0)
    log_ratio = r.choice(np.log([0.5, 0.9, 1.0, 1.1, 1.6, 3.0, 6.0]), R)
    a = dict(advantages=r.choice([-1.5, -0.3, 0.0, 0.4, 2.0], R), old_logprobs=lp - log_ratio, ref_logprobs=lp + r.normal(0, 0.4, R),
             weights=np.where(r.random(R) < 0.25, 0.0, r.random(R) + 0.1))
    a["sampler_logprobs"] = a["old_logprobs"] + r.choice([-1.0, -0.2, 0.3], R)
    return {k: torch.from_numpy(v.astype(np.float32)).cuda() for k, v in a.items()}, want


def check(got, x, targets, a, want, o, T, dtype):
    n = {k: f64(v) for k, v in a.items()}
    R = x.shape[0]
    w = n.get("weights", np.ones(R))
    tn = targets.cpu().numpy()
    live = (w != 0) & (tn >= 0) & (tn < x.shape[1])
    tol = plain.tolerance(f64(x), T)
    loss, g, h = (np.zeros(R) for _ in range(3))
    for t in np.flatnonzero(live):
        loss[t], g[t], h[t] = plain.token_loss(want["logprobs"][t], want["entropy"][t], n["advantages"][t], n["old_logprobs"][t], w[t],
                                               n["sampler_logprobs"][t] if "sampler_logprobs" in n else None, n["ref_logprobs"][t] if "ref_logprobs" in n else 0.0, o)
    want = dict(want, live=live)
    # a log-probability off by 2 tol moves ratio, importance weight and divergence by that share; each is a handful of roundings further
    ratio = np.exp(np.where(live, want["logprobs"] - n["old_logprobs"], 0.0))
    k = np.exp(np.abs(np.where(live, n["ref_logprobs"] - want["logprobs"], 0.0))) if "ref_logprobs" in n else 1.0
    sens = np.abs(w) * (o["sampler_cap"] * np.abs(n["advantages"]) * np.maximum(ratio, 1.0) + abs(o["kl_coef"]) * k + abs(o["entropy_coef"]) * (2 + want["entropy"])) if \
        "sampler_logprobs" in n else np.abs(w) * (np.abs(n["advantages"]) * np.maximum(ratio, 1.0) + abs(o["kl_coef"]) * k + abs(o["entropy_coef"]) * (2 + want["entropy"]))
    near = lambda a, b, t: (np.abs(f64(a) - b) <= t).all()  # noqa: E731
    assert near(got.logprobs, np.where(live, want["logprobs"], 0), 2 * tol)
    assert near(got.entropy, np.where(live, want["entropy"], 0), tol * (2 + want["entropy"]))
    assert near(got.loss, loss, sens * (2 * tol + 2.0 ** -20))
    if got.grad_logits is not None:
        d, size = plain.logit_gradient(want, tn, g, h, T)
        at_target = np.arange(x.shape[1]) == np.clip(tn, 0, x.shape[1] - 1)[:, None]
        off = (sens * (2 * tol + 2.0 ** -20))[:, None] * (want["p"] + at_target) / T
        bound = 4 * tol[:, None] * size + ROUND[dtype] * np.abs(d) + off + (2.0 ** -24 if dtype == "f16" else 1e-38)
        assert (np.abs(f64(got.grad_logits) - d) <= np.where(live[:, None], bound, 0)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,pad,offset,T", [(1, 1, 0, 0, 1.0), (60, 9, 1, 1, 0.8), (64, 1024, 0, 0, 1.0), (31, 1025, 7, 3, 1.0), (4, 32000, 0, 0, 1.2), (3, 33003, 5, 1, 1.0),
                                                     (2, 151936, 0, 0, 1.0), (5, 152005, 3, 0, 1.0), (1, 262147, 0, 1, 1.0), (700, 517, 0, 0, 1.0)])
def test_against_the_formulas(learner, dtype, rows, vocab, pad, offset, T):
    x, targets, r = make(rows, vocab, dtype, vocab + rows, pad, offset)
    a, want = inputs(x, targets, r, T)
    got = learner.policy_loss(x, targets, temperature=T, **a, **COEF)
    check(got, x, targets, a, want, COEF, T, dtype)
    alone = learner.policy_loss(x, targets, temperature=T, want_grad=False, **a, **COEF)
    assert alone.grad_logits is None
    np.testing.assert_allclose(f64(alone.loss), f64(got.loss), rtol=1e-4, atol=1e-5)
    wide = torch.full((rows, vocab + 3), 7.0, dtype=DT[dtype], device="cuda")
    again = learner.policy_loss(x, targets, temperature=T, grad_out=wide[:, :vocab], **a, **COEF)
    assert torch.equal(again.grad_logits, got.grad_logits) and (wide[:, vocab:] == 7.0).all() and torch.equal(again.loss, got.loss)
    place = learner.policy_loss(x, targets, temperature=T, grad_out=x, **a, **COEF)
    assert place.grad_logits.data_ptr() == x.data_ptr() and torch.equal(x, got.grad_logits) and torch.equal(place.loss, got.loss)


@pytest.mark.parametrize("dtype,rows,vocab", [("bf16", 175, 100003), ("bf16", 176, 100003), ("bf16", 257, 75001), ("f16", 176, 90113), ("f32", 95, 90001), ("f32", 96, 90001), ("f32", 257, 70001)])
def test_long_rows_whole_and_in_parts(learner, dtype, rows, vocab):
    """Row counts on both sides of where a row is cut; rows longer than what a workgroup keeps of them, with and without a place of their own for the gradient."""
    x, targets, r = make(rows, vocab, dtype, rows + vocab)
    a, want = inputs(x, targets, r, 1.0)
    got = learner.policy_loss(x, targets, **a, **COEF)
    check(got, x, targets, a, want, COEF, 1.0, dtype)
    place = learner.policy_loss(x, targets, grad_out=x, **a, **COEF)
    assert torch.equal(x, got.grad_logits) and torch.equal(place.loss, got.loss)


@pytest.mark.parametrize("dtype,vocab", [("bf16", 2000), ("bf16", 151936), ("f32", 40000)])
def test_absent_terms(learner, dtype, vocab):
    x, targets, r = make(40, vocab if vocab < 100000 else vocab, dtype, 8)
    x, targets = x[:12], targets[:12]
    a, want = inputs(x, targets, r, 1.0)
    for drop, o in ((("weights",), COEF), (("sampler_logprobs",), COEF), (("ref_logprobs",), dict(COEF, kl_coef=0.0)),
                    (("weights", "sampler_logprobs", "ref_logprobs"), dict(COEF, kl_coef=0.0, entropy_coef=0.0, ratio_cap=float("inf"), sampler_cap=float("inf")))):
        b = {k: v for k, v in a.items() if k not in drop}
        check(learner.policy_loss(x, targets, **b, **o), x, targets, b, want, o, 1.0, dtype)


@pytest.mark.parametrize("dtype,vocab", [("f32", 900), ("f32", 152003), ("bf16", 900), ("bf16", 152003)])
def test_rows_that_take_no_part_are_not_read(learner, dtype, vocab):
    x, targets, r = make(9, vocab, dtype, 12)
    a, want = inputs(x, targets, r, 1.0)
    a["weights"][:] = 1.0
    a["weights"][2] = 0.0
    for row, t in ((0, -1), (5, vocab), (8, -2 ** 31)):
        targets[row] = t
    for row in (0, 2, 5, 8):
        x[row] = float("nan")
        a["advantages"][row] = float("nan")
    x[4] = -float("inf")                      # takes part, without weight anywhere
    got = learner.policy_loss(x, targets, **a, **dict(COEF, kl_coef=0.0))
    for row in (0, 2, 5, 8):
        assert got.loss[row] == 0 and got.logprobs[row] == 0 and got.entropy[row] == 0 and (got.grad_logits[row] == 0).all()
    assert got.logprobs[4] == -np.inf and (got.grad_logits[4] == 0).all()
    for row in (1, 3, 6, 7):
        assert torch.isfinite(got.grad_logits[row]).all() and torch.isfinite(got.loss[row])
    x[3, 7] = float("nan")
    x[6, 1] = float("inf")
    got = learner.policy_loss(x, targets, **a, **COEF)
    for row in (3, 6):
        assert torch.isnan(got.loss[row]) and torch.isnan(got.grad_logits[row]).all()
    assert torch.isfinite(got.grad_logits[1]).all()


def test_entries_that_are_ruled_out(learner):
    for dtype, vocab in (("bf16", 152001), ("f16", 700), ("f32", 30001)):
        x, targets, r = make(6, vocab, dtype, 31, banned=0.97)
        x[torch.arange(6), targets.long()] = 0.5
        x[3] = torch.finfo(x.dtype).min
        a, want = inputs(x, targets, r, 1.0)
        got = learner.policy_loss(x, targets, **a, **COEF)
        check(got, x, targets, a, want, COEF, 1.0, dtype)
        assert (got.grad_logits[:3][x[:3] == -np.inf] == 0).all()


def test_gradient_against_differences(learner):
    """Central differences of the loss: values good to the tolerance of a log-probability times at most 10, third derivative below 60."""
    x, targets, r = make(40, 5, "f32", 78, spread=1.0)
    a, want = inputs(x, targets, r, 0.8)
    grad = f64(learner.policy_loss(x, targets, temperature=0.8, **a, **COEF).grad_logits)
    step = 2.0 ** -7
    slope = np.zeros((40, 5))
    for j in range(5):
        v = []
        for s in (step, -step):
            y = x.clone()
            y[:, j] += s
            v.append(f64(learner.policy_loss(y, targets, temperature=0.8, want_grad=False, **a, **COEF).loss))
        slope[:, j] = (v[0] - v[1]) / (2 * step)
    tol = 2 * 10 * 2 * float(plain.tolerance(f64(x), 0.8).max()) / (2 * step) + step ** 2 / 6 * 60
    assert np.abs(slope - grad).max() < tol
    # and carried into a network: logits = h W
    h, W = torch.randn(40, 3, device="cuda"), torch.randn(3, 5, device="cuda", requires_grad=True)
    logits = h @ W
    out = learner.policy_loss(logits.detach(), targets, temperature=0.8, **a, **COEF)
    logits.backward(out.grad_logits)
    assert torch.allclose(W.grad, h.t() @ out.grad_logits, atol=1e-5)


def test_same_bits_again_and_recorded_into_a_graph(learner):
    for dtype, rows, vocab in (("bf16", 20, 151936), ("f32", 33, 40001)):
        x, targets, r = make(rows, vocab, dtype, 6)
        a, _ = inputs(x, targets, r, 1.0)
        first = learner.policy_loss(x, targets, **a, **COEF)
        second = learner.policy_loss(x, targets, **a, **COEF)
        for u, v in zip(first, second):
            assert torch.equal(u, v)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = learner.policy_loss(x, targets, **a, **COEF)
        for i in range(3):
            x.copy_(torch.from_numpy(r.normal(0, 3, (rows, vocab))).to(x.dtype))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for u, v in zip(out, learner.policy_loss(x, targets, **a, **COEF)):
                assert torch.equal(u, v)


def test_refusals(learner):
    from paper_2602_02192_amd.echo import EchoError
    x, targets, r = make(4, 100, "f32", 1)
    z = torch.zeros(4, device="cuda")
    for name, value in (("clip_low", -0.1), ("clip_high", float("nan")), ("ratio_cap", 0.0), ("sampler_cap", -1.0), ("kl_coef", float("inf")), ("entropy_coef", float("nan"))):
        with pytest.raises(EchoError, match=name):
            learner.policy_loss(x, targets, z, z, ref_logprobs=z, **{name: value})
    with pytest.raises(EchoError, match="ref_logprobs"):
        learner.policy_loss(x, targets, z, z, kl_coef=0.1)
    with pytest.raises(EchoError, match="temperature"):
        learner.policy_loss(x, targets, z, z, temperature=0.0)
    for kw in (dict(weights=z[:3]), dict(sampler_logprobs=z.double()), dict(ref_logprobs=z.cpu()), dict(grad_out=torch.empty(4, 100, device="cuda").bfloat16())):
        with pytest.raises(ValueError):
            learner.policy_loss(x, targets, z, z, **kw)
    assert learner.policy_loss(x[:0], targets[:0], z[:0], z[:0]).loss.shape == (0,)
