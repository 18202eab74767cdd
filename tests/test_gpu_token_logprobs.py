"""echo_token_logprobs and its gradient against the formulas in 64 bits: sizes, types, strides, alignments, rows that take no part, entries that are
ruled out, rows without weight, ties, NaN and infinities; the gradient against differences too."""
import numpy as np
import pytest
import torch

import learner_plain as plain

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ROUND = {"f32": 2.0 ** -23, "bf16": 2.0 ** -8, "f16": 2.0 ** -10}     # one rounding of an output, with room for a neighbouring one


@pytest.fixture(scope="module")
def learner():
    from paper_2602_02192_amd import learner as l
    return l


def make(rows, vocab, dtype, seed, pad=0, offset=0, banned=0.0, quantum=0.0, spread=3.0):
    """Logits in a larger buffer whose other elements are NaN: `offset` elements in front, `pad` between rows."""
    r = np.random.default_rng(seed)
    x = torch.from_numpy(r.normal(0, spread, (rows, vocab)).astype(np.float32))
    if quantum:
        x = torch.round(x / quantum) * quantum
    if banned:
        x[torch.from_numpy(r.random((rows, vocab)) < banned)] = -np.inf
    store = torch.full((offset + rows * (vocab + pad) + 64,), float("nan"), dtype=DT[dtype], device="cuda")
    view = store[offset:offset + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]
    view.copy_(x.to(DT[dtype]))
    targets = torch.from_numpy(r.integers(0, vocab, rows).astype(np.int32)).cuda()
    return view, targets, r


def f64(t):
    return t.detach().to("cpu", torch.float64).numpy()


def check(learner, x, targets, T, k):
    got = learner.token_logprobs(x, targets, temperature=T, top_k=k)
    tn = None if targets is None else targets.cpu().numpy()
    want = plain.rows(f64(x), tn, T, k)
    tol = np.maximum(plain.tolerance(f64(x), T), 0)
    close = lambda a, b, t: np.testing.assert_array_less(np.abs(np.where(np.isfinite(b), f64(a) - b, np.where(f64(a) == b, 0, np.inf))) - t, 1e-30)  # noqa: E731
    close(got.lse, want["lse"], tol)
    close(got.entropy, want["entropy"], tol * (2 + want["entropy"]))
    if tn is not None:
        close(got.logprobs, want["logprobs"], 2 * tol)
    else:
        assert got.logprobs is None
    if k:
        assert np.array_equal(got.top_ids.cpu().numpy(), want["top_ids"])
        close(got.top_logprobs, want["top_logprobs"], 2 * tol[:, None])
    return got, want


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,pad,offset,T,k", [
    (1, 1, 0, 0, 1.0, 1), (3, 2, 0, 0, 0.7, 2), (5, 7, 1, 1, 1.0, 5), (4, 255, 0, 3, 1.3, 4), (4, 256, 8, 0, 1.0, 20), (3, 1025, 7, 1, 1.0, 64), (2, 4097, 0, 5, 0.5, 20),
    (70, 1024, 0, 0, 1.0, 8), (3, 16385, 3, 2, 1.0, 20), (2, 32768, 0, 0, 1.0, 0), (2, 33001, 1, 0, 1.0, 33), (1, 151936, 0, 0, 1.0, 20), (1, 262147, 0, 1, 1.0, 7),
    (600, 2049, 1, 0, 1.0, 3)])
def test_against_the_formulas(learner, dtype, rows, vocab, pad, offset, T, k):
    x, targets, _ = make(rows, vocab, dtype, rows * 7 + vocab, pad, offset)
    check(learner, x, targets, T, k)


def test_no_rows(learner):
    x = torch.empty(0, 50, device="cuda")
    got = learner.token_logprobs(x, torch.empty(0, dtype=torch.int32, device="cuda"), top_k=3)
    assert got.logprobs.shape == (0,) and got.top_ids.shape == (0, 3)
    z = torch.empty(0, device="cuda")
    assert learner.token_logprobs_grad(x, torch.empty(0, dtype=torch.int32, device="cuda"), z, z, z).shape == (0, 50)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_without_targets(learner, dtype):
    x, _, r = make(9, 3001, dtype, 5, banned=0.2)
    got, want = check(learner, x, None, 0.9, 6)
    h = torch.from_numpy(r.normal(0, 1, 9).astype(np.float32)).cuda()
    out = learner.token_logprobs_grad(x, None, got.lse, got.entropy, None, h, temperature=0.9)
    check_grad(out, x, want, None, np.zeros(9), f64(h), 0.9, dtype)


@pytest.mark.parametrize("dtype,vocab", [("f32", 900), ("bf16", 900), ("f16", 17001), ("bf16", 152003)])
def test_rows_that_take_no_part_are_not_read(learner, dtype, vocab):
    x, targets, r = make(8, vocab, dtype, 11)
    for row, t in ((0, -1), (3, vocab), (5, 2 ** 31 - 1), (6, -2 ** 31)):
        x[row] = float("nan")
        targets[row] = t
    keep = [1, 2, 4, 7]
    got = learner.token_logprobs(x, targets, top_k=4)
    want = plain.rows(np.nan_to_num(f64(x)), targets.cpu().numpy(), 1.0, 4)
    for t in (0, 3, 5, 6):
        assert got.logprobs[t] == 0 and got.entropy[t] == 0 and got.lse[t] == 0 and (got.top_ids[t] == -1).all() and (got.top_logprobs[t] == 0).all()
    assert np.array_equal(got.top_ids.cpu().numpy()[keep], want["top_ids"][keep])
    np.testing.assert_allclose(f64(got.logprobs)[keep], want["logprobs"][keep], atol=1e-4)
    g = torch.ones(8, device="cuda")
    grad = learner.token_logprobs_grad(x, targets, got.lse, got.entropy, g, g)
    assert (grad[[0, 3, 5, 6]] == 0).all() and torch.isfinite(grad).all() and (grad[keep].float().abs().amax(1) > 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab,banned", [(300, 0.9), (40000, 0.999), (151936, 0.9999)])
def test_entries_that_are_ruled_out(learner, dtype, vocab, banned):
    x, targets, r = make(6, vocab, dtype, 3, banned=banned)
    x[1] = -np.inf                       # nothing left
    x[2] = -np.inf
    x[2, vocab - 1] = -2.5               # a single entry left, the given one
    targets[2] = vocab - 1
    x[3] = torch.finfo(x.dtype).min      # the lowest value of the type is a value
    x[4, 0] = 1.0                        # the given entry is ruled out
    x[4, 5] = -np.inf
    targets[4] = 5
    got, want = check(learner, x, targets, 1.0, 10)
    assert got.logprobs[1] == -np.inf and got.lse[1] == -np.inf and got.entropy[1] == 0 and (got.top_ids[1] == -1).all()
    assert got.logprobs[2] == 0 and got.entropy[2] == 0 and got.top_ids[2, 0] == vocab - 1 and (got.top_ids[2, 1:] == -1).all()
    assert got.top_ids[3].tolist() == list(range(10))
    assert got.logprobs[4] == -np.inf
    g = torch.from_numpy(r.normal(0, 1, 6).astype(np.float32)).cuda()
    h = torch.from_numpy(r.normal(0, 1, 6).astype(np.float32)).cuda()
    out = learner.token_logprobs_grad(x, targets, got.lse, got.entropy, g, h)
    assert (out[1] == 0).all()
    check_grad(out, x, want, targets.cpu().numpy(), f64(g), f64(h), 1.0, dtype)


@pytest.mark.parametrize("vocab,quantum", [(1000, 4.0), (20000, 1.0), (151936, 0.5), (151936, 100.0)])
def test_ties_go_to_the_lowest_index(learner, vocab, quantum):
    x, targets, _ = make(4, vocab, "bf16", 9, quantum=quantum)      # quantum 100: every logit is a zero, of either sign
    check(learner, x, targets, 1.0, 64)
    x[1] = 0.75
    got, _ = check(learner, x, targets, 1.0, 64)
    assert got.top_ids[1].tolist() == list(range(64))
    x[2] = torch.arange(vocab, device="cuda") % 3 - 5.0
    check(learner, x, targets, 1.0, 50)


def test_rising_and_falling_rows(learner):
    for vocab in (151936, 70001):
        x = torch.stack([torch.arange(vocab, device="cuda"), torch.arange(vocab, 0, -1, device="cuda")]).float() / 4096
        check(learner, x, torch.tensor([5, vocab - 1], dtype=torch.int32, device="cuda"), 1.0, 64)


@pytest.mark.parametrize("vocab", [300, 70001])
def test_nan_and_infinity_give_nan(learner, vocab):
    x, targets, _ = make(5, vocab, "f32", 21)
    x[0, 17] = float("nan")
    x[1, 200] = float("inf")
    x[2] = float("nan")
    x[3] = float("inf")
    got = learner.token_logprobs(x, targets, top_k=5)
    for t in range(4):
        assert torch.isnan(got.logprobs[t]) and torch.isnan(got.entropy[t]) and torch.isnan(got.lse[t])
        assert ((got.top_ids[t] >= -1) & (got.top_ids[t] < vocab)).all()
    assert torch.isfinite(got.logprobs[4])
    one = torch.ones(5, device="cuda")
    grad = learner.token_logprobs_grad(x, targets, got.lse, got.entropy, one)
    assert torch.isnan(grad[:4]).all() and torch.isfinite(grad[4]).all()


def check_grad(out, x, want, targets, g, h, T, dtype):
    d, size = plain.logit_gradient(want, targets, g, h, T)
    tol = np.maximum(plain.tolerance(f64(x), T), 0)[:, None]
    # the log-sum and the entropy that go in carry their own error; a half below 2^-14 is a multiple of 2^-24
    bound = 4 * tol * size + ROUND[dtype] * np.abs(d) + (2.0 ** -24 if dtype == "f16" else 1e-38) + (np.abs(h)[:, None] * want["p"] * tol * (2 + want["entropy"][:, None]) / T)
    assert (np.abs(f64(out) - d) <= bound).all(), float((np.abs(f64(out) - d) - bound).max())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,pad,offset,T", [(1, 1, 0, 0, 1.0), (5, 7, 1, 1, 0.7), (3, 255, 0, 1, 1.0), (40, 1024, 8, 0, 1.0), (3, 16385, 3, 5, 1.3), (2, 151936, 0, 0, 1.0),
                                                     (300, 2051, 1, 0, 1.0)])
def test_gradient_against_the_formula(learner, dtype, rows, vocab, pad, offset, T):
    x, targets, r = make(rows, vocab, dtype, vocab + 1, pad, offset)
    got, want = check(learner, x, targets, T, 0)
    g, h = (torch.from_numpy(r.normal(0, 1, rows).astype(np.float32)).cuda() for _ in range(2))
    for gg, hh in ((g, h), (g, None), (None, h)):
        out = learner.token_logprobs_grad(x, targets, got.lse, got.entropy if hh is not None else None, gg, hh, temperature=T)
        check_grad(out, x, want, targets.cpu().numpy(), f64(gg) if gg is not None else np.zeros(rows), f64(hh) if hh is not None else np.zeros(rows), T, dtype)
    # into rows that lie further apart, and in place of the logits
    wide = torch.full((rows, vocab + 5), 7.0, dtype=DT[dtype], device="cuda")
    again = learner.token_logprobs_grad(x, targets, got.lse, got.entropy, g, h, temperature=T, out=wide[:, :vocab])
    full = learner.token_logprobs_grad(x, targets, got.lse, got.entropy, g, h, temperature=T)
    assert torch.equal(again, full) and (wide[:, vocab:] == 7.0).all()
    assert learner.token_logprobs_grad(x, targets, got.lse, got.entropy, g, h, temperature=T, out=x).data_ptr() == x.data_ptr()
    assert torch.equal(x, full)


def test_gradient_against_differences(learner):
    """Central differences of the operator itself: its values are good to `tolerance`, the third derivative of logprob + entropy is below 30 here."""
    x, targets, r = make(2, 6, "f32", 77, spread=1.0)
    g, h = torch.tensor([1.0, -0.5], device="cuda"), torch.tensor([0.7, 1.0], device="cuda")
    T, step = 0.8, 2.0 ** -6
    x.requires_grad_(False)
    leaf = x.detach().clone().requires_grad_(True)
    out = learner.token_logprobs(leaf, targets, temperature=T, top_k=2)
    assert out.logprobs.requires_grad and out.entropy.requires_grad and not out.lse.requires_grad and not out.top_logprobs.requires_grad
    (out.logprobs * g + out.entropy * h).sum().backward()
    tol = 2 * float(plain.tolerance(f64(x), T).max()) * 4 / step + step ** 2 / 6 * 30
    for t in range(2):
        for j in range(6):
            v = []
            for s in (step, -step):
                y = x.clone()
                y[t, j] += s
                o = learner.token_logprobs(y, targets, temperature=T)
                v.append(float((o.logprobs.double() * g + o.entropy.double() * h)[t]))
            assert abs((v[0] - v[1]) / (2 * step) - float(leaf.grad[t, j])) < tol
    only = x.detach().clone().requires_grad_(True)
    learner.token_logprobs(only, targets, temperature=T).logprobs.sum().backward()
    want = plain.rows(f64(x), targets.cpu().numpy(), T)
    check_grad(only.grad, x, want, targets.cpu().numpy(), np.ones(2), np.zeros(2), T, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [5, 1000, 40003, 151936])
def test_rows_in_which_everything_is_ruled_out_by_a_large_number(learner, dtype, vocab):
    """Equal entries of any size are a uniform distribution; beside an ordinary entry they have no weight."""
    values = [-1e4, -6.1e5, -1e9, -1.3e9, -1e10, -1e15, -3e20, 1e10, 7e25, 3e38, -3e38]
    x = torch.tensor(values, device="cuda")[:, None].expand(-1, vocab).to(DT[dtype]).contiguous()
    rows = len(values)
    targets = torch.full((rows,), vocab - 1, dtype=torch.int32, device="cuda")
    one, loss = torch.ones(rows, device="cuda"), dict(clip_low=0.2, clip_high=0.2, kl_coef=0.0, entropy_coef=0.1)
    for T in (1.0, 1.25):
        got = learner.token_logprobs(x, targets, temperature=T, top_k=3)
        for v in (got.logprobs, got.top_logprobs[:, 0], got.top_logprobs[:, 2], -got.entropy):
            np.testing.assert_allclose(f64(v), -np.log(vocab), atol=1e-5)
        assert (got.top_ids == torch.arange(3, device="cuda")).all()
        out = learner.policy_loss(x, targets, one, got.logprobs, temperature=T, **loss)
        # ratio 1: d loss / d x_j = -(1[j = target] - p) / T, entropy at its largest
        np.testing.assert_allclose(f64(out.logprobs), -np.log(vocab), atol=1e-5)
        want = np.full(vocab, 1 / vocab) / T
        want[-1] -= 1 / T
        np.testing.assert_allclose(f64(out.grad_logits), np.broadcast_to(want, (rows, vocab)), rtol=ROUND[dtype] + 1e-4, atol=1e-6 / vocab)
        grad = learner.token_logprobs_grad(x, targets, got.lse, got.entropy, one, one, temperature=T)
        assert torch.isfinite(grad).all() and (grad.float().abs() <= 2 * (1 + np.log(vocab)) / T).all()
    x[:, 1] = torch.where(x[:, 1] < 0, 2.0, x[:, 1].float()).to(x.dtype)
    got = learner.token_logprobs(x, targets.clamp(max=0) + 1)
    below = [i for i, v in enumerate(values) if v < 0]
    assert (got.logprobs[below] == 0).all() and (got.entropy[below] == 0).all() and (got.lse[below] == 2.0).all()


def test_temperatures_of_every_size(learner):
    x, targets, _ = make(6, 3001, "f32", 91)
    for T in (1e-6, 1e-3, 50.0, 1e6, 1e30):
        check(learner, x, targets, T, 4)
        check(learner, x * T, targets, T, 4)


def test_same_bits_again_and_on_another_stream(learner):
    x, targets, _ = make(130, 40007, "bf16", 2)
    a = learner.token_logprobs(x, targets, top_k=9)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = learner.token_logprobs(x, targets, top_k=9)
    torch.cuda.current_stream().wait_stream(s)
    for u, v in zip(a, b):
        assert torch.equal(u, v)


def test_recorded_into_a_graph(learner):
    x, targets, r = make(33, 20011, "bf16", 4)
    one = torch.ones(33, device="cuda")
    learner.token_logprobs(x, targets, top_k=5)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = learner.token_logprobs(x, targets, top_k=5)
        grad = learner.token_logprobs_grad(x, targets, out.lse, out.entropy, one, one)
    for i in range(4):
        x.copy_(torch.from_numpy(r.normal(0, 3, (33, 20011))).to(x.dtype))
        targets.copy_(torch.from_numpy(r.integers(-1, 20011, 33)))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = learner.token_logprobs(x, targets, top_k=5)
        for a, b in zip(out, want):
            assert torch.equal(a, b)
        assert torch.equal(grad, learner.token_logprobs_grad(x, targets, want.lse, want.entropy, one, one))


def test_rows_beyond_32_bits_of_elements(learner):
    rows, vocab = 15000, 151936          # 2.28e9 elements: the last rows start beyond 2^31
    x = torch.empty(rows, vocab, dtype=torch.bfloat16, device="cuda")
    x.normal_(0, 2)
    targets = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    targets[[0, 14135, 14999]] = torch.tensor([3, 151935, 77], dtype=torch.int32, device="cuda")
    got = learner.token_logprobs(x, targets, top_k=3)
    at = [0, 14135, 14999]
    few = learner.token_logprobs(x[at].clone(), targets[at], top_k=3)
    assert torch.equal(got.top_ids[at], few.top_ids)
    np.testing.assert_allclose(f64(got.logprobs[at]), f64(few.logprobs), atol=1e-5)
    one = torch.ones(rows, device="cuda")
    learner.token_logprobs_grad(x, targets, got.lse, got.entropy, one, out=x)
    assert (x[14999, 77] > 0) and (x[1] == 0).all() and (x[14998] == 0).all() and x[14999].float().abs().sum() > 0


def test_refusals(learner):
    from paper_2602_02192_amd.echo import EchoError
    x, targets, _ = make(4, 100, "f32", 1)
    z = torch.zeros(4, device="cuda")
    for bad in (0.0, -1.0, float("nan"), float("inf"), 1e-39):
        with pytest.raises(EchoError) as e:
            learner.token_logprobs(x, targets, temperature=bad)
        assert e.value.code == -1 and "temperature" in str(e.value)
    for k in (-1, 65, 101):
        with pytest.raises(EchoError, match="top_k"):
            learner.token_logprobs(x, targets, top_k=k)
    with pytest.raises(EchoError, match="top_k"):
        learner.token_logprobs(x[:, :3], targets, top_k=4)
    with pytest.raises(EchoError, match="grad_logprobs or grad_entropy"):
        learner.token_logprobs_grad(x, targets, z, z, None)
    with pytest.raises(EchoError, match="entropy"):
        learner.token_logprobs_grad(x, targets, z, None, z, z)
    with pytest.raises(EchoError, match="targets"):
        learner.token_logprobs_grad(x, None, z, z, z)
    store = torch.zeros(4 * 120, device="cuda")
    with pytest.raises(EchoError, match="row stride"):
        learner.token_logprobs_grad(store.as_strided((4, 100), (120, 1)), targets, z, z, z, out=store.as_strided((4, 100), (100, 1)))
    for wrong in (x.t(), x.double(), x[0], x.cpu(), x.as_strided((4, 100), (50, 1))):
        with pytest.raises(ValueError):
            learner.token_logprobs(wrong, targets)
    for wrong in (targets.long(), targets[:3], targets.cpu(), targets.view(2, 2)):
        with pytest.raises(ValueError):
            learner.token_logprobs(x, wrong)
    with pytest.raises(ValueError):
        learner.token_logprobs_grad(x, targets, z.half(), z, z)
    with pytest.raises(ValueError):
        learner.token_logprobs_grad(x, targets, z, z, z, out=torch.empty(4, 99, device="cuda"))


def test_no_second_derivative(learner):
    """Refused, not left out of the sum that it belongs to."""
    x, targets, r = make(5, 40, "f32", 3)
    x = x.clone().requires_grad_()
    first, = torch.autograd.grad((learner.token_logprobs(x, targets).logprobs ** 2).sum() + (x ** 3).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        first.sum().backward()


def test_what_is_written_in_place_counts_as_changed(learner):
    """A backward pass that still needs the old values is refused by torch, as after its own operations in place."""
    x, targets, r = make(5, 40, "f32", 4)
    z, w = torch.zeros(5, device="cuda"), torch.ones(5, 40, device="cuda", requires_grad=True)
    for write in (lambda y: learner.policy_loss(y, targets, z, z, grad_out=y),
                  lambda y: learner.token_logprobs_grad(y, targets, z, None, z, out=y),
                  lambda y: learner.adamw_step([y], [torch.ones_like(y)], torch.zeros(256, device="cuda"), torch.zeros(256, device="cuda"), step=1, lr=0.1)):
        y = x.clone().contiguous()
        later = (y * w).sum()
        write(y)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            later.backward()
    p, g, s, out = (torch.zeros(300, device="cuda") for _ in range(4))
    m, v, short = torch.zeros(512, device="cuda"), torch.zeros(512, device="cuda"), torch.zeros(300, dtype=torch.bfloat16, device="cuda")
    norm = torch.zeros((), device="cuda")
    learner.grad_norm([g], out=norm)
    learner.adamw_step([p], [g], m, v, step=1, lr=0.1, snapshot=[short])
    assert all(t._version > 0 for t in (norm, p, m, v, short)) and g._version == 0
