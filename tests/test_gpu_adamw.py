"""echo_grad_norm and echo_adamw_step: bit for bit the operations that the header states, close to the formulas in 64 bits; 8-bit states and bf16
parameters rounded by the stated random bits, without bias; tensors of all sizes and alignments; steps that must not happen."""
import numpy as np
import pytest
import torch

import learner_plain as plain

pytestmark = pytest.mark.gpu

HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-8)
SIZES = [1, 3, 4, 255, 256, 257, 1000, 4096, 4097, 12289, 0, 5, 70001]


@pytest.fixture(scope="module")
def learner():
    from paper_2602_02192_amd import learner as l
    return l


def pieces(sizes, dtype, values, offset):
    """Views into one buffer, each `offset` elements behind the one before: alignments of every kind."""
    store = torch.zeros(sum(sizes) + offset * (len(sizes) + 1), dtype=dtype, device="cuda")
    out, at = [], offset
    for n in sizes:
        out.append(store[at:at + n])
        at += n + offset
    for t, v in zip(out, values):
        t.copy_(torch.from_numpy(v))
    return out


def problem(sizes, seed, grads="f32", params="f32", offset=1):
    r = np.random.default_rng(seed)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}
    p = pieces(sizes, dt[params], [r.normal(0, 0.05, n).astype(np.float32) for n in sizes], offset)
    g = pieces(sizes, dt[grads], [(r.normal(0, 1, n) * np.exp(r.normal(0, 2, n)) * 1e-3 * (r.random(n) > 0.1)).astype(np.float32) for n in sizes], offset)
    return p, g, r


def host(t):
    return t.detach().float().cpu().numpy()


def starts(sizes):
    return np.concatenate([[0], np.cumsum([-(-n // 256) * 256 for n in sizes])])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("sizes", [[1], [0], [7, 0, 300], SIZES, [16384, 16385, 100000], [3] * 150, [5_000_001]])
def test_norm(learner, dtype, sizes):
    r = np.random.default_rng(len(sizes))
    g = pieces(sizes, dtype, [(r.normal(0, 1, n) * np.exp(r.normal(0, 1, n))).astype(np.float32) for n in sizes], 1)
    want = np.sqrt(sum((host(t).astype(np.float64) ** 2).sum() for t in g))
    got = learner.grad_norm(g)
    # squares are exact in 64 bits and their sum is off by less than 2^-40 of it: one rounding to f32
    assert abs(float(got) - want) <= 2.0 ** -24 * 1.0001 * want
    out = torch.zeros(1, device="cuda")
    assert learner.grad_norm(g, out=out) is out and float(out) == float(got)


def test_norm_of_large_small_and_wrong_values(learner):
    g = [torch.full((1000,), 1e30, device="cuda"), torch.full((10,), 1e-30, device="cuda")]
    assert abs(float(learner.grad_norm(g)) / (1e30 * np.sqrt(1000)) - 1) < 2e-7         # the sum of squares is beyond f32
    assert abs(float(learner.grad_norm(g[1:])) / (1e-30 * np.sqrt(10)) - 1) < 2e-7
    g[0][17] = float("inf")
    assert float(learner.grad_norm(g)) == float("inf")
    g[1][3] = float("nan")
    assert np.isnan(float(learner.grad_norm(g)))


@pytest.mark.parametrize("grads", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("clip", [None, 0.01, 1e9])
def test_32_bit_states(learner, grads, offset, clip):
    p, g, r = problem(SIZES, 3, grads, offset=offset)
    decay = [0.1 if i % 2 else 0.0 for i in range(len(SIZES))]
    n = learner.state_numel(p)
    m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    snap = pieces(SIZES, torch.bfloat16, [np.zeros(k, np.float32) for k in SIZES], offset)
    ref = [(host(a), np.zeros(a.numel(), np.float32), np.zeros(a.numel(), np.float32)) for a in p]
    ref64 = [tuple(x.astype(np.float64) for x in t) for t in ref]
    at = starts(SIZES)
    for step in (1, 2, 3):
        norm = learner.grad_norm(g) if clip else None
        learner.adamw_step(p, g, m, v, step=step, weight_decay=decay, snapshot=snap, norm=norm, max_norm=clip or float("inf"), **HYPER)
        f = np.float32(1)
        if clip and float(norm) > clip:
            f = np.float32(clip) / np.float32(float(norm))
        for i, a in enumerate(p):
            ref[i] = plain.adamw(ref[i][0], host(g[i]), *ref[i][1:], decay[i], step=step, factor=f, **HYPER)
            ref64[i] = plain.adamw(ref64[i][0], host(g[i]), *ref64[i][1:], decay[i], step=step, factor=float(f), dtype=np.float64, **HYPER)
            k = a.numel()
            assert np.array_equal(host(a), ref[i][0]), (step, i)
            assert np.array_equal(host(m[at[i]:at[i] + k]), ref[i][1]) and np.array_equal(host(v[at[i]:at[i] + k]), ref[i][2])
            assert (m[at[i] + k:at[i + 1]] == 0).all() and (v[at[i] + k:at[i + 1]] == 0).all()
            assert np.array_equal(snap[i].view(torch.int16).cpu().numpy().view(np.uint16), plain.to_bf16(ref[i][0]))
            # eight roundings a step on the update, one on p: each at most 2^-24 of p or of the update (below 11 lr)
            assert (np.abs(ref[i][0] - ref64[i][0]) <= step * 2.0 ** -23 * (np.abs(ref64[i][0]) + 8 * 11 * HYPER["lr"])).all()
        for t in g:
            t.mul_(-0.7).add_(1e-4)


def test_nothing_beyond_the_tensors_is_written(learner):
    store, grads = torch.full((5000,), 3.0, device="cuda"), torch.ones(5000, device="cuda")
    p, g = [store[7:7 + 4099], store[4200:4203]], [grads[7:7 + 4099], grads[4200:4203]]
    n = learner.state_numel(p)
    m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    learner.adamw_step(p, g, m, v, step=1, **HYPER)
    inside = torch.zeros(5000, dtype=torch.bool, device="cuda")
    inside[7:7 + 4099] = inside[4200:4203] = True
    assert (store[~inside] == 3.0).all() and (store[inside] != 3.0).all()


def philox16(first, n, step, purpose, seed):
    w = plain.philox(first, n, step, purpose, seed)
    return (w & 0xFFFF).astype(np.int64), (w >> 16).astype(np.int64)


@pytest.mark.parametrize("params,grads", [("f32", "bf16"), ("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
def test_8_bit_states_and_bf16_parameters(learner, params, grads):
    p, g, r = problem(SIZES, 5, grads, params)
    n, at, seed = learner.state_numel(p), starts(SIZES), (7 << 40) + 12345
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    ms, vs = torch.zeros(n // 256, device="cuda"), torch.zeros(n // 256, device="cuda")
    codes = {k: np.zeros(n, np.uint8) for k in "mv"}
    scales = {k: np.zeros(n // 256, np.float32) for k in "mv"}
    P = [host(t) for t in p]
    for step in range(1, 5):
        learner.adamw_step(p, g, m, v, step=step, weight_decay=0.1, m_scale=ms, v_scale=vs, seed=seed, **HYPER)
        for i, a in enumerate(p):
            k, b0, b1 = a.numel(), at[i] // 256, at[i + 1] // 256
            old = [(plain.E4M3[codes[s][at[i]:at[i + 1]]].reshape(-1, 256) * scales[s][b0:b1, None]).reshape(-1)[:k] for s in "mv"]
            new, *state = plain.adamw(P[i], host(g[i]), *old, 0.1, step=step, factor=1.0, **HYPER)
            bits = philox16(at[i], at[i + 1] - at[i], step, 0, seed)
            for s, x, b in zip("mv", state, bits):
                codes[s][at[i]:at[i + 1]], scales[s][b0:b1] = plain.encode(np.pad(x, (0, at[i + 1] - at[i] - k)), b, s == "v")
            if params == "bf16":
                up = philox16(at[i], k, step, 1, seed)[0]
                new = ((new.view(np.uint32) + up.astype(np.uint32)) & np.uint32(0xFFFF0000)).view(np.float32)
            P[i] = new
            assert np.array_equal(host(a), new), (step, i)
        assert np.array_equal(m.view(torch.uint8).cpu().numpy(), codes["m"]) and np.array_equal(host(ms), scales["m"])
        assert np.array_equal(v.view(torch.uint8).cpu().numpy(), codes["v"]) and np.array_equal(host(vs), scales["v"])
        for t in g:
            t.mul_(-0.8).add_(1e-5)


def test_rounding_by_chance_has_no_bias(learner):
    """A constant gradient: averages reach it to the noise of the rounding, although a step moves them by far less than a code; the mean of 65536
    values with steps of 1/8 of their size at most is within 5 sigma of the average's value."""
    n = 65536
    p = [torch.zeros(n, dtype=torch.bfloat16, device="cuda")]
    r = np.random.default_rng(1)
    g = [torch.from_numpy(np.exp(r.normal(0, 1, n)).astype(np.float32)).cuda()]
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    ms, vs = torch.zeros(n // 256, device="cuda"), torch.zeros(n // 256, device="cuda")
    for step in range(1, 401):
        learner.adamw_step(p, g, m, v, step=step, lr=1e-4, beta1=0.9, beta2=0.99, m_scale=ms, v_scale=vs, seed=9)
    gn = g[0].double().cpu().numpy()
    val = lambda c, s: (c.float().view(-1, 256) * s[:, None]).view(-1).double().cpu().numpy()  # noqa: E731
    for got, want, fresh in ((val(m, ms), gn, 0.1), (val(v, vs), gn ** 2 * (1 - 0.99 ** 400), 0.01)):
        # one rounding: sigma at most 1/16 of the value; the average of past ones adds 1 / sqrt(2 fresh) of that
        rel = got / want - 1
        sigma = 1 / 16 * np.sqrt(1 / (2 * fresh) + 1)
        large = want > 1e-3 * np.repeat(want.reshape(-1, 256).max(1), 256)
        assert abs(rel[large].mean()) < 5 * sigma / np.sqrt(large.sum()), rel[large].mean()
    # each bf16 parameter has gone about -400 lr, in steps below its own spacing from 2^-6 on
    assert abs(float(p[0].float().mean()) / (-400 * 1e-4) - 1) < 0.03


def test_a_norm_that_is_not_finite_changes_nothing(learner):
    for states in (torch.float32, torch.float8_e4m3fn):
        p, g, _ = problem([1000, 5], 4)
        g[0][3] = float("nan")
        opt = learner.AdamW(p, lr=1e-3, max_norm=1.0, state_dtype=states, weight_decay=0.1)
        before = [t.clone() for t in p]
        assert np.isnan(float(opt.step(g)))
        assert all(torch.equal(a, b) for a, b in zip(p, before)) and (opt.m.float() == 0).all() and opt.steps == 1
        g[0][3] = 1.0
        assert np.isfinite(float(opt.step(g))) and not torch.equal(p[0], before[0])


def test_gradients_that_are_not_finite_without_a_norm(learner):
    for states in (torch.float32, torch.float8_e4m3fn):
        p, g, _ = problem([1000], 4)
        g[0][3], g[0][700] = float("nan"), float("inf")
        opt = learner.AdamW(p, lr=1e-3, state_dtype=states)
        opt.step(g)
        assert torch.isnan(p[0][3]) and torch.isnan(p[0][700]) and torch.isfinite(p[0][256:512]).all()
        assert torch.isfinite(p[0][:3]).all() and torch.isnan(opt.m.float()[3])


def test_bf16_parameters_that_are_not_finite_stay_so(learner):
    for states in (torch.float32, torch.float8_e4m3fn):
        p, g, _ = problem([1000], 4, "bf16", "bf16")
        g[0][:].add_(1e-3)
        bad = {3: float("nan"), 4: float("inf"), 700: float("-inf"), 999: float("nan")}
        for i, v in bad.items():
            p[0][i] = v
        opt = learner.AdamW(p, lr=1e-3, weight_decay=0.1, state_dtype=states)
        for _ in range(3):
            opt.step(g)
        assert torch.isnan(p[0][[3, 999]]).all() and p[0][4] == float("inf") and p[0][700] == float("-inf")
        assert torch.isfinite(p[0][[i for i in range(1000) if i not in bad]]).all()


def test_zero_gradients_and_tiny_ones(learner):
    for states in (torch.float32, torch.float8_e4m3fn):
        p = [torch.ones(600, device="cuda")]
        g = [torch.zeros(600, device="cuda")]
        opt = learner.AdamW(p, lr=1e-2, state_dtype=states)
        opt.step(g)
        assert (p[0] == 1).all()
        g[0][:300] = 1e-25           # squares vanish in f32: m / eps
        opt.step(g)
        assert torch.isfinite(p[0]).all() and (p[0][300:] == 1).all()


def test_square_root_and_quotient_bit_for_bit():
    import os
    import subprocess
    from paper_2602_02192_amd import build
    if not os.path.exists(build.UPDATE_SWEEP):
        build.build_sweep()
    r = subprocess.run([build.UPDATE_SWEEP], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout.split() == ["roots", "0", "reciprocals", "0", "quotients", "0"], r.stdout + r.stderr


@pytest.mark.parametrize("scale", [1e-30, 1e-18, 1e-13, 1e-3, 1e12, 1e18])
def test_averages_of_every_size(learner, scale):
    """From squares that vanish in f32 to squares near its end: the bits of the operations as written, whichever form computes them."""
    n = 5000
    r = np.random.default_rng(2)
    gn = (r.normal(0, 1, n) * np.exp(r.normal(0, 3, n)) * scale).astype(np.float32)
    gn[::7] = 0
    gn[4096:4400] = 0
    for eps, root in ((1e-8, 0.999), (1e-30, 0.999), (1e-8, 0.0)):
        p, g = [torch.ones(n, device="cuda")], [torch.from_numpy(gn).cuda()]
        m, v = torch.zeros(5120, device="cuda"), torch.zeros(5120, device="cuda")
        hyper = dict(lr=1e-3, beta1=0.9, beta2=root, eps=eps)
        learner.adamw_step(p, g, m, v, step=1, **hyper)
        want = plain.adamw(np.ones(n, np.float32), gn, np.zeros(n, np.float32), np.zeros(n, np.float32), 0.0, step=1, factor=1.0, **hyper)
        for got, ref in zip((p[0], m[:n], v[:n]), want):
            assert np.array_equal(host(got), ref)


def test_states_far_apart(learner):
    """Averages that do not go together, as a damaged checkpoint has them: large m over the root of a small v passes the end of f32."""
    n = 1024
    r = np.random.default_rng(3)
    m0 = np.ldexp(r.normal(0, 1, n), r.integers(-100, 100, n)).astype(np.float32)
    v0 = np.ldexp(np.abs(r.normal(0, 1, n)), r.integers(-100, 100, n)).astype(np.float32)
    m0[256:512], v0[256:512] = np.ldexp(m0[256:512], 0) * 0 + 2.0 ** 79, 2.0 ** -79
    for eps in (1e-8, 2.0 ** -60):
        p, g = [torch.ones(n, device="cuda")], [torch.zeros(n, device="cuda")]
        m, v = torch.from_numpy(m0).cuda(), torch.from_numpy(v0).cuda()
        hyper = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=eps)
        learner.adamw_step(p, g, m, v, step=100000, **hyper)
        want = plain.adamw(np.ones(n, np.float32), np.zeros(n, np.float32), m0, v0, 0.0, step=100000, factor=1.0, **hyper)
        for got, ref in zip((p[0], m, v), want):
            assert np.array_equal(host(got), ref, equal_nan=True)


def test_state_dict_and_graph(learner):
    p, g, _ = problem([5000, 77], 8, grads="bf16", params="bf16")
    opt = learner.AdamW(p, lr=1e-3, state_dtype=torch.float8_e4m3fn, seed=3, max_norm=1.0)
    opt.step(g)
    saved = {k: (t.clone() if torch.is_tensor(t) else t) for k, t in opt.state_dict().items()}
    before = [t.clone() for t in p]
    opt.step(g)
    after = [t.clone() for t in p]
    other = learner.AdamW(before, lr=1e-3, state_dtype=torch.float8_e4m3fn, max_norm=1.0)
    other.load_state_dict(saved)
    other.step(g)
    assert all(torch.equal(a, b) for a, b in zip(before, after)) and torch.equal(other.m.view(torch.uint8), opt.m.view(torch.uint8))
    with pytest.raises(ValueError):
        learner.AdamW(p, lr=1e-3).load_state_dict(saved)
    # a step that is recorded reads the gradients that are there when it is replayed
    p, g, _ = problem([5000, 77], 8)
    q = [t.clone() for t in p]
    n = learner.state_numel(p)
    state = [torch.zeros(n, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = learner.grad_norm(g)
        learner.adamw_step(p, g, state[0], state[1], step=5, norm=norm, max_norm=0.1, **HYPER)
    for i in range(3):
        for t in g:
            t.mul_(0.9)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        learner.adamw_step(q, g, state[2], state[3], step=5, norm=learner.grad_norm(g), max_norm=0.1, **HYPER)
        assert all(torch.equal(a, b) for a, b in zip(p, q)) and torch.equal(state[0], state[2])


def test_tensors_beyond_32_bits_of_elements(learner):
    n = 2 ** 31 + 5000                               # the parameter's end lies beyond 2^32 bytes, the last elements beyond 2^31
    p, g = [torch.full((1000,), 0.5, dtype=torch.bfloat16, device="cuda"), torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda")], []
    g = [torch.ones(1000, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")]
    g[1][-4000:] = 2.0
    g[1][:300] = 1.0
    norm = learner.grad_norm(g)
    assert abs(float(norm) / np.sqrt(1300 + 4 * 4000) - 1) < 2e-7
    opt = learner.AdamW(p, lr=0.125, state_dtype=torch.float8_e4m3fn, seed=5)
    opt.step(g)
    # the first step moves by lr against the gradient's sign: 0.375 is a bf16, and next to it what rounding by chance gives
    assert ((p[1][-4000:].float() - 0.375).abs() < 0.004).all() and ((p[1][:300].float() - 0.375).abs() < 0.004).all()
    assert (p[1][300:1000] == 0.5).all() and (p[1][2 ** 31 - 3000:2 ** 31 + 500] == 0.5).all()
    at = n // 256 * 256 + 1024
    assert (opt.m[1024 + n - 4000:1024 + n].float() > 0).all() and (opt.m[1024 + n:].float() == 0).all() and at > 0


def test_refusals(learner):
    from paper_2602_02192_amd.echo import EchoError
    p, g = [torch.zeros(300, device="cuda")], [torch.zeros(300, device="cuda")]
    m, v = torch.zeros(512, device="cuda"), torch.zeros(512, device="cuda")
    s = torch.zeros(2, device="cuda")
    ok = dict(step=1, lr=1e-3)
    for bad, word in ((dict(step=0), "step"), (dict(lr=-1.0), "lr"), (dict(beta1=1.0), "beta"), (dict(beta2=-0.1), "beta"), (dict(eps=0.0), "eps"), (dict(lr=float("nan")), "lr"),
                      (dict(norm=s[:1], max_norm=0.0), "max_norm"), (dict(weight_decay=float("inf")), "weight_decay"), (dict(m_scale=s, v_scale=s), "scales")):
        with pytest.raises(EchoError, match=word):
            learner.adamw_step(p, g, m, v, **{**ok, **bad})
    f8 = torch.zeros(512, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    with pytest.raises(EchoError, match="scales"):
        learner.adamw_step(p, g, f8, f8.clone(), **ok)
    half = [torch.zeros(300, dtype=torch.bfloat16, device="cuda")]
    with pytest.raises(EchoError, match="snapshot"):
        learner.adamw_step(half, g, m, v, snapshot=[half[0].clone()], **ok)
    with pytest.raises(EchoError, match="aligned"):
        learner.adamw_step(p, g, torch.zeros(513, device="cuda")[1:], v, **ok)
    for args in (([p[0].half()], g, m, v), (p, [g[0][:200]], m, v), (p, g + g, m, v), (p, g, m[:300], v), (p, g, m.bfloat16(), v), (p, [g[0].cpu()], m, v), ([], [], m, v),
                 ([torch.zeros(600, device="cuda")[::2]], g, m, v)):
        with pytest.raises(ValueError):
            learner.adamw_step(*args, **ok)
    with pytest.raises(ValueError):
        learner.adamw_step(p, g, m, v, weight_decay=[0.0, 0.1], **ok)
    with pytest.raises(ValueError):
        learner.grad_norm([torch.zeros(4)])
