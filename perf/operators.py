"""The learner's operators as cases that can be timed and compared: log-probabilities of given tokens with entropy and top
alternatives, their gradient, the policy loss with its gradient, and the clipped AdamW step over many tensors.

With `own` set, a pass makes the calls a learner makes of paper_2602_02192_amd.learner; otherwise the same mathematics runs in
elementary torch operations.  Vocabulary sizes, widths and batch sizes are those of the repository's decoder shapes (tiny, 4B, 8B,
32B) and workloads.
"""
import math

import torch

own = False

_TINY = dict(hidden=256, q_heads=4, kv_heads=2, head_dim=64, ffn=704, vocab=1024)
_4B = dict(hidden=2560, q_heads=32, kv_heads=8, head_dim=128, ffn=9728, vocab=151936)
_8B = dict(hidden=4096, q_heads=32, kv_heads=8, head_dim=128, ffn=12288, vocab=151936)
_32B = dict(hidden=5120, q_heads=64, kv_heads=8, head_dim=128, ffn=25600, vocab=151936)

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_SIZES = {"f32": 4, "bf16": 2, "f16": 2}

_CLIP_LOW, _CLIP_HIGH, _RATIO_CAP, _IS_CAP, _KL, _ENTROPY = 0.2, 0.2, 4.0, 2.0, 0.04, 0.01
_LR, _BETA1, _BETA2, _EPS, _DECAY = 1e-6, 0.9, 0.999, 1e-8, 0.1
_BLOCK = 256          # elements that share a scale of the 8-bit states
_E4M3_MAX = 448.0


def _logits(name, kind, rows, vocab, dtype, pad=0, skipped=0.0, banned=0.0, temperature=1.0, **more):
    """`rows` rows of logits over `vocab` entries, `pad` further columns between rows; the share `skipped` of the rows takes no
    part (prompt, padding, another speaker's turn); the share `banned` of the entries is -inf (constrained answers)."""
    c = dict(kind=kind, rows=rows, vocab=vocab, dtype=dtype, pad=pad, skipped=skipped, banned=banned, temperature=temperature, **more)
    return dict(c, name=name) if name else c


def _adamw(name, model, layers, states, params, grads, embed=True, snapshot=False):
    """One step over the tensors of a decoder: `layers` layers and, with `embed`, the embedding table and the final norm."""
    c = dict(kind="adamw", layers=layers, states=states, params=params, grads=grads, embed=embed, snapshot=snapshot, **model)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decoded token whose alternatives a user looks at: nothing but latency
        _logits("logprobs-1x151936-top20", "logprobs", 1, 151936, "f32", top_k=20),
        # a decode step of the benchmark's batch, alternatives for every sequence
        _logits("logprobs-64x151936-top8", "logprobs", 64, 151936, "bf16", top_k=8),
        # an odd vocabulary in half precision, rows with padding between them, answers constrained to some entries
        _logits("logprobs-999x32001-f16-ragged", "logprobs", 999, 32001, "f16", pad=31, skipped=0.3, banned=0.5, temperature=0.8, top_k=5),
        # a scoring pass of the learner: 4096 positions, no alternatives
        _logits("logprobs-4096x151936", "logprobs", 4096, 151936, "bf16", top_k=0),
        # gradients for a loss of the user's own, a micro-batch
        _logits("grad-512x151936", "grad", 512, 151936, "bf16"),
        # the same in 32 bits over an odd vocabulary
        _logits("grad-777x32001-f32-ragged", "grad", 777, 32001, "f32", pad=7, skipped=0.3, temperature=0.8),
        # the policy loss of config 1's tiny model
        _logits("loss-64x1024-f32", "loss", 64, 1024, "f32"),
        # the policy loss of a micro-batch of 32-bit logits
        _logits("loss-300x151936-f32", "loss", 300, 151936, "f32", skipped=0.1),
        # the policy loss of a long multi-turn record, a third of whose tokens are not the policy's
        _logits("loss-4096x151936-turns", "loss", 4096, 151936, "bf16", skipped=0.35),
        # the update of config 1's tiny model: many small tensors
        _adamw("adamw-tiny", _TINY, 2, "f32", "f32", "f32"),
        # 32-bit states and master weights, bf16 gradients, and the bf16 snapshot that is published
        _adamw("adamw-4b-2layers+embed", _4B, 2, "f32", "f32", "bf16", snapshot=True),
        # 8-bit states and bf16 weights without a master copy: the form that fits the largest policy on one GPU
        _adamw("adamw-32b-1layer-e4m3", _32B, 1, "e4m3", "bf16", "bf16", embed=False),
    ]


def draw(rng):
    def span(lo, hi):   # log-uniform whole number, odd ones among them
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = max(work(c)["bytes"] for c in listed())
    while True:
        kind = rng.choice(["logprobs", "logprobs", "grad", "loss", "loss", "adamw", "adamw"])
        if kind == "adamw":
            hd, kv, grp = rng.choice([64, 128]), rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 8])
            h = span(64, 4096)
            m = rng.choice([_4B, _8B, dict(hidden=h, q_heads=kv * grp, kv_heads=kv, head_dim=hd, ffn=span(h, 4 * h), vocab=span(1000, 40000))])
            params = rng.choice(["f32", "bf16"])
            c = _adamw(None, m, rng.randint(1, 3), rng.choice(["f32", "e4m3"]), params, rng.choice(["f32", "bf16"]), embed=m["vocab"] < 50000,
                       snapshot=params == "f32" and rng.random() < 0.5)
        else:
            c = _logits(None, kind, span(1, 4096), rng.choice([151936, 32000, span(1000, 152000), span(1000, 152000)]), rng.choice(["bf16", "bf16", "f32", "f16"]),
                        pad=rng.choice([0, 0, span(1, 200)]), skipped=rng.choice([0.0, rng.uniform(0, 0.7)]), banned=rng.choice([0.0, 0.0, rng.uniform(0, 0.9)]),
                        temperature=rng.choice([1.0, 0.8, 1.3]))
            if kind == "logprobs":
                c["top_k"] = rng.choice([0, 1, rng.randint(2, 20)])
        if work(c)["bytes"] <= most:
            return c


# ---- inputs ------------------------------------------------------------------------------------------------------------

def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _logit_inputs(c, seed):
    """Background logits N(0, 2^2), the given token up to 18 above it (from hopeless to all but certain), as policies have them;
    recorded log-probabilities near the policy's own, on both sides of the clipping."""
    dev = _device()
    g = torch.Generator(device=dev).manual_seed(seed)
    R, V = c["rows"], c["vocab"]
    store = torch.empty(R, V + c["pad"], dtype=_DTYPES[c["dtype"]], device=dev)
    targets = torch.randint(0, V, (R,), generator=g, device=dev, dtype=torch.int32)
    lift = torch.rand(R, generator=g, device=dev) * 18
    lse = torch.empty(R, device=dev)
    step = max(1, (1 << 26) // V)
    for a in range(0, R, step):
        x = torch.randn(min(step, R - a), V + c["pad"], generator=g, device=dev) * 2
        if c["banned"]:
            x[torch.rand(x.shape, generator=g, device=dev) < c["banned"]] = -math.inf
        at = targets[a:a + step, None].long()
        x.scatter_(1, at, lift[a:a + step, None])
        store[a:a + step] = x.to(store.dtype)
        lse[a:a + step] = torch.logsumexp(store[a:a + step, :V].float() / c["temperature"], 1)
    logits = store[:, :V]
    lp = logits.gather(1, targets[:, None].long())[:, 0].float() / c["temperature"] - lse

    def noise(scale):
        return torch.randn(R, generator=g, device=dev) * scale

    skip = torch.rand(R, generator=g, device=dev) < c["skipped"]
    s = dict(case=c, logits=logits, lse=lse)
    if c["kind"] == "loss":
        s.update(advantages=noise(1.0), old_logprobs=lp + noise(0.15), ref_logprobs=lp + noise(0.2))
        s["sampler_logprobs"] = s["old_logprobs"] + noise(0.3)
        s["weights"] = torch.where(skip, 0.0, 0.5 + 0.5 * torch.rand(R, generator=g, device=dev))
    else:
        targets = torch.where(skip, -1, targets)
    if c["kind"] == "grad":
        s.update(grad_logprobs=noise(1.0), grad_entropy=noise(0.05))
        ent = torch.empty(R, device=dev)
        for a in range(0, R, step):
            y = logits[a:a + step].float() / c["temperature"]
            ent[a:a + step] = lse[a:a + step] - torch.nan_to_num(torch.exp(y - lse[a:a + step, None]) * y, nan=0.0).sum(1)
        s["entropy"] = ent
    s["targets"] = targets
    return s


def _tensors(c):
    """(elements, decayed) of every tensor of the decoder, in the order of a policy blob."""
    H, hd, Q, KV, F = c["hidden"], c["head_dim"], c["q_heads"] * c["head_dim"], c["kv_heads"] * c["head_dim"], c["ffn"]
    layer = [(H, False), (Q * H, True), (KV * H, True), (KV * H, True), (H * Q, True), (H, False), (F * H, True), (F * H, True), (H * F, True)]
    return ([(c["vocab"] * H, True)] if c["embed"] else []) + layer * c["layers"] + ([(H, False)] if c["embed"] else [])


def _padded(n):
    return -(-n // _BLOCK) * _BLOCK


def _adamw_inputs(c, seed):
    """Weights N(0, 0.02^2); gradients over several orders of magnitude, none for a good part of the embedding's rows, whose states
    are zero; states as some steps of such gradients leave them.  The states hold each tensor from a multiple of 256 elements on."""
    dev = _device()
    g = torch.Generator(device=dev).manual_seed(seed)
    sizes = _tensors(c)
    n, padded = sum(k for k, _ in sizes), sum(_padded(k) for k, _ in sizes)
    f8 = c["states"] == "e4m3"
    s = dict(case=c, params=torch.empty(n, dtype=_DTYPES[c["params"]], device=dev), grads=torch.empty(n, dtype=_DTYPES[c["grads"]], device=dev),
             m=torch.zeros(padded, dtype=torch.float8_e4m3fn if f8 else torch.float32, device=dev),
             v=torch.zeros(padded, dtype=torch.float8_e4m3fn if f8 else torch.float32, device=dev), step=7, seed=seed)
    if f8:
        s["m_scale"] = torch.zeros(padded // _BLOCK, device=dev)
        s["v_scale"] = torch.zeros(padded // _BLOCK, device=dev)
    s["snapshot"] = torch.zeros(n, dtype=torch.bfloat16, device=dev) if c["snapshot"] else None
    at, first = 0, 0
    for i, (k, _) in enumerate(sizes):
        step = (1 << 26) // _BLOCK * _BLOCK
        for a in range(0, k, step):
            b = min(k, a + step)
            grad = torch.randn(b - a, generator=g, device=dev) * 1e-4
            grad *= torch.exp2(3 * torch.rand(b - a, generator=g, device=dev) - 2)
            if c["embed"] and i == 0:
                grad *= ((torch.arange(a, b, device=dev) // c["hidden"]) % 8 < 3).float()
            s["params"][at + a:at + b] = (torch.randn(b - a, generator=g, device=dev) * 0.02).to(s["params"].dtype)
            s["grads"][at + a:at + b] = grad.to(s["grads"].dtype)
            past = torch.randn(_padded(b - a), generator=g, device=dev)
            past[b - a:] = 0
            past[:b - a] *= grad.abs()
            m, v = past * 0.4, past * past * 0.006
            if f8:
                for name, x in (("m", m), ("v", v)):
                    x = x.view(-1, _BLOCK)
                    scale = x.abs().amax(1) / _E4M3_MAX
                    code = (x / torch.where(scale > 0, scale, 1.0)[:, None]).to(torch.float8_e4m3fn)
                    s[name].view(torch.uint8)[first + a:first + a + code.numel()] = code.view(torch.uint8).view(-1)
                    s[name + "_scale"][(first + a) // _BLOCK:(first + a + code.numel()) // _BLOCK] = scale
            else:
                s["m"][first + a:first + b], s["v"][first + a:first + b] = m[:b - a], v[:b - a]
        at, first = at + k, first + _padded(k)
    lens = [k for k, _ in sizes]
    s["param_list"], s["grad_list"] = list(s["params"].split(lens)), list(s["grads"].split(lens))
    s["snapshot_list"] = list(s["snapshot"].split(lens)) if c["snapshot"] else None
    s["decays"] = [_DECAY if d else 0.0 for _, d in sizes]
    # about half of all steps are clipped: the largest norm allowed is what this gradient has, times 0.5 to 2
    s["max_norm"] = float(s["grads"].float().norm()) * (0.5 if seed % 2 else 2.0)
    return s


def prepare(case, seed):
    return _adamw_inputs(case, seed) if case["kind"] == "adamw" else _logit_inputs(case, seed)


# ---- the plain forms -----------------------------------------------------------------------------------------------------

def _row_statistics(y):
    """Maximum, sum of exponentials, log of the sum, probabilities and entropy of every row; a row of -inf is a distribution without weight."""
    top = y.amax(1)
    safe = torch.where(torch.isneginf(top), 0.0, top)
    e = torch.exp(y - safe[:, None])
    total = e.sum(1)
    lse = safe + torch.log(total)
    p = e / torch.where(total == 0, 1.0, total)[:, None]
    entropy = torch.where(total == 0, 0.0, lse - torch.where(p == 0, 0.0, p * y).sum(1))
    return lse, p, entropy


def _given(y, targets, lse):
    """Log-probability of the given entry of every row."""
    x = y.gather(1, targets.long().clamp(0)[:, None])[:, 0]
    return torch.where(torch.isneginf(x), x, x - lse)


def _plain_logprobs(s):
    c, targets = s["case"], s["targets"]
    x = s["logits"].float()
    y = x / c["temperature"]
    live = targets >= 0
    lse, _, entropy = _row_statistics(y)
    out = dict(logprobs=torch.where(live, _given(y, targets, lse), 0.0), entropy=torch.where(live, entropy, 0.0), lse=torch.where(live, lse, 0.0))
    if c["top_k"]:
        # one whole number per entry, larger for a larger logit and, among equal ones, for the lower index
        bits = (x + 0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * (1 << 32) + (c["vocab"] - 1 - torch.arange(c["vocab"], device=x.device))
        ids = c["vocab"] - 1 - (order.topk(c["top_k"], 1).values & 0xFFFFFFFF)
        z = y.gather(1, ids)
        out["top_ids"] = torch.where(live[:, None] & ~torch.isneginf(z), ids, -1).to(torch.int32)     # what is ruled out is no alternative
        out["top_logprobs"] = torch.where(live[:, None], torch.where(torch.isneginf(z), z, z - lse[:, None]), 0.0)
    return out


def _logit_gradient(y, p, lse, entropy, targets, live, g, h, temperature):
    """g (1[j = a] - p_j) - h p_j (ln p_j + H), over the temperature."""
    d = -p * (g[:, None] + h[:, None] * torch.where(p == 0, 0.0, y - lse[:, None] + entropy[:, None]))
    d.scatter_add_(1, targets.long().clamp(0)[:, None], g[:, None])
    return torch.where(live[:, None], d / temperature, 0.0)


def _plain_grad(s):
    c = s["case"]
    y = s["logits"].float() / c["temperature"]
    p = torch.exp(y - s["lse"][:, None])
    d = _logit_gradient(y, p, s["lse"], s["entropy"], s["targets"], s["targets"] >= 0, s["grad_logprobs"], s["grad_entropy"], c["temperature"])
    return dict(grad_logits=d.to(s["logits"].dtype))


def _plain_loss(s):
    c, w, A, old = s["case"], s["weights"], s["advantages"], s["old_logprobs"]
    y = s["logits"].float() / c["temperature"]
    live = w != 0
    lse, p, entropy = _row_statistics(y)
    logp = _given(y, s["targets"], lse)
    ratio = torch.exp(logp - old)
    correction = torch.exp(old - s["sampler_logprobs"]).clamp(max=_IS_CAP)
    free, held = ratio.clamp(max=_RATIO_CAP) * A, ratio.clamp(1 - _CLIP_LOW, 1 + _CLIP_HIGH) * A
    off = s["ref_logprobs"] - logp
    kl = torch.exp(off) - off - 1
    loss = w * (-correction * torch.minimum(free, held) + _KL * kl - _ENTROPY * entropy)
    slope = torch.where((free <= held) & (ratio < _RATIO_CAP), A * ratio, 0.0)
    g = w * (-correction * slope + _KL * (1 - torch.exp(off)))
    d = _logit_gradient(y, p, lse, entropy, s["targets"], live, g, -_ENTROPY * w, c["temperature"])
    return dict(loss=torch.where(live, loss, 0.0), logprobs=torch.where(live, logp, 0.0), entropy=torch.where(live, entropy, 0.0), grad_logits=d.to(s["logits"].dtype))


def _draws(first, n, step, seed, purpose, device):
    """16 or 32 random bits for each of the elements first .. first + n - 1 (first a multiple of 4): word i mod 4 of Philox-4x32-10 with
    counter (i / 4 in 64 bits, step, purpose) and the seed as its key (Salmon et al., SC'11)."""
    q = torch.arange(first // 4, (first + n + 3) // 4, dtype=torch.int64, device=device)
    mask = 0xFFFFFFFF
    w = [q & mask, q >> 32, torch.full_like(q, step & mask), torch.full_like(q, purpose)]
    keys = [seed & mask, (seed >> 32) & mask]

    def product(a, b):   # high and low half of a 64-bit product
        return (a * (b >> 16) + (a * (b & 0xFFFF) >> 16)) >> 16, (a * b) & mask

    for r in range(10):
        h0, l0 = product(0xD2511F53, w[0])
        h1, l1 = product(0xCD9E8D57, w[2])
        w = [h1 ^ w[1] ^ ((keys[0] + r * 0x9E3779B9) & mask), l1, h0 ^ w[3] ^ ((keys[1] + r * 0xBB67AE85) & mask), l0]
    return torch.stack(w, 1).view(-1)[:n]


def _to_e4m3(x, bits16, at_least_one):
    """Blocks of 256 values as 8-bit codes and a scale each, rounded up or down by 16 random bits; with `at_least_one`, what is positive
    keeps a positive code."""
    x = torch.nn.functional.pad(x, (0, _padded(x.numel()) - x.numel())).view(-1, _BLOCK)
    r = torch.nn.functional.pad(bits16, (0, x.numel() - bits16.numel())).view(-1, _BLOCK)
    top = x.abs().amax(1)
    scale = torch.where(top < 2.0 ** -100, 0.0, top * (1 / _E4M3_MAX))
    inv = torch.where(scale > 0, 1.0 / scale, 0.0)
    z = (x.abs() * inv[:, None]).clamp(max=_E4M3_MAX)
    normal = ((z.view(torch.int32) + (r << 4).to(torch.int32)) >> 20) - (120 << 3)
    tiny = torch.floor(z * 512 + r.float() * 2.0 ** -16).to(torch.int32)     # z < 2^-6: multiples of 2^-9
    code = torch.where(z < 2.0 ** -6, tiny, normal).clamp(max=0x7E)
    if at_least_one:
        code = torch.where((x > 0) & (scale[:, None] > 0) & (code == 0), 1, code)
    code = code | torch.where((x < 0) & (code > 0), 0x80, 0)
    return code.to(torch.uint8).view(-1).view(torch.float8_e4m3fn), scale


def _plain_adamw(s):
    c = s["case"]
    s["step"] += 1
    t = s["step"]
    norm = s["grads"].double().square().sum().sqrt().float()     # summed in 64 bits, as the operator is defined
    factor = torch.where(norm > s["max_norm"], torch.full_like(norm, s["max_norm"]) / norm, 1.0)
    size, root = _LR / (1 - _BETA1 ** t), 1 / math.sqrt(1 - _BETA2 ** t)
    first = 0
    for i, (p, grad, decay) in enumerate(zip(s["param_list"], s["grad_list"], s["decays"])):
        n = p.numel()
        whole, blocks = slice(first, first + n), slice(first // _BLOCK, (first + _padded(n)) // _BLOCK)
        g = grad.float() * factor
        if c["states"] == "f32":
            m, v = s["m"][whole], s["v"][whole]
        else:
            m, v = ((s[k][first:first + _padded(n)].float().view(-1, _BLOCK) * s[k + "_scale"][blocks, None]).view(-1)[:n] for k in ("m", "v"))
        m = m * _BETA1 + g * (1 - _BETA1)
        v = v * _BETA2 + (g * (1 - _BETA2)) * g
        new = p.float() * (1 - _LR * decay) - (m / (torch.sqrt(v) * root + _EPS)) * size
        if c["params"] == "f32":
            p.copy_(new)
        else:
            up = _draws(first, n, t, s["seed"], 1, p.device) & 0xFFFF
            p.copy_(((new.view(torch.int32) + up.to(torch.int32)) & -65536).view(torch.float32))
        if c["snapshot"]:
            s["snapshot_list"][i].copy_(new)
        if c["states"] == "f32":
            s["m"][whole], s["v"][whole] = m, v
        else:
            bits = _draws(first, n, t, s["seed"], 0, p.device)
            for k, x, r in (("m", m, bits & 0xFFFF), ("v", v, bits >> 16)):
                code, s[k + "_scale"][blocks] = _to_e4m3(x, r, k == "v")
                s[k][first:first + _padded(n)].view(torch.uint8).copy_(code.view(torch.uint8))
        first += _padded(n)
    return _adamw_outputs(s, norm)


def _adamw_outputs(s, norm):
    return {"norm": norm, **{k: s[k] for k in ("params", "m", "v", "m_scale", "v_scale", "snapshot") if s.get(k) is not None}}


# ---- one pass ------------------------------------------------------------------------------------------------------------

def run(state):
    s, c = state, state["case"]
    if not own:
        return {"logprobs": _plain_logprobs, "grad": _plain_grad, "loss": _plain_loss, "adamw": _plain_adamw}[c["kind"]](s)
    from paper_2602_02192_amd import learner
    if c["kind"] == "logprobs":
        r = learner.token_logprobs(s["logits"], s["targets"], temperature=c["temperature"], top_k=c["top_k"])
        out = dict(logprobs=r.logprobs, entropy=r.entropy, lse=r.lse)
        return dict(out, top_ids=r.top_ids, top_logprobs=r.top_logprobs) if c["top_k"] else out
    if c["kind"] == "grad":
        return dict(grad_logits=learner.token_logprobs_grad(s["logits"], s["targets"], s["lse"], s["entropy"], s["grad_logprobs"], s["grad_entropy"],
                                                            temperature=c["temperature"]))
    if c["kind"] == "loss":
        r = learner.policy_loss(s["logits"], s["targets"], s["advantages"], s["old_logprobs"], weights=s["weights"], sampler_logprobs=s["sampler_logprobs"],
                                ref_logprobs=s["ref_logprobs"], temperature=c["temperature"], clip_low=_CLIP_LOW, clip_high=_CLIP_HIGH, ratio_cap=_RATIO_CAP,
                                sampler_cap=_IS_CAP, kl_coef=_KL, entropy_coef=_ENTROPY)
        return dict(loss=r.loss, logprobs=r.logprobs, entropy=r.entropy, grad_logits=r.grad_logits)
    s["step"] += 1
    norm = learner.grad_norm(s["grad_list"])
    learner.adamw_step(s["param_list"], s["grad_list"], s["m"], s["v"], step=s["step"], lr=_LR, beta1=_BETA1, beta2=_BETA2, eps=_EPS, weight_decay=s["decays"],
                       m_scale=s.get("m_scale"), v_scale=s.get("v_scale"), snapshot=s["snapshot_list"], norm=norm, max_norm=s["max_norm"], seed=s["seed"])
    return _adamw_outputs(s, norm)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------

def work(case):
    c = case
    if c["kind"] == "adamw":
        n = sum(k for k, _ in _tensors(c))
        p, g = _SIZES[c["params"]], _SIZES[c["grads"]]
        states = 16 if c["states"] == "f32" else 4 + 16 / _BLOCK
        return {"bytes": n * (2 * p + g + states + 2 * c["snapshot"]), "flops": 18 * n}
    e, V = _SIZES[c["dtype"]], c["vocab"]
    live = c["rows"] * (1 - c["skipped"])
    if c["kind"] == "logprobs":
        return {"bytes": live * V * e + c["rows"] * (16 + 8 * c["top_k"]), "flops": 6 * live * V}
    return {"bytes": (live + c["rows"]) * V * e + c["rows"] * (24 if c["kind"] == "grad" else 36), "flops": (6 if c["kind"] == "grad" else 12) * live * V}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------------

def _exact_rows(logits, targets, temperature):
    """A row's log-sum, log-probabilities, entropy, and the given entry's log-probability."""
    z = torch.log_softmax(logits.double() / temperature, 1)
    p = z.exp()
    return z, p, -torch.special.xlogy(p, p).sum(1), z.gather(1, targets.long().clamp(0)[:, None])[:, 0]


def _exact_adamw(s):
    c = s["case"]
    t = s["step"] + 1
    norm = s["grads"].double().norm()
    factor = min(1.0, s["max_norm"] / float(norm))
    out = {k: torch.empty(s[k].numel(), dtype=torch.float64, device=s[k].device) for k in ("params", "m", "v", "m_scale", "v_scale", "snapshot") if s.get(k) is not None}
    at = first = 0
    for n, decay in zip((p.numel() for p in s["param_list"]), s["decays"]):
        pad, blocks = _padded(n), slice(first // _BLOCK, (first + _padded(n)) // _BLOCK)
        p, g = s["params"][at:at + n].double(), s["grads"][at:at + n].double() * factor
        state = {}
        for k, beta, fresh in (("m", _BETA1, g), ("v", _BETA2, g * g)):
            x = s[k][first:first + pad].double()
            if c["states"] != "f32":
                x = (x.view(-1, _BLOCK) * s[k + "_scale"][blocks, None].double()).view(-1)
            x[:n] = beta * x[:n] + (1 - beta) * fresh
            state[k] = x
        p = p - _LR * (decay * p + state["m"][:n] / (1 - _BETA1 ** t) / ((state["v"][:n] / (1 - _BETA2 ** t)).sqrt() + _EPS))
        if c["snapshot"]:
            out["snapshot"][at:at + n] = p
        if c["params"] == "bf16":
            ulp = torch.exp2(torch.floor(torch.log2(p.abs().clamp(min=2.0 ** -126))) - 7)
            p = torch.sign(p) * ulp * torch.floor(p.abs() / ulp + (_draws(first, n, t, s["seed"], 1, p.device) & 0xFFFF) / 65536.0)
        out["params"][at:at + n] = p
        bits = _draws(first, pad, t, s["seed"], 0, p.device) if c["states"] != "f32" else None
        for k, x in state.items():
            if bits is not None:
                x = x.view(-1, _BLOCK)
                scale = x.abs().amax(1) / _E4M3_MAX
                out[k + "_scale"][blocks] = scale
                x = x / torch.where(scale > 0, scale, 1.0)[:, None]
                unit = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
                up = (bits & 0xFFFF if k == "m" else bits >> 16).view(-1, _BLOCK) / 65536.0
                y = (unit * torch.floor(x.abs() / unit + up)).clamp(max=_E4M3_MAX)
                x = (torch.sign(x) * (y.clamp(min=2.0 ** -9) if k == "v" else y)).view(-1)
            out[k][first:first + pad] = x
        at, first = at + n, first + pad
    return {"norm": norm, **out}


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "adamw":
        return _exact_adamw(s)
    R, T = c["rows"], c["temperature"]
    step = max(1, (1 << 27) // c["vocab"])
    parts = []
    for a in range(0, R, step):
        cut = {k: x[a:a + step] for k, x in s.items() if isinstance(x, torch.Tensor)}
        at = cut["targets"].long().clamp(0)[:, None]
        live = cut["weights"] != 0 if c["kind"] == "loss" else cut["targets"] >= 0
        z, p, entropy, logp = _exact_rows(cut["logits"], cut["targets"], T)
        if c["kind"] == "logprobs":
            lse = torch.logsumexp(cut["logits"].double() / T, 1)
            parts.append([torch.where(live, v, 0.0) for v in (logp, entropy, lse)])
            if c["top_k"]:
                parts[-1].append(torch.where(live[:, None], z.sort(1, descending=True).values[:, :c["top_k"]], 0.0))
            continue
        if c["kind"] == "grad":
            # the recorded statistics are inputs here
            z = cut["logits"].double() / T - cut["lse"].double()[:, None]
            p, entropy = z.exp(), cut["entropy"].double()
            g, h = cut["grad_logprobs"].double(), cut["grad_entropy"].double()
            more = []
        else:
            w, A, old = (cut[k].double() for k in ("weights", "advantages", "old_logprobs"))
            r, trust = (logp - old).exp(), (old - cut["sampler_logprobs"].double()).exp().clamp(max=_IS_CAP)
            first, second = A * torch.clamp(r, max=_RATIO_CAP), A * torch.clamp(r, 1 - _CLIP_LOW, 1 + _CLIP_HIGH)
            away = cut["ref_logprobs"].double() - logp
            loss = w * (_KL * (torch.expm1(away) - away) - trust * torch.minimum(first, second) - _ENTROPY * entropy)
            g = w * (-trust * A * r * ((first <= second) & (r < _RATIO_CAP)) - _KL * torch.expm1(away))
            h = -_ENTROPY * w
            more = [torch.where(live, v, 0.0) for v in (loss, logp, entropy)]
        d = torch.zeros_like(p).scatter_(1, at, g[:, None]) - p * g[:, None] - h[:, None] * (torch.special.xlogy(p, p) + p * entropy[:, None])
        parts.append(more + [torch.where(live[:, None], d / T, 0.0)])
    got = [torch.cat(x) for x in zip(*parts)]
    names = {"logprobs": ["logprobs", "entropy", "lse", "top_logprobs"], "grad": ["grad_logits"], "loss": ["loss", "logprobs", "entropy", "grad_logits"]}[c["kind"]]
    out = dict(zip(names, got))
    return dict(out, top_ids=None) if c["kind"] == "logprobs" and c["top_k"] else out
