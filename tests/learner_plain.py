"""The learner's operators in numpy, from their formulas: rows of logits in 64 bits, the AdamW step in 64 bits and, operation by
operation, in 32.  Test infrastructure; shares no code with the library."""
import numpy as np

BLOCK = 256


def rows(x, targets, T, top_k=0, live=None):
    """x float64 [R, V] -> dict of logprobs, entropy, lse, p [R, V], top_ids, top_logprobs."""
    R, V = x.shape
    if live is None:
        live = np.ones(R, bool) if targets is None else (targets >= 0) & (targets < V)
    out = dict(logprobs=np.zeros(R), entropy=np.zeros(R), lse=np.zeros(R), p=np.zeros((R, V)), live=live,
               top_ids=np.full((R, top_k), -1), top_logprobs=np.zeros((R, top_k)))
    for t in range(R):
        if not live[t]:
            continue
        y = x[t] / T
        m = y.max()
        if m == -np.inf:
            out["lse"][t] = out["logprobs"][t] = -np.inf
            out["top_logprobs"][t] = -np.inf
            continue
        e = np.exp(y - m)
        lse = m + np.log(e.sum())
        p = np.exp(y - lse)
        out["lse"][t], out["p"][t] = lse, p
        has = p > 0
        out["entropy"][t] = -(p[has] * (y[has] - lse)).sum()
        if targets is not None:
            out["logprobs"][t] = y[targets[t]] - lse
        order = np.argsort(-x[t], kind="stable")[:top_k]
        for k, j in enumerate(order):
            out["top_ids"][t, k] = j if y[j] > -np.inf else -1
            out["top_logprobs"][t, k] = y[j] - lse
    return out


def tolerance(x, T):
    """How far a log-sum of f32 arithmetic may be from the exact one.  In units of ln 2 the terms are x c - ref with two roundings in c, one in
    ref and one in the fma, each relative to at most the largest |x c|; exp2 and log2 are good to 2 ulp; a sum of V terms in parts
    of V / 256 and a tree loses at most V / 256 + 16 roundings; the result is scaled once more."""
    finite = np.where(np.isfinite(x), np.abs(x), 0).max(axis=1) / T * 1.4427
    return 2.0 ** -24 * (10 * finite + x.shape[1] / 256 + 64)


def logit_gradient(r, targets, g, h, T):
    """Gradient rows for d/dlogprob = g and d/dentropy = h, and the size of the terms it is made of."""
    p, R = r["p"], len(g)
    lnp = np.log(np.where(p > 0, p, 1.0))
    d = -p * (g[:, None] + h[:, None] * (lnp + r["entropy"][:, None]))
    size = p * (np.abs(g)[:, None] + np.abs(h)[:, None] * (np.abs(lnp) + r["entropy"][:, None]))
    if targets is not None:
        ok = r["live"] & np.isfinite(r["lse"])
        d[np.arange(R)[ok], targets[ok]] += g[ok]
        size[np.arange(R)[ok], targets[ok]] += np.abs(g[ok])
    dead = ~r["live"] | (r["lse"] == -np.inf)
    d[dead] = 0
    size[dead] = 0
    return d / T, size / T


def token_loss(lp, H, A, old, w, sampler, ref, o):
    """(loss, dloss/dlogprob, dloss/dentropy) of one token; o: the coefficients by name."""
    r = np.exp(lp - old)
    c = min(np.exp(old - sampler), o["sampler_cap"]) if sampler is not None else 1.0
    free, held = min(r, o["ratio_cap"]) * A, min(max(r, 1 - o["clip_low"]), 1 + o["clip_high"]) * A
    loss, g = -c * min(free, held) - o["entropy_coef"] * H, 0.0
    if free <= held and r < o["ratio_cap"]:
        g = -c * A * r
    if o["kl_coef"]:
        k = ref - lp
        loss += o["kl_coef"] * (np.exp(k) - k - 1)
        g += o["kl_coef"] * (1 - np.exp(k))
    return w * loss, w * g, -w * o["entropy_coef"]


def philox(first, n, step, purpose, seed):
    """Words of Philox-4x32-10 for elements first .. first + n - 1: word i mod 4 for counter (i / 4, step, purpose), key seed."""
    i = np.arange(first, first + n, dtype=np.uint64)
    q = i // 4
    M = np.uint64(0xFFFFFFFF)
    c = [q & M, q >> np.uint64(32), np.full(n, step, np.uint64), np.full(n, purpose, np.uint64)]
    k = [np.uint64(seed & 0xFFFFFFFF), np.uint64(seed >> 32)]
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> np.uint64(32)) ^ c[1] ^ k[0], b & M, (a >> np.uint64(32)) ^ c[3] ^ k[1], a & M]
        k = [(k[0] + np.uint64(0x9E3779B9)) & M, (k[1] + np.uint64(0xBB67AE85)) & M]
    return np.choose((i % 4).astype(np.int64), c).astype(np.uint32)


E4M3 = np.array([(-1.0 if c & 0x80 else 1.0) * (np.nan if c & 0x7F == 0x7F else (c & 7) * 2.0 ** -9 if c & 0x78 == 0 else (8 + (c & 7)) * 2.0 ** ((c >> 3 & 15) - 10))
                 for c in range(256)], np.float32)


def encode(x, bits, keep):
    """f32 values (a multiple of BLOCK) -> (codes, scales), by the definition: the two neighbouring codes of |x| / scale, the upper one where the
    16 bits exceed what is missing to it."""
    f = np.float32
    x = x.reshape(-1, BLOCK)
    bits = bits.reshape(-1, BLOCK)
    top = np.abs(x).max(1)
    scale = np.where(top < f(2.0 ** -100), f(0), top * f(1 / 448))
    inv = np.divide(f(1), scale, out=np.zeros_like(scale), where=scale > 0)
    z = np.minimum(np.abs(x) * inv[:, None], f(448)).astype(np.float64)
    unit = 2.0 ** (np.floor(np.log2(np.maximum(z, 2.0 ** -6))) - 3)
    low = np.where(z < 2.0 ** -6, np.floor((z / unit).astype(f) + bits * f(2.0 ** -16)), np.floor(z / unit + bits / 65536.0)) * unit
    values = E4M3[:0x7F].astype(np.float64)
    code = np.searchsorted(values, np.minimum(low, 448.0))
    assert np.array_equal(values[code], np.minimum(low, 448.0))
    if keep:
        code[(x > 0) & (code == 0) & (scale > 0)[:, None]] = 1
    code |= np.where((x < 0) & (code > 0), 0x80, 0)
    return code.astype(np.uint8).reshape(-1), scale


def adamw(p, g, m, v, decay, lr, beta1, beta2, eps, step, factor, dtype=np.float32):
    """One tensor's step in `dtype`, an operation at a time: (p, m, v)."""
    f = dtype
    g = g.astype(f) * f(factor)
    m = m * f(beta1) + g * f(1 - beta1)
    v = v * f(beta2) + g * f(1 - beta2) * g
    den = np.sqrt(v) * f(1 / np.sqrt(1 - beta2 ** step)) + f(eps)
    return p.astype(f) * f(1 - lr * decay) - m / den * f(lr / (1 - beta1 ** step)), m, v


def to_bf16(x):
    """f32 -> nearest bf16 (even), as bits."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32)
    return ((u + np.uint32(0x7FFF) + ((u >> np.uint32(16)) & np.uint32(1))) >> np.uint32(16)).astype(np.uint16)


def from_bf16(b):
    return (b.astype(np.uint32) << np.uint32(16)).view(np.float32)
