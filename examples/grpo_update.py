"""The paper's loop on one GPU at the size of the tiny model: rollouts under a snapshot, advantages, the learner's loss and gradient, the
update, the next snapshot.

    python examples/grpo_update.py [updates]

A policy of random weights answers prompts; the reward of an answer is the share of its tokens from the lower half of the vocabulary, so the mean
reward starts near one half and grows.  The network itself is a plain torch decoder over float32 master weights (the learner's
own business); everything between its logits and the snapshot that the rollout side installs is the library's."""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2602_02192_amd import echo, learner, synth  # noqa: E402

SHAPE = synth.TINY.replace(dtype="bf16")
PROMPTS, G, PROMPT_LEN, NEW, TURN = 8, 8, 24, 32, 7
LR, MAX_NORM, KL, ENTROPY = 2e-3, 1.0, 0.01, 0.001


def rms_norm(x, gain):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + SHAPE.rms_eps) * gain


def rotary(x):
    """x [sequences, length, heads, head_dim]: element i of the first half turns with element i of the second."""
    L, half = x.shape[1], SHAPE.head_dim // 2
    angle = torch.arange(L, device=x.device)[:, None] * SHAPE.rope_base ** (-torch.arange(half, device=x.device) / half)
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)


def forward(w, tokens):
    """Logits of the next token at every position, [sequences, length, vocab]."""
    N, L = tokens.shape
    hd, group = SHAPE.head_dim, SHAPE.n_q_heads // SHAPE.n_kv_heads
    causal = torch.full((L, L), float("-inf"), device=tokens.device).triu(1)
    h = w["embed"][tokens]
    for i in range(SHAPE.n_layers):
        p = f"layers.{i}."
        x = rms_norm(h, w[p + "attn_norm"])
        q, k, v = ((x @ w[p + n].t()).view(N, L, -1, hd) for n in ("wq", "wk", "wv"))
        q, k = rotary(q).transpose(1, 2), rotary(k).transpose(1, 2).repeat_interleave(group, 1)
        v = v.transpose(1, 2).repeat_interleave(group, 1)
        a = torch.softmax(q @ k.transpose(2, 3).contiguous() * hd ** -0.5 + causal, -1) @ v
        h = h + a.transpose(1, 2).reshape(N, L, -1) @ w[p + "wo"].t()
        x = rms_norm(h, w[p + "ffn_norm"])
        h = h + (torch.nn.functional.silu(x @ w[p + "w_gate"].t()) * (x @ w[p + "w_up"].t())) @ w[p + "w_down"].t()
    return rms_norm(h, w["final_norm"]) @ w["lm_head"].t()


class Learner:
    """Master weights, optimiser and the flat bf16 blob that is published."""

    def __init__(self, blob, seed):
        self.blob = blob.cuda()      # in the order of echo_load_policy
        self.w, views, decay = {}, [], []
        for name, (at, shape) in synth.blob_offsets(SHAPE).items():
            view = self.blob[at:at + int(np.prod(shape))]
            self.w[name] = view.float().view(shape).requires_grad_(True)
            views.append(view)
            decay.append(0.0 if len(shape) == 1 else 0.01)
        self.optimiser = learner.AdamW(list(self.w.values()), LR, weight_decay=decay, max_norm=MAX_NORM, snapshot=views, seed=seed)

    def update(self, tokens, lens, mask, advantages, sampler_logprobs, reference_logprobs):
        """One step on a batch of records; host arrays [sequences, length].  Returns numbers to look at."""
        N, L = tokens.shape
        on_gpu = lambda a, dt: torch.from_numpy(np.ascontiguousarray(a[:, 1:]).reshape(-1)).to("cuda", dt)  # noqa: E731
        targets, mine = on_gpu(tokens, torch.int32), on_gpu(mask, torch.float32)
        weights = mine / mine.sum().clamp(min=1)
        logits = forward(self.w, torch.from_numpy(tokens).long().cuda())[:, :-1].reshape(N * (L - 1), -1)
        now = learner.token_logprobs(logits.detach(), targets)
        out = learner.policy_loss(logits.detach(), targets, on_gpu(advantages, torch.float32), now.logprobs, weights=weights,
                                  sampler_logprobs=on_gpu(sampler_logprobs, torch.float32), ref_logprobs=on_gpu(reference_logprobs, torch.float32),
                                  sampler_cap=2.0, kl_coef=KL, entropy_coef=ENTROPY)
        for p in self.w.values():
            p.grad = None
        logits.backward(out.grad_logits)
        norm = self.optimiser.step()
        off = (now.logprobs - on_gpu(sampler_logprobs, torch.float32)).abs() * mine
        return dict(loss=float(out.loss.sum()), entropy=float((now.entropy * mine).sum() / mine.sum()), grad_norm=float(norm), largest_ratio=float(off.max().exp()))


def records(prompts, out):
    """Prompts and answers as records [sequences, length], with the sampler's log-probabilities at the tokens it drew."""
    tokens = np.concatenate([np.repeat(prompts, G, axis=0), np.where(out["tokens"] < 0, 0, out["tokens"])], axis=1)
    lens = PROMPT_LEN + out["lens"]
    sampled = np.zeros(tokens.shape, np.float32)
    sampled[:, PROMPT_LEN:] = out["logprobs"]
    return tokens.astype(np.int32), lens.astype(np.int32), sampled


def main(updates: int = 12, seed: int = 0, say=print):
    blob = synth.make_weights(SHAPE, seed)
    ctx = echo.Context(echo.desc_from_shape(SHAPE, PROMPTS * G, PROMPT_LEN + NEW))
    ctx.load_policy(0, blob)
    # the first snapshot stays the reference policy of the divergence
    reference = echo.Context(echo.desc_from_shape(SHAPE, PROMPTS * G, PROMPT_LEN + NEW))
    reference.load_policy(0, blob)
    me, history = Learner(blob, seed), []
    for step in range(updates):
        prompts, plens = synth.make_prompts(SHAPE.vocab, PROMPTS, PROMPT_LEN, seed=seed + step)
        prompts[prompts == TURN] += 1
        prompts[:, [0, 4, PROMPT_LEN - 1]] = TURN      # system turn, user's turn, and the answer's turn begins
        out = ctx.rollout(prompts, plens, G, NEW, 1.0, seed=1000 * seed + step)
        rewards = np.where(out["tokens"] >= 0, out["tokens"] < SHAPE.vocab // 2, 0).sum(1) / out["lens"]
        tokens, lens, sampled = records(prompts, out)
        mask, _, advantages = ctx.grpo_tensors(tokens, lens, G, TURN, rewards)
        mask[:, :PROMPT_LEN] = 0                        # (the token that begins the turn is not the policy's)
        seen = me.update(tokens, lens, mask, advantages, sampled, reference.logprobs(tokens, lens))
        ctx.load_policy(step + 1, me.blob.cpu())        # the next version
        history.append(dict(seen, reward=float(rewards.mean()), version=int(ctx.stats().active_version)))
        say(f"update {step}: reward {history[-1]['reward']:.3f}  loss {seen['loss']:+.4f}  entropy {seen['entropy']:.3f}  gradient norm {seen['grad_norm']:.3f}  "
            f"learner and sampler apart by a factor of {seen['largest_ratio']:.4f} at most")
    # the learner's log-probabilities of a batch against those of the snapshot it published
    theirs = ctx.logprobs(tokens, lens)
    with torch.no_grad():
        logits = forward(me.w, torch.from_numpy(tokens).long().cuda())[:, :-1].reshape(len(tokens) * (tokens.shape[1] - 1), -1)
    ours = learner.token_logprobs(logits, torch.from_numpy(np.ascontiguousarray(tokens[:, 1:]).reshape(-1)).cuda()).logprobs.cpu().numpy().reshape(len(tokens), -1)
    live = np.arange(1, tokens.shape[1])[None] < lens[:, None]
    apart = float(np.abs(np.where(live, ours - theirs[:, 1:], 0)).max())
    say(f"log-probabilities of the learner and of its published snapshot differ by {apart:.4f} at most")
    ctx.close()
    reference.close()
    return history, apart


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 12)
