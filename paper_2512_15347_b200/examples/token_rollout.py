"""Expand-and-Prune on a token policy, end to end on one GPU: G prompts enter a paged cache, are expanded to
N trajectories each, decode with one attention call per layer and step, are pruned to k with Optimal
Variance Filtering half-way, finish, get their group-relative advantages and give the gradient of one policy update.

The policy is a small random-weight transformer stand-in (queries, keys, values and logits are plain torch
products); what the library does is the cache, the attention, the sampling rules, the selection, the
advantages and the update from the logits to their gradient.  The library has no attention of several new tokens of a row, and the stand-in none for its prompts: their keys
and values of every layer are products of the embeddings alone, not of what the layers before make of them.  A policy in earnest
runs its own prompt pass there and appends what it gives.  `python -m paper_2512_15347_b200.examples.token_rollout`
"""
from __future__ import annotations

import math

import torch

from .. import binding as B
from ..kvcache import PagedCache
from ..token_update import TokenUpdate, score


class Policy:
    """Random weights of a decoder without positions or feed-forward layers; enough to drive the calls."""

    def __init__(self, layers=2, q_heads=8, kv_heads=2, dim=64, vocab=1000, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: (torch.randn(*s, generator=g, device="cuda") / math.sqrt(s[0])).to(dtype)
        self.width, self.q_heads, self.kv_heads, self.dim, self.vocab = q_heads * dim, q_heads, kv_heads, dim, vocab
        self.embed = (torch.randn(vocab, self.width, generator=g, device="cuda")).to(dtype)
        self.qkv = [rnd(self.width, (q_heads + 2 * kv_heads) * dim) for _ in range(layers)]
        self.proj = [rnd(self.width, self.width) for _ in range(layers)]
        self.head = rnd(self.width, vocab)

    def split(self, layer, x):
        """q, k, v of [tokens, width] as slices of one product."""
        y = (x @ self.qkv[layer]).view(x.shape[0], -1, self.dim)
        return y[:, : self.q_heads], y[:, self.q_heads: self.q_heads + self.kv_heads], y[:, self.q_heads + self.kv_heads:]

    def logits(self, x):
        return x @ self.head


def decode(policy, cache, tokens):
    """One step of all rows: their newest tokens [rows] in, logits [rows, vocab] out."""
    x = policy.embed[tokens.long()]
    for layer in range(len(policy.qkv)):
        q, k, v = policy.split(layer, x)
        a = cache.attend(layer, q, k, v)
        x = x + a.reshape(x.shape[0], -1) @ policy.proj[layer]
    return policy.logits(x)


def rollout(policy, prompts, n_expand, n_keep, steps, prune_at, page_size=16, seed=0, temperature=0.9, repetition=1.1, frequency=0.1):
    """prompts: list of int32 token tensors.  -> (tokens [rows, steps] of the survivors, log-probs, advantages, kept, cache)."""
    dev, G = "cuda", len(prompts)
    layers = len(policy.qkv)
    lens = torch.tensor([p.numel() for p in prompts], device=dev, dtype=torch.int32)
    longest = int(lens.max())
    rows = G * n_expand
    per_row = -(-(longest + steps) // page_size)
    cache = PagedCache(G * per_row + rows * (2 + -(-steps // page_size)), page_size, layers, policy.kv_heads, policy.dim, rows,
                       longest + steps, policy.embed.dtype)
    g = torch.Generator(device=dev).manual_seed(seed)

    # prompts: their keys and values from the embeddings (all but each one's last token, which the first step brings)
    cache.admit(G)
    cache.extend(lens - 1)
    start = torch.cat([lens.new_zeros(1), torch.cumsum(lens - 1, 0).to(torch.int32)])
    x = policy.embed[torch.cat([p[:-1] for p in prompts]).long()]
    for layer in range(layers):
        _, k, v = policy.split(layer, x)
        cache.append(layer, k, v, start)
    cache.expand(n_expand)

    fan = n_expand
    history = torch.full((rows, longest + steps), -1, device=dev, dtype=torch.int32)
    for i, p in enumerate(prompts):
        history[i * fan: (i + 1) * fan, longest - p.numel(): longest] = p
    made = torch.zeros((rows, steps), device=dev, dtype=torch.int32)
    logp = torch.zeros((rows, steps), device=dev)
    newest = history[:, longest - 1].contiguous()
    h = B.rollout_init(B.make_config(G, n_expand, 4, 2, [(0, n_keep)], seed, B.VEL_F32))
    keep = None
    try:
        for s in range(steps):
            if s == prune_at:
                # the stand-in for a reward model on the partial rollouts: their mean log-prob
                score = logp[:, :s].mean(1).contiguous()
                keep, src = (torch.empty(G * n_keep, device=dev, dtype=torch.int32) for _ in range(2))
                B.prune_ovf(h, 0, score, keep, src)
                cache.prune(src, n_keep)
                idx = src.long()
                history, made, logp, newest, fan = history[idx].contiguous(), made[idx].contiguous(), logp[idx].contiguous(), newest[idx], n_keep
            cache.extend(1)
            raw = decode(policy, cache, newest)
            n = raw.shape[0]
            full = torch.full((n,), longest + s, device=dev, dtype=torch.int32)
            rules = B.make_logits_rules(tokens=history, n_tokens=full, n_prompt=torch.full_like(full, longest),
                                        repetition=torch.full((n,), repetition, device=dev), frequency=torch.full((n,), frequency, device=dev),
                                        temperature=torch.full((n,), temperature, device=dev))
            out = torch.empty(raw.shape, device=dev)
            B.logits_process(raw, out, rules)
            lp = torch.log_softmax(out, -1)
            noise = -torch.log(-torch.log(torch.rand(out.shape, generator=g, device=dev).clamp_(1e-9, 1 - 1e-7)))
            newest = (lp + noise).argmax(-1).to(torch.int32)
            made[:, s] = newest
            logp[:, s] = lp.gather(1, newest[:, None].long())[:, 0]
            history[:, longest + s] = newest
        rewards = logp.mean(1).contiguous()
        adv = torch.empty_like(rewards)
        B.advantages(h, rewards, adv)
        cache.check()
    finally:
        torch.cuda.synchronize()
        B.rollout_destroy(h)
    return made, logp, adv, keep, cache


def hidden(policy, prompt, made):
    """States [steps, width] from which a survivor's made tokens were drawn, all positions at once: the stand-in's pass with the
    made tokens given, in plain torch products."""
    n0, d = prompt.numel() - 1, policy.dim
    tokens = torch.cat([prompt, made])[:-1].long()
    first = policy.embed[tokens]
    x = first
    causal = torch.ones(tokens.numel(), tokens.numel(), device=x.device, dtype=torch.bool).tril()
    per = policy.q_heads // policy.kv_heads
    for layer in range(len(policy.qkv)):
        q, k, v = policy.split(layer, x)
        _, k0, v0 = policy.split(layer, first)       # prompt tokens but the last enter the cache from their embeddings alone
        k, v = (torch.cat([b[:n0], a[n0:]]).repeat_interleave(per, 1).float() for a, b in ((k, k0), (v, v0)))
        s = torch.einsum("thd,uhd->htu", q.float(), k) / math.sqrt(d)
        a = torch.softmax(s.masked_fill(~causal, -math.inf), -1)
        x = x + torch.einsum("htu,uhd->thd", a, v).to(x.dtype).reshape(x.shape[0], -1) @ policy.proj[layer]
    return x[n0:]


def update(policy, prompts, made, logp, adv, reference=None, temperature=0.9, n_top=20, entropy_coef=0.01, distill_coef=0.1):
    """One update step on the survivors: the objective of their tokens at the rollout's temperature, with an entropy bonus and the
    divergence from a reference policy known by its n_top likeliest tokens a position (None: this policy before the step).
    -> (what TokenUpdate.step gives, gradient of the objective to policy.head, states [tokens, width])."""
    keep = made.shape[0] // len(prompts)
    x = torch.cat([hidden(policy, prompts[r // keep], made[r]) for r in range(made.shape[0])])
    n, dev = x.shape[0], x.device
    logits = policy.logits(x)
    start = torch.arange(0, n + 1, made.shape[1], device=dev, dtype=torch.int32)
    tau = torch.full((n,), temperature, device=dev)
    teacher = score((reference or policy).logits(x), n_top=n_top, temperature=tau)
    rule = TokenUpdate(clip_high=0.28, entropy_coef=entropy_coef, distill_coef=distill_coef, kind="reverse_rest", norm="tokens")
    u = rule.step(logits, made.reshape(-1).contiguous(), start, adv, logp.reshape(-1).contiguous(), teacher=(teacher.top_ids, teacher.top_logp),
                  temperature=tau)
    rule.check()
    return u, x.T @ u.dlogits, x


def main():
    g = torch.Generator(device="cuda").manual_seed(1)
    policy = Policy()
    prompts = [torch.randint(0, policy.vocab, (n,), generator=g, device="cuda", dtype=torch.int32) for n in (37, 120, 200, 75)]
    made, logp, adv, keep, cache = rollout(policy, prompts, n_expand=16, n_keep=8, steps=24, prune_at=12)
    print(f"{len(prompts)} prompts x 16 -> 8: tokens {tuple(made.shape)}, mean log-prob {logp.mean().item():.3f}")
    print("kept slots of the first group:", keep[:8].tolist())
    print("advantages of the first group:", [round(a, 3) for a in adv[:8].tolist()])
    print(f"pages in use: {int((cache.refs > 0).sum())} of {cache.refs.numel()}")
    # an update on trajectories that were drawn from the policy at its temperature alone
    made, logp, adv, _, _ = rollout(policy, prompts, n_expand=16, n_keep=8, steps=24, prune_at=12, repetition=1.0, frequency=0.0)
    u, grad, _ = update(policy, prompts, made, logp, adv)
    print(f"update: objective {u.objective.item():+.4f}, entropy {u.entropy.mean().item():.3f}, clipped {u.stats[4].item():.3f}, "
          f"gradient to the head {grad.float().norm().item():.4f}")


if __name__ == "__main__":
    main()
