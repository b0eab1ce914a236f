"""The cache driver and the token-rollout example: the paged, forked, pruned path against the same policy
with every trajectory's keys and values recomputed from its tokens."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_example_rollout_agrees_with_recomputation():
    from paper_2512_15347_b200.examples import token_rollout as T
    g = torch.Generator(device="cuda").manual_seed(3)
    policy = T.Policy(layers=2, q_heads=8, kv_heads=2, dim=64, vocab=500)
    prompts = [torch.randint(0, policy.vocab, (n,), generator=g, device="cuda", dtype=torch.int32) for n in (33, 150, 96)]
    made, logp, adv, keep, cache = T.rollout(policy, prompts, n_expand=16, n_keep=8, steps=20, prune_at=9, seed=4)
    assert made.shape == (24, 20) and torch.isfinite(logp).all() and (logp <= 0).all()
    assert adv.view(3, 8).mean(1).abs().max() < 1e-4
    # recompute every survivor's log-probs with plain attention in fp32
    for r in range(24):
        p = prompts[r // 8]
        tokens = torch.cat([p, made[r]])
        x = policy.embed[tokens.long()].float()
        T_all = tokens.numel()
        causal = torch.ones(T_all, T_all, device="cuda", dtype=torch.bool).tril()
        prompt_x = policy.embed[tokens.long()]
        for layer in range(2):
            y = (x.to(torch.bfloat16) @ policy.qkv[layer]).view(T_all, -1, 64)
            q = y[:, :8].float()
            # prompt tokens but the last enter the cache from their embeddings alone (the example's stand-in)
            y0 = (prompt_x @ policy.qkv[layer]).view(T_all, -1, 64)
            n0 = p.numel() - 1
            k = torch.cat([y0[:n0, 8:10], y[n0:, 8:10]]).float().repeat_interleave(4, 1)
            v = torch.cat([y0[:n0, 10:], y[n0:, 10:]]).float().repeat_interleave(4, 1)
            s = torch.einsum("thd,uhd->htu", q, k) / 8.0
            a = torch.softmax(s.masked_fill(~causal, -math.inf), -1)
            o = torch.einsum("htu,uhd->thd", a, v).to(torch.bfloat16)
            x = (x.to(torch.bfloat16) + o.reshape(T_all, -1) @ policy.proj[layer]).float()
        raw = policy.logits(x.to(torch.bfloat16))[p.numel() - 1: -1].float()
        n = p.numel()
        want = []
        for s in range(20):
            z = raw[s].clone()
            seen = torch.bincount(tokens[: n + s].long(), minlength=500) > 0
            count = torch.bincount(tokens[n: n + s].long(), minlength=500).float()
            z = torch.where(seen, torch.where(z > 0, z / 1.1, z * 1.1), z) - 0.1 * count
            want.append(torch.log_softmax(z / 0.9, -1)[tokens[n + s].long()])
        got = logp[r]
        # bf16 logits of size ~ 4 carry roundings of ~ 0.02 each, and so do the activations: two computations of one number
        assert (got - torch.stack(want)).abs().max() < 0.5
        assert (got - torch.stack(want)).abs().mean() < 0.08


def test_driver_keeps_counts_and_refuses():
    from paper_2512_15347_b200 import binding as B
    from paper_2512_15347_b200.kvcache import PagedCache
    c = PagedCache(64, 16, 2, 2, 64, 32, 256)
    c.admit(2)
    c.extend(torch.tensor([40, 17], device="cuda", dtype=torch.int32))
    assert c.len.tolist() == [40, 17] and int((c.refs > 0).sum()) == 5
    c.expand(8)
    assert c.n_rows == 16 and c.group == 8 and c.shared.tolist() == [32, 16]
    assert int((c.refs > 0).sum()) == 5 + 14 and int(c.refs[c.table[0, 0]]) == 8
    q = torch.randn(16, 4, 64, device="cuda", dtype=torch.bfloat16)
    kv = torch.randn(16, 2, 64, device="cuda", dtype=torch.bfloat16)
    c.extend(1)
    out = c.attend(1, q, kv, kv)
    assert torch.isfinite(out).all()
    c.prune(torch.tensor([1, 3, 8, 15], device="cuda", dtype=torch.int32), 2)
    assert c.len.tolist() == [41, 41, 18, 18] and c.group == 2
    assert int(c.refs[c.table[0, 0]]) == 2
    c.pack()
    live = int((c.refs > 0).sum())
    assert (c.refs[:live] > 0).all() and (c.refs[live:] == 0).all()
    c.check()
    with pytest.raises(ValueError):
        c.prune(torch.zeros(3, device="cuda", dtype=torch.int32), 2)
    with pytest.raises(ValueError):
        c.expand(64)
    c.extend(16 * 60)
    with pytest.raises(B.PgError) as e:
        c.check()
    assert e.value.code == B.ENOPAGES
    c.status.zero_()
    c.admit(1)
    assert (c.refs == 0).all() and c.n_rows == 1
