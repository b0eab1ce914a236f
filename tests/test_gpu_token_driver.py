"""The update driver and the example's update step: the calls together, as a trainer makes them."""
import ctypes
import math

import pytest
import torch

from tests import token_reference as ref
from tests.test_gpu_token_update import HALF_STEP, SUM, U, check_gradient, make, reference, tiles_of

pytestmark = pytest.mark.gpu


def check_update(u, c, adv, old, start, kind, rule):
    J, dlogp, weight, _, _ = ref.objective(start, u.logp, adv, old=old, entropy=u.entropy, distill=u.distill, **rule)
    assert abs(float(u.objective) - J) <= 2 * U * abs(J) + 1e-9
    w = torch.tensor(weight, device="cuda", dtype=torch.float64)
    c = dict(c, dlogp=torch.tensor(dlogp, device="cuda")[:, None], dentropy=rule["entropy_coef"] * w, ddistill=-rule["distill_coef"] * w)
    check_gradient(c, u.dlogits, reference(c, kind))
    assert torch.allclose(u.weight.double(), w, rtol=1e-7, atol=0)


@pytest.mark.parametrize("kind", ["forward", "forward_rest", "reverse_rest"])
def test_driver_scores_steps_and_checks(kind):
    from paper_2512_15347_b200 import binding as B
    from paper_2512_15347_b200.token_update import TokenUpdate, score
    V, lens = 9001, [3, 0, 7, 2]
    n = sum(lens)
    c = make(n, V, torch.bfloat16, 3, masks=False)
    teacher = (c["x"].float() + torch.randn(c["x"].shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))).to(torch.bfloat16)
    lists = score(teacher, n_top=16, temperature=c["tau"])
    assert lists.logp is None and lists.top_ids.shape == (n, 16)
    own = score(c["x"], c["ids"], temperature=c["tau"])
    c["list_ids"], c["list_logp"] = lists.top_ids, lists.top_logp
    start = torch.tensor([0] + [sum(lens[: i + 1]) for i in range(4)], device="cuda", dtype=torch.int32)
    adv = torch.tensor([1.0, 3.0, -0.5, 0.25], device="cuda")
    old = (own.logp[:, 0] + 0.1 * torch.randn(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))).contiguous()
    rule = TokenUpdate(clip_high=0.25, entropy_coef=0.125, distill_coef=0.5, kind=kind)
    u = rule.step(c["x"], c["ids"].view(-1), start, adv, old, teacher=(lists.top_ids, lists.top_logp), temperature=c["tau"])
    # with a bucket the list's logits are summed apart from the others: the same terms in another order
    few = U * 2 * (SUM + 16 * tiles_of(V, torch.bfloat16))
    assert (u.logp - own.logp[:, 0]).abs().max() <= (0 if kind == "forward" else few * 2)
    assert ((u.entropy - own.entropy).abs() <= (0 if kind == "forward" else few * (1 + 3 * own.entropy))).all()
    f = lambda v: ctypes.c_float(v).value
    check_update(u, c, adv, old, start, kind, dict(clip_low=f(0.2), clip_high=f(0.25), entropy_coef=0.125, distill_coef=0.5))
    rule.check()
    # the same step captured, replayed on other logits, beside one on another stream
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        g = rule.step(c["x"], c["ids"].view(-1), start, adv, old, teacher=(lists.top_ids, lists.top_logp), temperature=c["tau"])
    kept = u.dlogits.clone()
    with torch.cuda.stream(side):
        again = rule.step(c["x"], c["ids"].view(-1), start, adv, old, teacher=(lists.top_ids, lists.top_logp), temperature=c["tau"])
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(g.dlogits, kept) and torch.equal(again.dlogits, kept)
    # in place, without a teacher
    plain = TokenUpdate(clip_low=0.1, norm="sum")
    x = c["x"].clone()
    u = plain.step(x, c["ids"].view(-1), start, adv, old, temperature=c["tau"], dlogits=x)
    assert u.dlogits is x and u.distill is None
    c.pop("list_ids")
    check_update(u, c, adv, old, start, "forward", dict(clip_low=f(0.1), clip_high=f(0.2), entropy_coef=0.0, distill_coef=0.0, norm="sum"))
    for bad in (lambda: rule.step(c["x"], c["ids"].view(-1), start, adv, old), lambda: TokenUpdate(kind="other"), lambda: TokenUpdate(norm="mean"),
                lambda: TokenUpdate(beta=0.1).step(c["x"], c["ids"].view(-1), start, adv, old),
                lambda: plain.step(c["x"], c["ids"].view(-1)[:3], start, adv, old)):
        with pytest.raises(ValueError):
            bad()
    start[2] = 99
    plain.step(c["x"], c["ids"].view(-1), start, adv, old)
    with pytest.raises(B.PgError):
        plain.check()


def test_padded_batch_and_no_tokens():
    from paper_2512_15347_b200.token_update import TokenUpdate, score
    V, n, used = 5003, 16, 12
    c = make(n, V, torch.bfloat16, 8, masks=False)
    c["x"][used:] = math.nan                                       # what lies behind the last row's tokens
    c["ids"][used + 1:] = -1
    lists = score(torch.nan_to_num(c["x"]), n_top=10, temperature=c["tau"])
    c["list_ids"], c["list_logp"] = lists.top_ids, lists.top_logp
    start = torch.tensor([0, 3, 3, 10, used], device="cuda", dtype=torch.int32)
    adv = torch.tensor([1.0, 3.0, -0.5, 0.25], device="cuda")
    old = score(c["x"], c["ids"], temperature=c["tau"]).logp[:, 0].contiguous()
    rule = TokenUpdate(entropy_coef=0.125, distill_coef=0.5, kind="reverse_rest", norm="tokens")
    u = rule.step(c["x"], c["ids"].view(-1), start, adv, old, teacher=(lists.top_ids, lists.top_logp), temperature=c["tau"])
    rule.check()
    assert (u.dlogits[used:] == 0).all() and (u.weight[used:] == 0).all()
    f = lambda v: ctypes.c_float(v).value
    few = {k: v[:used] for k, v in c.items()}
    cut = u._replace(dlogits=u.dlogits[:used], logp=u.logp[:used], entropy=u.entropy[:used], distill=u.distill[:used], weight=u.weight[:used])
    check_update(cut, few, adv, old[:used], start, "reverse_rest", dict(clip_low=f(0.2), clip_high=f(0.2), entropy_coef=0.125, distill_coef=0.5,
                                                                       norm="tokens"))
    u = rule.step(c["x"][:0], c["ids"].view(-1)[:0], torch.zeros(5, device="cuda", dtype=torch.int32), adv, old[:0],
                  teacher=(lists.top_ids[:0], lists.top_logp[:0]), temperature=c["tau"][:0])
    rule.check()
    assert float(u.objective) == 0 and u.dlogits.shape == (0, V) and (u.stats == 0).all()


def test_two_graphs_of_one_driver_run_at_once():
    from paper_2512_15347_b200.token_update import TokenUpdate
    V, n_rows = 4001, 600
    rule, g = TokenUpdate(entropy_coef=0.1), torch.Generator(device="cuda").manual_seed(5)
    start = torch.arange(n_rows + 1, device="cuda", dtype=torch.int32) * 8      # more tokens than one CTA of the objective takes
    sides, graphs, eager = [torch.cuda.Stream() for _ in range(2)], [], []
    for i in range(2):
        x = torch.randn(n_rows * 8, V, device="cuda", generator=g).to(torch.bfloat16)
        ids = torch.randint(0, V, (n_rows * 8,), device="cuda", generator=g, dtype=torch.int32)
        adv, old = torch.randn(n_rows, device="cuda", generator=g), torch.full((n_rows * 8,), -8.0, device="cuda")
        eager.append(rule.step(x, ids, start, adv, old))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            u = rule.step(x, ids, start, adv, old)
        graphs.append((graph, u, (x, ids, adv, old)))           # a graph reads its inputs where they were
    torch.cuda.synchronize()
    for _ in range(20):
        for side, (graph, _, _) in zip(sides, graphs):
            with torch.cuda.stream(side):
                graph.replay()
    torch.cuda.synchronize()
    for (_, u, _), e in zip(graphs, eager):
        assert torch.equal(u.objective, e.objective) and torch.equal(u.stats, e.stats) and torch.equal(u.dlogits, e.dlogits)
    rule.check()


def test_example_update_gives_the_objectives_gradient():
    from paper_2512_15347_b200.examples import token_rollout as T
    g = torch.Generator(device="cuda").manual_seed(3)
    policy, reference_policy = T.Policy(layers=2, q_heads=8, kv_heads=2, dim=64, vocab=500), T.Policy(layers=2, q_heads=8, kv_heads=2, dim=64, vocab=500, seed=9)
    prompts = [torch.randint(0, policy.vocab, (n,), generator=g, device="cuda", dtype=torch.int32) for n in (33, 90)]
    made, logp, adv, _, _ = T.rollout(policy, prompts, n_expand=8, n_keep=4, steps=10, prune_at=5, seed=4, repetition=1.0, frequency=0.0)
    u, grad, x = T.update(policy, prompts, made, logp, adv, reference=reference_policy)
    n = made.numel()
    # bf16 logits of the paged pass and of this one carry roundings of ~ 0.02 each: two computations of one number
    assert (u.logp.view(made.shape) - logp).abs().max() < 0.5 and (u.logp.view(made.shape) - logp).abs().mean() < 0.08
    # the gradient to the logits by autograd in 64 bits, from the definitions
    tau = 0.9
    z = policy.logits(x).double().requires_grad_(True)
    lp = torch.log_softmax(z / tau, -1)
    q = torch.log_softmax(reference_policy.logits(x).double() / tau, -1)
    ids = torch.stack([ref.alternatives(r, 20) for r in reference_policy.logits(x)])
    tl = q.gather(1, ids).float().double()
    rest = torch.ones_like(lp, dtype=torch.bool).scatter(1, ids, False)
    lr = torch.logsumexp(lp.masked_fill(~rest, -math.inf), -1)
    tr = (1 - tl.exp().sum(-1)).clamp(min=ref.LEAST_REST)
    pi = lp.gather(1, ids)
    div = (pi.exp() * (pi - tl)).sum(-1) + lr.exp() * (lr - tr.log())
    r = (lp.gather(1, made.view(-1, 1).long())[:, 0] - logp.view(-1).double()).exp()
    a = adv.double().repeat_interleave(made.shape[1])
    surr = torch.minimum(r * a, r.clamp(1 - ctypes.c_float(0.2).value, 1 + ctypes.c_float(0.28).value) * a)
    J = (surr + ctypes.c_float(0.01).value * -(lp.exp() * lp).sum(-1) - ctypes.c_float(0.1).value * div).mean()
    J.backward()
    assert abs(float(u.objective) - float(J)) <= 1e-5 * (1 + abs(float(J)))
    # fp32 statistics (about 200 roundings of what the gradient is made of) and one rounding to bf16
    size = (a.abs()[:, None] * r.detach()[:, None] * lp.detach().exp() + 20 * lp.detach().exp()) / n / tau
    size.scatter_add_(1, made.view(-1, 1).long(), (a.abs() * r.detach() / n / tau)[:, None])
    tol = U * (2 * (SUM + 16 * tiles_of(500, torch.bfloat16)) + 456) * size + HALF_STEP[torch.bfloat16] * z.grad.abs() * 1.01 + 1e-30
    assert ((u.dlogits.double() - z.grad).abs() <= tol).all()
    # the product with the states is torch's own
    assert torch.equal(grad, x.T @ u.dlogits)


def test_example_runs(capsys):
    from paper_2512_15347_b200.examples import token_rollout as T
    T.main()
    out = capsys.readouterr().out
    assert "pages in use" in out and "update: objective" in out
