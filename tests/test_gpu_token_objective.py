"""The objective of token rows where log-probs lie far apart: a reference policy or a rollout that masks a token, by -inf or by the
type's lowest value; terms that are only watched; long rows."""
import math

import pytest
import torch

from paper_2512_15347_b200 import binding as B
from tests.test_gpu_token_update import HALF_STEP, U, check_gradient, make, reference

pytestmark = pytest.mark.gpu

F32 = lambda v: torch.tensor(v, dtype=torch.float32).item()
DIFFERENCES = [0.0, 1e-6, 0.34, 0.36, 0.7, 5.0, 50.0, 87.0, 89.0, 100.0, 699.0, 701.0, 1e9, 3e38, math.inf]


def e(x):
    return math.inf if x > 709 else math.exp(x)


def em1(x):
    return math.inf if x > 709 else math.expm1(x)


def objective(new, adv, old=None, ref=None, beta=0.0, clip_low=0.2, clip_high=0.2, entropy=None, distill=None, entropy_coef=0.0, distill_coef=0.0, **_):
    """One row, weights 1, by the formulas in 64 bits with their limits at +-inf: (terms of each token, dlogp, ratio).  A term whose
    coefficient is 0 is none."""
    terms, dlogp, ratio = [], [], []
    lo, hi = 1 - F32(clip_low), 1 + F32(clip_high)
    for j, n in enumerate(new):
        d = 0.0 if old is None else n - old[j]
        r = e(d)
        free, held = (r * adv if adv else 0.0), min(max(r, lo), hi) * adv
        t, g = min(free, held), free if free <= held else 0.0
        if ref is not None and beta:
            x = ref[j] - n
            t -= F32(beta) * (math.inf if math.isinf(x) else em1(x) - x)
            g += F32(beta) * em1(x)
        t += F32(entropy_coef) * entropy[j] if entropy_coef else 0.0
        t -= F32(distill_coef) * distill[j] if distill_coef else 0.0
        terms.append(t)
        dlogp.append(g)
        ratio.append(r)
    return terms, dlogp, ratio


def run(new, adv, **kw):
    """The call on one row of weights 1."""
    dev = lambda v: torch.tensor(v, device="cuda", dtype=torch.float32)
    n = len(new)
    o = dict(objective=dev([7.0]), dlogp=dev([7.0] * n), ratio=dev([7.0] * n), weight=dev([7.0] * n), stats=dev([7.0] * 5))
    ws = torch.zeros(B.token_objective_workspace_bytes(n), device="cuda", dtype=torch.uint8)
    arrays = {k: dev(kw.pop(k)) for k in ("logp_old", "logp_ref", "entropy", "distill") if k in kw}
    B.token_objective(torch.tensor([0, n], device="cuda", dtype=torch.int32), dev(new), dev([adv]), workspace=ws, norm="sum", **o, **arrays, **kw)
    return {k: v.tolist() for k, v in o.items()}


def near(got, want, what, tol=0.0):
    """Polynomials good to 1e-11 and one rounding to 32 bits; what passes the largest number of 32 bits is infinite."""
    if math.isnan(want):
        assert math.isnan(got), (what, got, want)
    elif abs(want) > 3.4028235e38:
        assert got == math.copysign(math.inf, want) or abs(want) < 3.4028236e38, (what, got, want)
    else:
        assert abs(got - want) <= (U + 1e-10) * abs(want) + tol + 2.0 ** -149, (what, got, want)


@pytest.mark.parametrize("beta", [0.04, 3.0])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("adv", [0.0, 1.5, -2.0])
def test_derivative_of_the_divergence_from_a_reference(sign, adv, beta):
    new = [-2.0] * len(DIFFERENCES) if sign < 0 else [-1.0] * len(DIFFERENCES)
    ref = [F32(n + sign * d) for n, d in zip(new, DIFFERENCES)]
    _, dlogp, _ = objective(new, adv, ref=ref, beta=beta)
    o = run(new, adv, logp_ref=ref, beta=beta)
    for d, got, want in zip(DIFFERENCES, o["dlogp"], dlogp):
        # two terms of 64 bits, each good to 1e-10 of itself
        near(got, want, (sign * d, adv), 1e-10 * (abs(adv) + beta))
    # a token alone: the divergence too
    for n, r, d in zip(new, ref, DIFFERENCES):
        terms, dlogp, _ = objective([n], adv, ref=[r], beta=beta)
        o = run([n], adv, logp_ref=[r], beta=beta)
        near(o["objective"][0], terms[0], ("J", sign * d), 1e-10 * abs(adv) + U * abs(adv))


def test_a_reference_that_is_only_watched_moves_nothing():
    new = [-1.0, -2.0, -0.5, -3.0]
    plain = run(new, 1.25)
    for ref in ([-1.5, -math.inf, -3e38, -0.25], [math.inf, -1e9, 80.0, 800.0]):
        o = run(new, 1.25, logp_ref=ref)
        assert o["dlogp"] == plain["dlogp"] == [1.25] * 4


def test_an_update_step_against_a_reference_that_masks_tokens():
    from paper_2512_15347_b200.token_update import TokenUpdate, score
    V, lens = 5003, [3, 4, 5]
    n = sum(lens)
    c = make(n, V, torch.bfloat16, 21, masks=False)
    other = make(n, V, torch.bfloat16, 22, masks=False)["x"]
    at = c["ids"][:, 0].long()
    other[1, at[1]] = -math.inf
    other[5, at[5]] = torch.finfo(torch.bfloat16).min
    other[6, at[6]] = -60.0
    tau = c["tau"]
    ref = score(other, c["ids"], temperature=tau).logp[:, 0].contiguous()
    assert ref[1] == -math.inf and ref[5] < -1e38
    start = torch.tensor([0, 3, 7, 12], device="cuda", dtype=torch.int32)
    adv = torch.tensor([1.0, -0.5, 0.25], device="cuda")
    own = score(c["x"], c["ids"], temperature=tau).logp[:, 0].contiguous()
    old = own + 0.1
    for beta in (0.1, 0.0):
        rule = TokenUpdate(beta=beta, norm="sum", clip_high=0.3)
        u = rule.step(c["x"], c["ids"].view(-1), start, adv, old, logp_ref=ref, temperature=tau)
        dlogp = []
        for r in range(3):
            a, b = int(start[r]), int(start[r + 1])
            dlogp += objective(u.logp[a:b].tolist(), float(adv[r]), old=old[a:b].tolist(), ref=ref[a:b].tolist(), beta=beta, clip_high=0.3)[1]
        assert all(math.isfinite(d) for d in dlogp)
        w = dict(c, dlogp=torch.tensor(dlogp, device="cuda", dtype=torch.float64)[:, None], dentropy=torch.zeros(n, device="cuda"))
        check_gradient(w, u.dlogits, reference(w, entropy=False))
        assert bool(torch.isfinite(u.dlogits).all())


@pytest.mark.parametrize("term", ["distill", "entropy", "logp_ref"])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_term_without_weight_is_not_in_the_objective(term, bad):
    """Watched beside the objective: the divergence from a teacher of whose tokens the policy masks one is infinite."""
    new, old = [-1.0, -2.0, -0.5], [-1.1, -1.8, -0.5]
    kw = dict(entropy=[1.0, 2.0, 3.0], distill=[0.5, 0.25, 2.0], logp_ref=[-1.2, -2.0, -0.25])
    coef = dict(entropy="entropy_coef", distill="distill_coef", logp_ref="beta")
    use = dict(entropy_coef=0.01, distill_coef=0.5, beta=0.1)
    use[coef[term]] = 0.0
    kw[term] = [kw[term][0], bad, kw[term][2]]
    o = run(new, 1.5, logp_old=old, **kw, **use)
    terms, dlogp, _ = objective(new, 1.5, old=[F32(v) for v in old], ref=[F32(v) for v in kw["logp_ref"]], entropy=kw["entropy"], distill=kw["distill"], **use)
    near(o["objective"][0], sum(terms), term, 1e-10 + U * sum(map(abs, terms)))
    for j in range(3):
        near(o["dlogp"][j], dlogp[j], (term, j), 1e-10)
    at = dict(distill=3, entropy=2, logp_ref=1)[term]
    assert not math.isfinite(o["stats"][at])                 # what was watched is still told
    # with weight it is in there
    use[coef[term]] = 0.25
    assert not math.isfinite(run(new, 1.5, logp_old=old, **kw, **use)["objective"][0])


def test_an_update_step_watches_an_infinite_divergence():
    from paper_2512_15347_b200.token_update import TokenUpdate
    n, V = 5, 1000
    c = make(n, V, torch.float32, 4, n_list=8, masks=False)
    c["x"][2, int(c["list_ids"][2, 0])] = -math.inf
    c["ids"][2] = int(c["list_ids"][2, 1])
    start, adv = torch.tensor([0, n], device="cuda", dtype=torch.int32), torch.tensor([0.5], device="cuda")
    u = TokenUpdate(norm="tokens").step(c["x"], c["ids"].view(-1), start, adv, teacher=(c["list_ids"], c["list_logp"]), temperature=c["tau"])
    assert float(u.distill[2]) == math.inf and float(u.stats[3]) == math.inf
    assert abs(float(u.objective) - 0.5) <= U * 0.5 + 1e-9 and bool(torch.isfinite(u.dlogits).all())


@pytest.mark.parametrize("adv", [0.0, -0.0, 1.5, -2.0])
def test_ratios_beyond_all_numbers(adv):
    """A rollout's log-prob far below the policy's.  No advantage times a ratio of any size is 0, as it is for one of e^700."""
    new = [-1.0] * len(DIFFERENCES)
    for sign in (1, -1):
        for d in DIFFERENCES:
            old = F32(-1.0 - sign * d)
            o = run([-1.0], adv, logp_old=[old])
            terms, dlogp, ratio = objective([-1.0], adv, old=[old])
            for name, want in (("objective", terms), ("dlogp", dlogp), ("ratio", ratio)):
                near(o[name][0], want[0], (name, sign * d))
    # what is no number stays none
    for old, a in ((math.nan, adv), (-1.0, math.nan)):
        o = run([-1.0], a, logp_old=[old])
        assert math.isnan(o["objective"][0]) and math.isnan(o["dlogp"][0])


def test_what_lies_between_the_rows_enters_nothing():
    """Inputs of tokens of no row may hold anything."""
    start = torch.tensor([2, 4, 4, 7], device="cuda", dtype=torch.int32)
    adv = torch.tensor([1.0, -3.0, 0.5], device="cuda")
    values = [-torch.rand(9, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda") for i in range(5)]
    outs = []
    for bad in (0.0, math.nan, math.inf):
        new, old, ref, ent, div = (v.clone() for v in values)
        for v in (new, old, ref, ent, div):
            v[:2], v[7:] = bad, bad
        o = [torch.full((k,), 7.0, device="cuda") for k in (1, 9, 9, 9, B.TOKEN_STATS)]
        ws = torch.zeros(B.token_objective_workspace_bytes(9), device="cuda", dtype=torch.uint8)
        B.token_objective(start, new, adv, o[0], o[1], ws, logp_old=old, logp_ref=ref, entropy=ent, distill=div, beta=0.1, entropy_coef=0.1, distill_coef=0.1,
                          weight=o[2], ratio=o[3], stats=o[4])
        outs.append(o)
        assert o[1][:2].tolist() == o[1][7:].tolist() == o[2][:2].tolist() == o[2][7:].tolist() == [0.0, 0.0]
        assert o[3][:2].tolist() == o[3][7:].tolist() == [1.0, 1.0]
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))


@pytest.mark.parametrize("n", [3, 1021, 2 ** 24 - 1, 2 ** 24 + 1, 2 ** 25 - 1, 100000007, 2 ** 31 - 2 ** 20])
def test_weights_of_long_rows(n):
    """A row's tokens weigh 1 / n of it, up to the longest batch."""
    lp = torch.zeros(n, device="cuda")
    weight = torch.full((n,), 7.0, device="cuda")
    J = torch.zeros(1, device="cuda")
    ws = torch.zeros(B.token_objective_workspace_bytes(n), device="cuda", dtype=torch.uint8)
    B.token_objective(torch.tensor([0, n], device="cuda", dtype=torch.int32), lp, torch.ones(1, device="cuda"), J, lp, ws, weight=weight)
    near(float(weight[0]), 1 / n, n)
    for part in (weight, lp):                               # the derivative over the log-probs themselves: A w = w
        for a in range(0, n, 2 ** 28):
            assert bool((part[a: a + 2 ** 28] == weight[0]).all())
    near(float(J), 1.0, n, 1e-9)                            # n terms, added in 64 bits
    del lp, weight
    torch.cuda.empty_cache()
