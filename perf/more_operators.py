"""Cases for the policy update on token trajectories: log-probabilities of given tokens with entropy and top alternatives,
distillation from a teacher's top logits (both forward and backward), and the objective over ragged rows of tokens.

`run` computes a case in plain torch operations (32-bit arithmetic, 64 where that loses what matters, one rounding at the end) or,
where `own` is set, through the library's entry points.  `exact` is the definition in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
DEV = "cuda"
LEAST_REST = 2.0 ** -20                      # of a teacher's mass outside its list


# ------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # one row of one request, a small vocabulary: the token's log-prob and its alternatives, latency only
        dict(name="score-one-row", op="score", dtype="f32", rows=1, vocab=32000, ids=1, top=8, entropy=True, temperature=True),
        # a few rows of a decoding step over an odd vocabulary, long lists of alternatives
        dict(name="score-few-rows-top100", op="score", dtype="f16", rows=12, vocab=50001, ids=1, top=100, entropy=True, temperature=False),
        # a teacher's pass over 1024 tokens: the lists that a student learns from
        dict(name="score-teacher-lists", op="score", dtype="bf16", rows=1024, vocab=131072, ids=1, top=64, entropy=False, temperature=False),
        # the first update after a rollout: weights known before, log-probs and gradients in one go, an entropy bonus
        dict(name="train-odd-vocabulary", op="train", dtype="f16", rows=1000, vocab=50001, ids=1, top=0, entropy=True, temperature=True),
        # several candidates a position in fp32
        dict(name="train-candidates-fp32", op="train", dtype="f32", rows=700, vocab=32000, ids=5, top=0, entropy=False, temperature=False),
        # a small student with a short list
        dict(name="distill-small", op="distill", dtype="f32", rows=16, vocab=1000, list=10, kind="forward", temperature=False),
        # a long batch from lists of 64, the list renormalised
        dict(name="distill-lists", op="distill", dtype="bf16", rows=2048, vocab=131072, list=64, kind="forward", temperature=False),
        # odd vocabulary, the mass outside the list as one bucket
        dict(name="distill-rest", op="distill", dtype="bf16", rows=1500, vocab=50001, list=100, kind="forward_rest", temperature=True),
        # reverse divergence on the student's own tokens
        dict(name="distill-reverse", op="distill", dtype="f16", rows=900, vocab=65536, list=32, kind="reverse_rest", temperature=True),
        # the objective of a handful of short answers: latency only
        dict(name="objective-short-rows", op="objective", rows=16, hi=200, norm="rows", ref=True),
        # the survivors of 64 prompts x 12 with answers of up to 4096 tokens
        dict(name="objective-ragged-rows", op="objective", rows=768, hi=4096, norm="tokens", ref=True),
        # a whole update step: log-probs, objective, gradient with entropy bonus and a divergence from the reference's lists
        dict(name="update-step", op="update", dtype="bf16", rows=48, hi=120, vocab=65536, list=20, kind="reverse_rest", temperature=True, norm="rows"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["score", "score", "train", "train", "distill", "distill", "distill", "objective", "objective", "update"])
    if op == "objective":
        rows = _log(rng, 1, 1000)
        return dict(op=op, rows=rows, hi=_log(rng, 1, max(2, min(8192, 3_000_000 // rows))), norm=rng.choice(["rows", "tokens", "sum"]),
                    ref=rng.choice([True, False]))
    dt = rng.choice(["f32", "bf16", "bf16", "f16"])
    vocab = _log(rng, 1000, 160000)
    rows = _log(rng, 1, max(2, min(4096, 130_000_000 // vocab)))
    case = dict(op=op, dtype=dt, rows=rows, vocab=vocab, temperature=rng.choice([True, False]))
    if op in ("score", "train"):
        case.update(ids=rng.choice([1, 1, 1, 3, 8]), top=rng.choice([0, 1, 5, 20, 128]) if op == "score" else 0, entropy=rng.choice([True, False]))
    if op in ("distill", "update"):
        case.update(list=_log(rng, 1, 256), kind=rng.choice(["forward", "forward_rest", "reverse_rest"]))
    if op == "update":
        case.update(rows=_log(rng, 1, 64), norm=rng.choice(["rows", "tokens", "sum"]))
        case["hi"] = _log(rng, 2, max(3, min(4000, 130_000_000 // vocab // case["rows"])))
    return case


# --------------------------------------------------------------------------------- the inputs

def _lengths(case):
    """Row lengths spread evenly over the logarithm of [1, hi]; of more than three rows one is empty."""
    n = case["rows"]
    x = [max(1, min(case["hi"], round(math.exp((i + 1) / n * math.log(case["hi"]))))) for i in range(n)]
    return [0] + x[1:] if n > 3 else x


def _logits(g, R, V, dt, ids, dead):
    """Rows of different sharpness, the given tokens likelier than others; of many rows one with a grammar's mask, one masked by the
    type's lowest value, one that allows nothing."""
    x = torch.empty((R, V), device=DEV, dtype=dt).normal_(generator=g)
    x.mul_((1 + 2 * torch.rand((R, 1), generator=g, device=DEV)).to(dt))
    for j in range(ids.shape[1]):                        # one by one: a token may be given twice
        x.scatter_add_(1, ids[:, j: j + 1].clamp(min=0).long(), (9 * torch.rand((R, 1), generator=g, device=DEV)).to(dt))
    if R > 6:
        some = torch.rand(V, generator=g, device=DEV) < 0.6        # more stay allowed than the longest list has
        some[ids[1:3].clamp(min=0).long().view(-1)] = False
        x[1].masked_fill_(some, -math.inf)
        x[2].masked_fill_(some, torch.finfo(dt).min)
        if dead:
            x[3] = -math.inf
    return x


def _ids(g, R, V, n, padded):
    ids = torch.randint(0, V, (R, n), generator=g, device=DEV, dtype=torch.int32)
    if R > 6 and padded:
        ids[5, -1] = -1                                  # a padded position
    return ids


def _teacher(g, logits, n):
    """The n likeliest tokens of a teacher that half agrees, with their log-probs; lists of different lengths, padded by -1."""
    R, V = logits.shape
    n = min(n, V)
    ids, logp = torch.empty((R, n), device=DEV, dtype=torch.int32), torch.empty((R, n), device=DEV)
    step = max(1, 40_000_000 // V)
    for a in range(0, R, step):
        y = logits[a: a + step].float()
        y = y + torch.randn(y.shape, generator=g, device=DEV)
        lse = torch.logsumexp(y.double(), -1, keepdim=True)
        top, at = y.topk(n, -1)
        ids[a: a + step], logp[a: a + step] = at, (top.double() - lse).float()
    if R > 6:
        keep = torch.randint(1, n + 1, (R, 1), generator=g, device=DEV)
        keep[4] = 0
        keep[R // 2:] = n
        ids.masked_fill_(torch.arange(n, device=DEV)[None] >= keep, -1)
    none = ~(logp > -1e30)                               # a list ends where its teacher's mask begins
    return ids.masked_fill_(none, -1), logp.masked_fill_(none, 0.)


def _floats(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    s = dict(case=case)
    op = case["op"]
    if op in ("objective", "update"):
        R = case["rows"]
        lens = _lengths(case)
        n = s["tokens"] = sum(lens)
        lens = torch.tensor(lens, device=DEV, dtype=torch.int32)[torch.randperm(R, generator=g, device=DEV)]
        s["start"] = torch.cat([lens.new_zeros(1), torch.cumsum(lens, 0).to(torch.int32)])
        s["adv"] = 0.5 + _floats(g, R)                   # one rank's share of the groups: not centred by itself
        s["logp_new"] = -torch.rand(n, generator=g, device=DEV) * 4
        s["clip"], s["beta"], s["scale"] = (0.2, 0.28), 0.04, 0.5
    else:
        n = case["rows"]
    if op == "objective":
        s["logp_old"] = s["logp_new"] + 0.15 * _floats(g, n)
        s["logp_ref"] = s["logp_new"] + 0.05 * _floats(g, n) if case["ref"] else None
    else:
        V, dt = case["vocab"], DTYPES[case["dtype"]]
        s["ids"] = _ids(g, n, V, case.get("ids", 1), op != "update")
        s["logits"] = _logits(g, n, V, dt, s["ids"], op != "update")
        s["temperature"] = 0.6 + 0.8 * torch.rand(n, generator=g, device=DEV) if case["temperature"] else None
        if op in ("distill", "update"):
            s["list_ids"], s["list_logp"] = _teacher(g, s["logits"], case["list"])
            s["ddistill"] = 0.5 + torch.rand(n, generator=g, device=DEV)
        if op == "train":
            s["dlogp"] = _floats(g, n, case["ids"])
            s["dentropy"] = 0.3 + 0.2 * torch.rand(n, generator=g, device=DEV) if case["entropy"] else None
        if op == "update":                               # log-probs of the rollout: near the new ones
            x = s["logits"].float() / (1 if s["temperature"] is None else s["temperature"][:, None])
            lp = torch.log_softmax(x, -1).gather(1, s["ids"].clamp(min=0).long())[:, 0]
            s["logp_old"] = lp + 0.15 * _floats(g, n)
            s["logp_ref"] = None
            s["entropy_coef"], s["distill_coef"] = 0.01, 0.05
    if own:
        _handles(s)
    return s


def _handles(s):
    """Descriptors and buffers that a program keeps next to its own."""
    from paper_2512_15347_b200 import binding as B
    c = s["case"]
    op = c["op"]
    new = lambda *shape: torch.empty(shape, device=DEV)
    if op in ("objective", "update"):
        n = s["tokens"]
        s["status"] = torch.zeros(1, device=DEV, dtype=torch.int32)
        s["objective"], s["dlogp"], s["weight"], s["stats"] = new(1), new(n), new(n), new(B.TOKEN_STATS)
        s["workspace"] = torch.zeros(B.token_objective_workspace_bytes(n), device=DEV, dtype=torch.uint8)
    if op == "objective":
        return
    n = s["logits"].shape[0]
    s["terms"] = B.make_token_terms(temperature=s["temperature"], ids=s["ids"] if op != "distill" else None, n_top=c.get("top", 0),
                                    teacher_ids=s.get("list_ids"), teacher_logp=s.get("list_logp"), kind=c.get("kind", "forward"))
    if op != "distill":
        s["logp"] = new(n, s["ids"].shape[1])
    s["entropy"] = new(n) if op == "update" or c.get("entropy") else None
    s["lse"] = new(n) if op != "update" else None
    if c.get("top"):
        s["top_ids"], s["top_logp"] = torch.empty((n, c["top"]), device=DEV, dtype=torch.int32), new(n, c["top"])
    if op in ("distill", "update"):
        s["loss"] = new(n)
    if op != "score":
        s["dlogits"] = torch.empty_like(s["logits"])
    if op == "update":
        s["saved"] = new(n, B.TOKEN_SAVED)


# -------------------------------------------------------------------------------- one pass

def run(s):
    op = s["case"]["op"]
    if own:
        return _own(s, op)
    return {"score": _score, "train": _train, "distill": _distill, "objective": _objective, "update": _update}[op](s)


def _own(s, op):
    from paper_2512_15347_b200 import binding as B
    if op == "score":
        B.token_forward(s["logits"], s["terms"], logp=s["logp"], lse=s["lse"], entropy=s["entropy"], top_ids=s.get("top_ids"),
                        top_logp=s.get("top_logp"))
        return dict(logp=s["logp"], lse=s["lse"], entropy=s["entropy"], top_ids=s.get("top_ids"), top_logp=s.get("top_logp"))
    if op == "train":
        B.token_forward_backward(s["logits"], s["terms"], s["dlogits"], logp=s["logp"], lse=s["lse"], entropy=s["entropy"],
                                 dlogp=s["dlogp"], dentropy=s["dentropy"])
        return dict(logp=s["logp"], lse=s["lse"], entropy=s["entropy"], dlogits=s["dlogits"])
    if op == "distill":
        B.token_forward_backward(s["logits"], s["terms"], s["dlogits"], lse=s["lse"], distill=s["loss"], ddistill=s["ddistill"])
        return dict(loss=s["loss"], lse=s["lse"], dlogits=s["dlogits"])
    new = s["logp_new"]
    if op == "update":
        B.token_forward(s["logits"], s["terms"], logp=s["logp"], entropy=s["entropy"], distill=s["loss"], saved=s["saved"])
        new = s["logp"].view(-1)
    more = dict(entropy=s["entropy"], entropy_coef=s["entropy_coef"], distill=s["loss"], distill_coef=s["distill_coef"]) if op == "update" else {}
    B.token_objective(s["start"], new, s["adv"], s["objective"], s["dlogp"], s["workspace"], logp_old=s["logp_old"], logp_ref=s["logp_ref"],
                      clip_low=s["clip"][0], clip_high=s["clip"][1], beta=s["beta"], norm=s["case"]["norm"], scale=s["scale"],
                      weight=s["weight"], stats=s["stats"], status=s["status"], **more)
    out = dict(objective=s["objective"], dlogp=s["dlogp"], weight=s["weight"], stats=s["stats"])
    if op == "objective":
        return out
    B.token_backward(s["logits"], s["terms"], s["saved"], s["dlogits"], dlogp=s["dlogp"].view(-1, 1), dentropy=s["weight"],
                     entropy_scale=s["entropy_coef"], ddistill=s["weight"], distill_scale=-s["distill_coef"])
    return dict(out, logp=s["logp"], entropy=s["entropy"], loss=s["loss"], dlogits=s["dlogits"])


def _scaled(s):
    x = s["logits"].float()
    inv = None if s["temperature"] is None else 1 / s["temperature"][:, None]
    return (x if inv is None else x * inv), inv


def _softmax(x):
    """(x - lse, p, lse): of a row that allows nothing -inf, 0, -inf."""
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    some = total > 0
    lp = torch.where(some, (x - top) - torch.log(total), torch.full_like(x, -math.inf))
    return lp, e / torch.where(some, total, torch.ones_like(total)), (top + torch.log(total))[:, 0]


def _given(lp, ids):
    here = lp.gather(1, ids.clamp(min=0).long())
    return torch.where(ids >= 0, here, torch.zeros_like(here))


def _entropy(lp, p):
    return -(p * lp.clamp(min=-1e4)).sum(-1)


def _score(s):
    x, _ = _scaled(s)
    lp, p, lse = _softmax(x)
    out = dict(logp=_given(lp, s["ids"]), lse=lse, entropy=_entropy(lp, p) if s["case"]["entropy"] else None, top_ids=None, top_logp=None)
    if s["case"]["top"]:                                 # by value, then by the lowest index: one whole number for both
        bits = (s["logits"].float() + 0.0).view(torch.int32)
        key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * 2 ** 20 + (2 ** 20 - 1 - torch.arange(x.shape[1], device=DEV))
        at = key.topk(s["case"]["top"], -1).indices
        top = lp.gather(1, at)
        out["top_ids"], out["top_logp"] = torch.where(top == -math.inf, torch.full_like(at, -1), at).int(), top
    return out


def _logp_gradient(lp, p, entropy, ids, dlogp, dentropy):
    dlogp = torch.where(ids >= 0, dlogp, torch.zeros_like(dlogp))
    g = -p * dlogp.sum(-1, keepdim=True)
    if dentropy is not None:
        g = g - dentropy[:, None] * p * (lp.clamp(min=-1e4) + entropy[:, None])
    return g.scatter_add(1, ids.clamp(min=0).long(), dlogp)


def _train(s):
    x, inv = _scaled(s)
    lp, p, lse = _softmax(x)
    entropy = _entropy(lp, p) if s["case"]["entropy"] else None
    g = _logp_gradient(lp, p, entropy, s["ids"], s["dlogp"], s["dentropy"])
    g = torch.where((lse == -math.inf)[:, None], torch.zeros_like(g), g if inv is None else g * inv)
    return dict(logp=_given(lp, s["ids"]), lse=lse, entropy=entropy, dlogits=g.to(s["logits"].dtype))


def _divergence(x, lp, p, lse, ids, tl, kind):
    """Loss and its gradient to x."""
    used = ids >= 0
    at = ids.clamp(min=0).long()
    zero = torch.zeros_like(tl)
    tl = torch.where(used, tl, torch.full_like(tl, -math.inf))
    some = (used.any(-1) & (lse > -math.inf))[:, None]
    li, pi = lp.gather(1, at), p.gather(1, at)
    if kind == "forward":
        tl = torch.where(some, tl - torch.logsumexp(torch.where(some, tl, zero), -1, keepdim=True), tl)
        t = torch.exp(tl)
        loss = torch.where(used & some, t * (tl - li), zero).sum(-1)
        g = torch.where(some, p, torch.zeros_like(p)).scatter_add(1, at, torch.where(used & some, -t, zero))
        return loss, g
    t64 = torch.exp(tl.double())                         # what is left of 1 needs them
    tr64 = (1 - t64.sum(-1, keepdim=True)).clamp(min=LEAST_REST)
    t, tr = t64.float(), tr64.float()
    inside = torch.zeros(x.shape, device=DEV, dtype=torch.bool).scatter(1, torch.where(used, at, at[:, :1].expand_as(at)), used[:, :1].expand_as(at) | used)
    out_lp, out_p, out_lse = _softmax(x.masked_fill(inside, -math.inf))
    rest = (out_lse > -math.inf)[:, None]
    lr = torch.where(rest, (out_lse - lse)[:, None], torch.zeros_like(tr))
    pr = torch.where(rest, torch.exp(lr), torch.zeros_like(tr))
    none = (lse == -math.inf)[:, None]
    w = (t64.sum(-1, keepdim=True) + torch.where(rest, tr64, torch.zeros_like(tr64))).float()
    if kind == "forward_rest":
        loss = torch.where(used, t * (tl - li), zero).sum(-1, keepdim=True) + torch.where(rest, tr * (torch.log(tr) - lr), torch.zeros_like(tr))
        g = torch.where(inside, w * p, (pr * w - tr) * out_p).scatter_add(1, at, torch.where(used, -t, zero))
    else:
        loss = torch.where(used & (pi > 0), pi * (li - tl), zero).sum(-1, keepdim=True) + torch.where(rest, pr * (lr - torch.log(tr)), torch.zeros_like(tr))
        g = (pr * (lr - torch.log(tr) - loss)) * out_p
        g = g.scatter_add(1, at, torch.where(used & (pi > 0), pi * (li - tl - loss), zero))
    return torch.where(none, torch.zeros_like(loss), loss)[:, 0], torch.where(none, torch.zeros_like(g), g)


def _distill(s):
    x, inv = _scaled(s)
    lp, p, lse = _softmax(x)
    loss, g = _divergence(x, lp, p, lse, s["list_ids"], s["list_logp"], s["case"]["kind"])
    g = g * s["ddistill"][:, None]
    return dict(loss=loss, lse=lse, dlogits=(g if inv is None else g * inv).to(s["logits"].dtype))


def _objective_of(s, new, entropy=None, loss=None):
    """In 64 bits: differences of log-probs next to 0, and values next to the clip range."""
    start = s["start"].long()
    n, R = new.numel(), s["case"]["rows"]
    row = torch.searchsorted(start[1:], torch.arange(n, device=DEV), right=True)
    lens = (start[1:] - start[:-1]).double()
    weight = {"rows": 1 / (lens[row] * R), "tokens": torch.full_like(lens[row], 1 / max(n, 1)), "sum": torch.ones_like(lens[row])}[s["case"]["norm"]]
    weight = weight * s["scale"]
    a, new = s["adv"].double()[row], new.double()
    r = torch.exp(new - s["logp_old"].double())
    free, held = r * a, r.clamp(1 - s["clip"][0], 1 + s["clip"][1]) * a
    surr, moves = torch.minimum(free, held), free <= held
    kl, dkl = torch.zeros_like(r), torch.zeros_like(r)
    if s["logp_ref"] is not None:
        d = s["logp_ref"].double() - new
        kl, dkl = torch.expm1(d) - d, -torch.expm1(d)
    total = surr - s["beta"] * kl
    zero = torch.zeros_like(r)
    h, div = zero, zero
    if entropy is not None:
        h, div = entropy.double(), loss.double()
        total = total + s["entropy_coef"] * h - s["distill_coef"] * div
    dlogp = weight * (torch.where(moves, free, zero) - s["beta"] * dkl)
    mean = lambda v: (weight * v).sum()
    stats = torch.stack([mean(surr), mean(kl), mean(h), mean(div), (~moves).double().sum() / max(n, 1)])
    return dict(objective=mean(total).view(1).float(), dlogp=dlogp.float(), weight=weight.float(), stats=stats.float())


def _objective(s):
    return _objective_of(s, s["logp_new"])


def _update(s):
    x, inv = _scaled(s)
    lp, p, lse = _softmax(x)
    logp, entropy = _given(lp, s["ids"]), _entropy(lp, p)
    loss, g = _divergence(x, lp, p, lse, s["list_ids"], s["list_logp"], s["case"]["kind"])
    out = _objective_of(s, logp[:, 0], entropy, loss)
    g = g * (-s["distill_coef"] * out["weight"])[:, None]
    g = g + _logp_gradient(lp, p, entropy, s["ids"], out["dlogp"][:, None], s["entropy_coef"] * out["weight"])
    return dict(out, logp=logp, entropy=entropy, loss=loss, dlogits=(g if inv is None else g * inv).to(s["logits"].dtype))


# ------------------------------------------------------------------------------- the work

def work(case):
    op = case["op"]
    if op == "objective":
        n = sum(_lengths(case))
        return dict(bytes=4 * (n * (4 + case["ref"]) + 2 * case["rows"]), flops=20 * n)
    rows = sum(_lengths(case)) if op == "update" else case["rows"]
    cells = rows * case["vocab"]
    moved = cells * BYTES[case["dtype"]] * (1 if op == "score" else 2)
    small = 4 * rows * (2 * case.get("ids", 1) + 2 * case.get("top", 0) + 2 * case.get("list", 0) + 4)
    return dict(bytes=moved + small, flops=cells * (4 if op == "score" else 8))


# ----------------------------------------------------------------------- the definition, 64 bits

def exact(case, seed):
    """What run() returns, from the definitions: every part through the distribution over buckets that it is about."""
    s = prepare(case, seed)
    if case["op"] == "objective":
        return _exact_objective(s, s["logp_new"].double(), None, None)
    if case["op"] == "update":
        parts = _by_rows(s, lambda a, b: _exact_forward(s, a, b))
        out = _exact_objective(s, parts["logp"][:, 0], parts["entropy"], parts["loss"])
        s["dlogp"], s["dentropy"] = out["dlogp"][:, None], s["entropy_coef"] * out["weight"]
        s["ddistill"] = -s["distill_coef"] * out["weight"]
        return dict(out, **_by_rows(s, lambda a, b: _exact_forward(s, a, b, True)))
    every = _by_rows(s, lambda a, b: _exact_forward(s, a, b, case["op"] != "score"))
    names = {"score": ("logp", "lse", "entropy", "top_ids", "top_logp"), "train": ("logp", "lse", "entropy", "dlogits"),
             "distill": ("loss", "lse", "dlogits")}[case["op"]]
    return {k: every.get(k) for k in names}


def _by_rows(s, part):
    n, V = s["logits"].shape
    step = max(1, 30_000_000 // V)
    got = [part(a, min(n, a + step)) for a in range(0, n, step)]
    return {k: torch.cat([p[k] for p in got]) for k in got[0]}


def _exact_forward(s, a, b, gradient=False):
    c = s["case"]
    x = s["logits"][a:b].double()
    tau = 1.0 if s["temperature"] is None else s["temperature"][a:b, None].double()
    x = x / tau
    dead = (x == -math.inf).all(-1)
    y = torch.where(dead[:, None], torch.zeros_like(x), x)
    lp = torch.log_softmax(y, -1)
    p = torch.exp(lp)
    out = {}
    if c["op"] != "update":
        out["lse"] = torch.where(dead, torch.full_like(dead, -math.inf, dtype=torch.float64), torch.logsumexp(x, -1))
    g = torch.zeros_like(x)
    plogp = torch.special.entr(p)
    h = plogp.sum(-1, keepdim=True)
    if c["op"] != "distill":
        ids = s["ids"][a:b].long()
        pick = lp.gather(1, ids.clamp(min=0)).masked_fill(dead[:, None], -math.inf)
        out["logp"] = pick.masked_fill(ids < 0, 0.0)
        if c.get("entropy") or c["op"] == "update":
            out["entropy"] = h[:, 0].masked_fill(dead, 0.0)
        if c.get("top"):
            out["top_logp"] = lp.topk(c["top"], -1).values.masked_fill(dead[:, None], -math.inf)
        if gradient:
            w = s["dlogp"][a:b].double().masked_fill(ids < 0, 0.0)
            g.scatter_add_(1, ids.clamp(min=0), w)
            g -= p * w.sum(-1, keepdim=True)
            if s["dentropy"] is not None:
                g += s["dentropy"][a:b, None].double() * (plogp - p * h)
    if c["op"] in ("distill", "update"):
        loss, d = _exact_divergence(lp, p, s["list_ids"][a:b].long(), s["list_logp"][a:b].double(), c["kind"])
        out["loss"] = loss.masked_fill(dead, 0.0)
        if gradient:
            g += s["ddistill"][a:b, None].double() * d
    if gradient:
        out["dlogits"] = (g / tau).masked_fill(dead[:, None], 0.0)
    return out


def _exact_divergence(lp, p, ids, tl, kind):
    V = lp.shape[1]
    used = ids >= 0
    t = torch.where(used, torch.exp(tl), torch.zeros_like(tl))
    full = torch.zeros_like(lp).scatter_add_(1, ids.clamp(min=0), t)              # the teacher on its list
    listed_ = torch.zeros_like(lp).scatter_add_(1, ids.clamp(min=0), used.double()) > 0
    if kind == "forward":
        mass = t.sum(-1, keepdim=True)
        full = full / torch.where(mass > 0, mass, torch.ones_like(mass))
        loss = (torch.special.xlogy(full, full) - torch.where(listed_, full * lp, torch.zeros_like(lp))).sum(-1)
        return loss, torch.where(mass > 0, p, torch.zeros_like(p)) - full
    tr = (1 - t.sum(-1)).clamp(min=LEAST_REST)
    outside = lp.masked_fill(listed_, -math.inf)
    lr = torch.logsumexp(outside, -1)
    some = lr > -math.inf
    lr0 = torch.where(some, lr, torch.zeros_like(lr))
    pr = torch.where(some, torch.exp(lr0), torch.zeros_like(lr))
    share = torch.where(some[:, None], torch.exp(outside - lr0[:, None]), torch.zeros_like(p))
    lt = torch.zeros_like(lp).scatter_add_(1, ids.clamp(min=0), torch.where(used, tl, torch.zeros_like(tl)))
    if kind == "forward_rest":
        loss = torch.where(listed_, full * (lt - lp), torch.zeros_like(lp)).sum(-1) + torch.where(some, tr * (torch.log(tr) - lr0), torch.zeros_like(lr))
        mass = t.sum(-1) + torch.where(some, tr, torch.zeros_like(tr))
        g = mass[:, None] * p - full - torch.where(some, tr, torch.zeros_like(tr))[:, None] * share
        return loss, g
    gap = torch.where(listed_ & (p > 0), lp - lt, (lr0 - torch.log(tr))[:, None].expand_as(lp))
    loss = torch.where(listed_ & (p > 0), p * gap, torch.zeros_like(lp)).sum(-1) + torch.where(some, pr * (lr0 - torch.log(tr)), torch.zeros_like(lr))
    return loss, p * (gap - loss[:, None])


def _exact_objective(s, new, entropy, loss):
    """Row by row."""
    start, R, n = s["start"].tolist(), s["case"]["rows"], new.numel()
    lo, hi = s["clip"]
    total, stats = torch.zeros(1, device=DEV, dtype=torch.float64), torch.zeros(5, device=DEV, dtype=torch.float64)
    dlogp, weight = torch.zeros_like(new), torch.zeros_like(new)
    for i in range(R):
        a, b = start[i], start[i + 1]
        if a == b:
            continue
        w = s["scale"] * {"rows": 1 / ((b - a) * R), "tokens": 1 / n, "sum": 1.0}[s["case"]["norm"]]
        x, adv = new[a:b], s["adv"][i].double()
        r = (x - s["logp_old"][a:b].double()).exp()
        clipped = torch.where(adv > 0, r > 1 + hi, r < 1 - lo) & (adv != 0)
        surr = adv * torch.where(clipped, torch.full_like(r, 1 + hi) if adv > 0 else torch.full_like(r, 1 - lo), r)
        g = torch.where(clipped, torch.zeros_like(r), adv * r)
        kl = torch.zeros_like(r)
        if s["logp_ref"] is not None:
            d = s["logp_ref"][a:b].double() - x
            kl, g = torch.special.expm1(d) - d, g + s["beta"] * torch.special.expm1(d)
        row = torch.stack([surr.sum(), kl.sum(), entropy[a:b].sum() if entropy is not None else kl.new_zeros(()),
                           loss[a:b].sum() if loss is not None else kl.new_zeros(())])
        stats[:4] += w * row
        stats[4] += clipped.double().sum() / n
        mix = torch.tensor([1.0, -s["beta"], s.get("entropy_coef", 0.0), -s.get("distill_coef", 0.0)], device=DEV, dtype=torch.float64)
        total += w * (row * mix).sum()
        dlogp[a:b], weight[a:b] = w * g, w
    return dict(objective=total, dlogp=dlogp, weight=weight, stats=stats)
