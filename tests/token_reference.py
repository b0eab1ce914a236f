"""Plain 64-bit forms of the policy-update calls on token trajectories, row by row, with the sizes that rounding errors are
measured by."""
import math

import torch

LEAST_REST = 2.0 ** -20


def row_terms(l, tau=1.0, ids=(), list_ids=(), list_logp=(), kind="forward", dlogp=None, dentropy=0.0, ddistill=0.0):
    """One row in 64 bits, without infinities of its own but -inf: dict of logp, lse, entropy, distill, gradient; `size_*`: sums of the
    absolute values that go into them.  The gradient is that of torch's autograd on the allowed tokens."""
    V = l.numel()
    l = l.double()
    ids = [int(i) for i in ids]
    g = torch.zeros(V, dtype=torch.float64, device=l.device)
    allowed = torch.nonzero(l > -math.inf)[:, 0]
    if allowed.numel() == 0:
        return dict(logp=torch.tensor([-math.inf if 0 <= i < V else 0.0 for i in ids], dtype=torch.float64), lse=-math.inf, entropy=0.0,
                    distill=0.0, gradient=g, size_gradient=g.clone(), size_distill=0.0, spread=torch.zeros(len(ids), dtype=torch.float64))
    place = torch.full((V,), -1, dtype=torch.long, device=l.device)
    place[allowed] = torch.arange(allowed.numel(), device=l.device)
    x = l[allowed].clone().requires_grad_(True)
    lp = torch.log_softmax(x / tau, -1)
    p = lp.exp()
    entropy = -(p * torch.where(p > 0, lp, torch.zeros_like(lp))).sum()
    out = dict(lse=float(torch.logsumexp(x.detach() / tau, -1)), entropy=float(entropy.detach()))
    top = float(l.max()) / tau
    total = x.sum() * 0
    logp, spread, size = [], [], torch.zeros(V, dtype=torch.float64, device=l.device)
    weights = [0.0] * len(ids) if dlogp is None else [float(w) for w in dlogp]
    for i, w in zip(ids, weights):
        if not 0 <= i < V:
            logp.append(0.0)
            spread.append(0.0)
            continue
        at = int(place[i])
        logp.append(float(lp[at].detach()) if at >= 0 else -math.inf)
        spread.append(abs(float(l[i]) / tau - top) if at >= 0 else 0.0)
        if at >= 0:
            total = total + w * lp[at]
        elif w:                                     # d ln p_i / d x_v = [i = v] - p_v also where p_i is 0
            g[i] += w / tau
            g[allowed] -= w / tau * p.detach()
        size[allowed] += abs(w) / tau * p.detach()
        size[i] += abs(w) / tau
    out["logp"], out["spread"] = torch.tensor(logp, dtype=torch.float64), torch.tensor(spread, dtype=torch.float64)
    total = total + dentropy * entropy
    pd, ld = p.detach(), lp.detach().clamp(min=-1e4)
    size[allowed] += abs(dentropy) / tau * pd * (ld.abs() + out["entropy"])
    used = {}
    for i, tl in zip(list_ids, list_logp):
        if 0 <= int(i) < V and float(tl) != -math.inf:
            used[int(i)] = float(tl)                # the last one counts
    out["distill"], out["size_distill"] = 0.0, 0.0
    if used or (len(list_ids) and kind != "forward"):
        at = torch.tensor(list(used), dtype=torch.long, device=l.device)
        tl = torch.tensor(list(used.values()), dtype=torch.float64, device=l.device)
        if kind == "forward":
            tl = torch.log_softmax(tl, -1)
        t = tl.exp()
        inside = place[at]
        have = inside >= 0
        rest = torch.ones_like(lp, dtype=torch.bool)
        rest[inside[have]] = False
        some = bool(rest.any())
        size_d = float((t * tl.abs()).sum())
        if kind != "reverse_rest":
            loss = (t * torch.where(t > 0, tl, torch.zeros_like(tl))).sum() - (t[have] * lp[inside[have]]).sum()
            if bool((t[~have] > 0).any()):
                loss = loss + math.inf
                g[at[~have]] -= ddistill / tau * t[~have]       # as the formula has it
                g[allowed] += ddistill / tau * t[~have].sum() * pd
            size_d += float((t[have] * ld[inside[have]].abs()).sum())
        else:
            q, w = p[inside[have]], lp[inside[have]] - tl[have]
            q = torch.where(q > 0, q, torch.zeros_like(q))
            loss = torch.where(q > 0, q * w, torch.zeros_like(q)).sum()
            size_d = float((q.detach() * (ld[inside[have]].abs() + tl[have].abs())).sum())
        size[allowed] += abs(ddistill) / tau * pd
        size[at] += abs(ddistill) / tau * (t if kind != "reverse_rest" else torch.where(have, p.detach()[inside] * (tl.abs() + ld[inside].abs() + 1), torch.zeros_like(t)))
        if kind != "forward" and some:
            tr = max(1 - float(t.sum()), LEAST_REST)
            lr, share_of = rest_of(x, rest, tau)
            if kind == "forward_rest":
                loss = loss + tr * (math.log(tr) - lr)
                size_d += tr * (abs(math.log(tr)) + abs(float(lr)))
                share = tr
            else:
                loss = loss + lr.exp() * (lr - math.log(tr))
                size_d += float(lr.exp()) * (abs(math.log(tr)) + abs(float(lr)))
                share = float(lr.exp()) * (abs(math.log(tr)) + abs(float(lr)) + 1)
            size[allowed[rest]] += abs(ddistill) / tau * share * share_of
        out["distill"], out["size_distill"] = float(loss), size_d
        if kind == "reverse_rest":
            size[allowed] += abs(ddistill) / tau * pd * abs(float(loss))
        if ddistill:
            total = total + ddistill * (loss if bool(torch.isfinite(loss)) else loss_without_infinity(t, have, lp, inside, kind, lr if kind != "forward" and some else None))
    total.backward()
    g[allowed] += x.grad
    out["gradient"], out["size_gradient"] = g, size
    return out


def rest_of(x, rest, tau):
    """Logarithm of the mass of the tokens `rest` and their shares of it.  Next to the types' ends 64 bits lose small differences as
    well, so sums are taken from the largest logit of their own, and the derivative is put in as what it is: shares - p."""
    y, z = x[rest].detach(), x.detach()
    share, p = torch.softmax((y - y.max()) / tau, -1), torch.softmax((z - z.max()) / tau, -1)
    value = torch.logsumexp((y - y.max()) / tau, -1) - torch.logsumexp((z - z.max()) / tau, -1) + (y.max() - z.max()) / tau
    slope = ((share * x[rest]).sum() - (p * x).sum()) / tau
    return value + (slope - slope.detach()), share


def loss_without_infinity(t, have, lp, inside, kind, lr):
    """The terms that are finite: their gradient is what is left to compute."""
    loss = -(t[have] * lp[inside[have]]).sum()
    if kind == "forward_rest" and lr is not None:
        loss = loss - max(1 - float(t.sum()), LEAST_REST) * lr
    return loss


def alternatives(l, n):
    """Ids of the n largest logits, ties to the lowest index, -1 where there are too few."""
    x = l.double()
    x = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
    at = torch.sort(x, descending=True, stable=True).indices[:n]
    return torch.where(x[at] > -math.inf, at, torch.full_like(at, -1))


def objective(start, new, adv, old=None, ref=None, entropy=None, distill=None, clip_low=0.2, clip_high=0.2, beta=0.0, entropy_coef=0.0,
              distill_coef=0.0, scale=1.0, norm="rows"):
    """(objective, dlogp, weight, ratio, stats) in 64 bits on the host, token by token."""
    start, n, R = start.tolist(), new.numel(), adv.numel()
    f = lambda t: None if t is None else t.double().cpu().tolist()
    new, old, ref, entropy, distill, adv = f(new), f(old), f(ref), f(entropy), f(distill), f(adv)
    total = start[-1] - start[0]
    dlogp, weight, ratio, stats, J = [0.0] * n, [0.0] * n, [1.0] * n, [0.0] * 5, 0.0
    for i in range(R):
        a, b = start[i], start[i + 1]
        for j in range(a, b):
            w = scale * {"rows": 1 / ((b - a) * R), "tokens": 1 / total, "sum": 1.0}[norm]
            r = math.exp(new[j] - (new[j] if old is None else old[j]))
            free, held = r * adv[i], min(max(r, 1 - clip_low), 1 + clip_high) * adv[i]
            d = 0.0 if ref is None else ref[j] - new[j]
            k = math.expm1(d) - d
            h, q = 0.0 if entropy is None else entropy[j], 0.0 if distill is None else distill[j]
            J += w * (min(free, held) - beta * k + entropy_coef * h - distill_coef * q)
            dlogp[j] = w * ((free if free <= held else 0.0) - beta * -math.expm1(d))
            weight[j], ratio[j] = w, r
            for s, v in enumerate((min(free, held), k, h, q)):
                stats[s] += w * v
            stats[4] += (free > held) / total
    return J, dlogp, weight, ratio, stats
