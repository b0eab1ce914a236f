"""Plain 64-bit forms of the token-rollout calls, row by row from their definitions."""
import math

import torch


def ceil(a, b):
    return -(-a // b)


def attend(q, k, v, table, length, scale):
    """q [R, Hq, D], k, v [P, H, ps, D]; -> out, lse, and per output sum p|v| and the largest sum |q||k| * scale."""
    R, Hq, D = q.shape
    H, ps = k.shape[1], k.shape[2]
    out = torch.zeros(R, Hq, D, dtype=torch.float64, device=q.device)
    spread = torch.zeros_like(out)
    lse = torch.full((R, Hq), -math.inf, dtype=torch.float64, device=q.device)
    mass = torch.zeros(R, Hq, dtype=torch.float64, device=q.device)
    for r in range(R):
        n = int(length[r])
        if n == 0:
            continue
        pages = table[r, : ceil(n, ps)].long()
        kr = k[pages].double().transpose(0, 1).reshape(H, -1, D)[:, :n]
        vr = v[pages].double().transpose(0, 1).reshape(H, -1, D)[:, :n]
        qr = q[r].double().view(H, Hq // H, D)
        s = scale * torch.einsum("hgd,hnd->hgn", qr, kr)
        lse[r] = torch.logsumexp(s, -1).view(-1)
        p = torch.softmax(s, -1)
        out[r] = torch.einsum("hgn,hnd->hgd", p, vr).reshape(Hq, D)
        spread[r] = torch.einsum("hgn,hnd->hgd", p, vr.abs()).reshape(Hq, D)
        mass[r] = abs(scale) * torch.einsum("hgd,hnd->hgn", qr.abs(), kr.abs()).amax(-1).view(-1)
    return out, lse, spread, mass


def fork(table, length, refs, src, ps, n_pages):
    """-> table, length, refs, copies [(from, to)], whether pages ran out.  Lists of ints."""
    refs = list(refs)
    for t, n in zip(table, length):
        for p in t[: ceil(n, ps)]:
            refs[p] -= 1
    M = len(table[0])
    rows, lens, taken, wanted = [], [], set(), []
    for i, s in enumerate(src):
        if s < 0:
            rows.append([-1] * M)
            lens.append(0)
            continue
        n = length[s]
        used = ceil(n, ps)
        row = list(table[s][:used]) + [-1] * (M - used)
        full = n // ps
        for p in row[:full]:
            refs[p] += 1
        if n % ps:
            if s in taken:
                wanted.append((i, full))
            else:
                refs[row[full]] += 1
        taken.add(s)
        rows.append(row)
        lens.append(n)
    free = iter([p for p in range(n_pages) if refs[p] == 0])
    copies, short = [], False
    for i, j in wanted:
        p = next(free, None)
        if p is None:
            rows[i][j], lens[i], short = -1, j * ps, True
            continue
        copies.append((rows[i][j], p))
        rows[i][j], refs[p] = p, 1
    return rows, lens, refs, copies, short


def pack(table, length, refs, ps):
    refs = list(refs)
    n_live = sum(c > 0 for c in refs)
    holes = [p for p in range(n_live) if refs[p] == 0]
    movers = [p for p in range(n_live, len(refs)) if refs[p] > 0]
    to = {p: p for p, c in enumerate(refs) if c > 0}
    to.update(zip(movers, holes))
    for a, b in zip(movers, holes):
        refs[b], refs[a] = refs[a], 0
    rows = [[to[p] if j < ceil(n, ps) else -1 for j, p in enumerate(t)] for t, n in zip(table, length)]
    return rows, refs, list(zip(movers, holes)), [to.get(p, -1) for p in range(len(refs))]


def extend(table, length, refs, n_new, ps):
    refs, table, length = list(refs), [list(t) for t in table], list(length)
    M = len(table[0])
    free = iter([p for p, c in enumerate(refs) if c == 0])
    left = sum(c == 0 for c in refs)
    short = dry = False
    for r, add in enumerate(n_new):
        if length[r] + add > M * ps:
            short = True
            continue
        have, want = ceil(length[r], ps), ceil(length[r] + add, ps)
        if dry or want - have > left:
            dry = True
            short = short or add > 0
            continue
        for j in range(have, want):
            table[r][j] = next(free)
            refs[table[r][j]] = 1
        left -= want - have
        length[r] += add
    return table, length, refs, short


def logits(x, tokens, n_tokens, n_prompt, rho, pi, phi, tau, bias_ids, bias_values, mask):
    """[R, V] in 64 bits; any rule may be None."""
    R, V = x.shape
    out = x.double().clone()
    for r in range(R):
        y = out[r]
        if tokens is not None:
            n = tokens.shape[1] if n_tokens is None else int(n_tokens[r])
            n0 = 0 if n_prompt is None else int(n_prompt[r])
            every = tokens[r, :n].long()
            made = tokens[r, n0:n].long() if n0 < n else every[:0]
            seen = torch.bincount(every[(every >= 0) & (every < V)], minlength=V) > 0
            count = torch.bincount(made[(made >= 0) & (made < V)], minlength=V).double()
            if rho is not None:
                y = torch.where(seen, torch.where(y > 0, y / rho[r].double(), y * rho[r].double()), y)
            less = torch.zeros_like(y)
            if phi is not None:
                less = less + phi[r].double() * count
            if pi is not None:
                less = less + pi[r].double() * (count > 0)
            y = torch.where(count > 0, y - less, y)
        if bias_ids is not None:
            last = {int(i): float(b) for i, b in zip(bias_ids[r], bias_values[r]) if 0 <= int(i) < V}
            for i, b in last.items():
                y[i] += b
        if tau is not None:
            y = y / tau[r].double()
        if mask is not None:
            m = mask[r if mask.shape[0] > 1 else 0]
            bits = (m[:, None] >> torch.arange(32, device=m.device, dtype=torch.int32)) & 1
            y = torch.where(bits.view(-1)[:V] > 0, y, torch.full_like(y, -math.inf))
        out[r] = y
    return out
