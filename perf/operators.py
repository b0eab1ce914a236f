"""Cases for the operators of token rollouts over a paged key-value cache: single-token attention
over the pages, forking / pruning / packing of the pages, growing the cache by new tokens, and the
rules applied to the logits.

`run` computes a case in plain torch operations (32-bit arithmetic, one rounding at the end) or,
where `own` is set, through the library's entry points.  `exact` is the definition in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
DEV = "cuda"


# ------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # the first tokens of one request: nothing to read, latency only
        dict(name="attend-one-short-row", op="attend", dtype="f32", rows=1, group=1, q_heads=32, kv_heads=8, dim=128,
             page=16, shared=0, lo=37, hi=37, new=True),
        # survivors of 8 prompts x 12 in mid-generation, every length different, new token stored on the way
        dict(name="attend-ragged-batch", op="attend", dtype="bf16", rows=96, group=1, q_heads=32, kv_heads=8, dim=128,
             page=16, shared=0, lo=1, hi=8192, new=True),
        # one very long context: the work has to be split over its length
        dict(name="attend-one-long-row", op="attend", dtype="f16", rows=1, group=1, q_heads=32, kv_heads=8, dim=128,
             page=32, shared=0, lo=131071, hi=131071, new=False),
        # 16 prompts just expanded to 48 trajectories each: the prompt's pages are shared by the group
        dict(name="attend-expanded-groups", op="attend", dtype="bf16", rows=768, group=48, q_heads=32, kv_heads=8, dim=128,
             page=16, shared=2048, lo=1, hi=512, new=True),
        # the expansion of 16 prompts to 48 trajectories: partly filled last pages are copied, 8 layers
        dict(name="fork-expand-16x48", op="expand", dtype="bf16", groups=16, fan=48, kv_heads=8, dim=128, page=16, layers=8,
             lo=500, hi=2049),
        # a pruning stage 64 x 64 -> 64 x 32: tables are compacted and the dropped rows' pages freed
        dict(name="fork-prune-64x64-to-32", op="prune", dtype="bf16", groups=64, fan=64, keep=32, kv_heads=4, dim=64, page=16,
             layers=2, shared=512, lo=1, hi=700),
        # a pool with holes after many requests came and went, packed to its front
        dict(name="pack-half-empty-pool", op="pack", dtype="bf16", rows=64, kv_heads=8, dim=128, page=16, layers=4, pages=4096,
             live=0.5),
        # one decode step of 768 rows: one token a row, some rows open a page
        dict(name="append-one-token-a-row", op="append", dtype="bf16", rows=768, kv_heads=8, dim=128, page=16, lo=0, hi=1000, new_lo=1,
             new_hi=1),
        # prompts of very different lengths written into an empty cache
        dict(name="append-ragged-prompts", op="append", dtype="f32", rows=64, kv_heads=8, dim=128, page=16, lo=0, hi=40, new_lo=0,
             new_hi=4001),
        # one row, a small vocabulary: latency
        dict(name="logits-one-row", op="logits", dtype="f32", out="f32", rows=1, vocab=32000, hist=200, bias=4),
        # an odd vocabulary (rows start off any alignment), long histories, half-precision logits to fp32
        dict(name="logits-odd-vocabulary", op="logits", dtype="f16", out="f32", rows=96, vocab=50001, hist=8191, bias=33),
        # the survivors of 64 prompts x 16 over a large vocabulary
        dict(name="logits-1024-rows", op="logits", dtype="bf16", out="bf16", rows=1024, vocab=131072, hist=2048, bias=16),
    ]


def _log(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    n = max(lo, min(hi, n))
    return n + 1 if n == 3072 else n


def draw(rng):
    op = rng.choice(["attend", "attend", "expand", "prune", "pack", "append", "logits", "logits"])
    if op == "logits":
        dt = rng.choice(["f32", "bf16", "f16"])
        vocab = _log(rng, 1000, 160000)
        rows = _log(rng, 1, max(2, min(1024, 100_000_000 // vocab)))
        return dict(op=op, dtype=dt, out=rng.choice([dt, "f32"]), rows=rows, vocab=vocab, hist=_log(rng, 1, 16000),
                    bias=rng.choice([0, 1, 7, 300]))
    dt = rng.choice(["f32", "bf16", "bf16", "f16"])
    dim = rng.choice([64, 128, 128, 256])
    kv = rng.choice([1, 2, 4, 8, 8])
    page = rng.choice([8, 16, 16, 24, 32, 64])
    if op == "attend":
        if dim * kv > 1024:
            dim = 128
        per = rng.choice([1, 2, 4, 7, 8, 16])
        if kv * per * dim == 3072:
            per = 4
        group = rng.choice([1, 1, 8, 16, 24])
        if group > 1:
            groups = _log(rng, 1, 16)
            shared = _log(rng, 16, 4096) // page * page
            hi = _log(rng, 2, 700)
        else:
            groups, shared = _log(rng, 1, 256), 0
            hi = _log(rng, 2, 60000)
        rows = groups * group
        room = 600_000_000 // (kv * max(dim, 128) * rows) - shared
        if room < 2:
            shared, room = 0, max(2, 600_000_000 // (kv * max(dim, 128) * rows))
        hi = min(hi, room)
        hi = hi + 1 if hi == 3072 else hi
        lo = rng.choice([0, 1, 1, max(1, hi // 2), hi]) if group == 1 else 1
        case = dict(op=op, dtype=dt, rows=rows, group=group, q_heads=kv * per, kv_heads=kv, dim=dim, page=page, shared=shared,
                    lo=lo, hi=hi, new=rng.choice([True, False]))
        while work(case)["bytes"] > 5e8:                  # no more than the largest listed case
            case["lo"], case["hi"] = case["lo"] // 2, case["hi"] // 2 + 1
        return case
    if op == "expand":
        groups, fan = _log(rng, 1, 16), rng.choice([2, 8, 16, 24, 48])
        hi = _log(rng, 4, 2049)
        return dict(op=op, dtype=dt, groups=groups, fan=fan, kv_heads=kv, dim=dim if kv * dim <= 1024 else 64, page=min(page, 32),
                    layers=rng.choice([1, 2, 4]), lo=max(1, hi // 4), hi=hi)
    if op == "prune":
        fan = rng.choice([16, 24, 48, 64])
        return dict(op=op, dtype=dt, groups=_log(rng, 1, 64), fan=fan, keep=max(1, fan // rng.choice([1, 2, 3])), kv_heads=min(kv, 2),
                    dim=64, page=max(16, page), layers=1, shared=rng.choice([0, 128, 512]) // page * page, lo=1, hi=_log(rng, 2, 300))
    if op == "pack":
        pages = _log(rng, 64, 4096)
        return dict(op=op, dtype=dt, rows=min(_log(rng, 1, 64), pages // 4), kv_heads=kv, dim=dim if kv * dim <= 1024 else 64,
                    page=min(page, 16), layers=rng.choice([1, 2, 3]), pages=pages, live=rng.choice([0.1, 0.3, 0.7, 0.95]))
    rows = _log(rng, 1, 768)
    new = rng.choice([1, 1, 5, max(1, min(4001, 60000 // rows))])
    return dict(op=op, dtype=dt, rows=rows, kv_heads=kv, dim=dim if kv * dim <= 1024 else 64, page=page, lo=0, hi=_log(rng, 2, 200),
                new_lo=new if new < 6 else 0, new_hi=new)


# --------------------------------------------------------------------------------- the inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, dtype):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)


def _pool(g, case, layers, pages):
    shape = (layers, pages, case["kv_heads"], case["page"], case["dim"])
    dt = DTYPES[case["dtype"]]
    k, v = torch.empty(shape, device=DEV, dtype=dt), torch.empty(shape, device=DEV, dtype=dt)
    return k.normal_(generator=g), v.normal_(generator=g)


def _ints(g, lo, hi, n):
    return torch.randint(lo, hi + 1, (n,), generator=g, device=DEV, dtype=torch.int32)


def _ragged(g, lo, hi, n, log=True):
    """n lengths spread evenly over [lo, hi] (or over its logarithm) in an order of the seed's, the largest one hi."""
    u = (torch.randperm(n, generator=g, device=DEV) + 1) / n
    if log:
        a, b = math.log(max(lo, 1)), math.log(max(hi, 1))
        x = torch.exp(a + u * (b - a))
        if lo == 0 and n > 1:
            x = torch.where(u * n < 1.5, torch.zeros_like(x), x)
    else:
        x = lo + u * (hi - lo)
    return x.round().to(torch.int32).clamp(lo, hi)


def _shuffled_table(g, n_pages, counts, width):
    """Distinct pages in random order for rows of `counts` pages; -1 past a row's last page."""
    perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    col = torch.arange(width, device=DEV, dtype=torch.int32)
    used = col[None, :] < counts[:, None]
    at = (torch.cumsum(counts, 0) - counts).long()[:, None] + col[None, :].long()
    return torch.where(used, perm[at.clamp(max=n_pages - 1)], torch.full_like(at, -1, dtype=torch.int32))


def _ceil(a, b):
    return (a + b - 1) // b


def _refs(table, n_pages):
    return torch.bincount(table[table >= 0].long(), minlength=n_pages).to(torch.int32)


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case=case)
    op, dt = case["op"], DTYPES[case["dtype"]]
    if op == "logits":
        R, V, H = case["rows"], case["vocab"], case["hist"]
        s["logits"] = (torch.randn((R, V), generator=g, device=DEV) * 3).to(dt)
        s["tokens"] = (torch.rand((R, H), generator=g, device=DEV) ** 3 * V).to(torch.int32).clamp(0, V - 1)
        s["n_tokens"] = _ints(g, 0, H, R)
        s["n_tokens"][0] = H
        s["n_prompt"] = torch.minimum(_ints(g, 0, max(1, H // 2), R), s["n_tokens"])
        s["repetition"] = 1 + torch.rand(R, generator=g, device=DEV) * 0.5
        s["presence"] = torch.rand(R, generator=g, device=DEV)
        s["frequency"] = torch.rand(R, generator=g, device=DEV) * 0.3
        s["temperature"] = 0.5 + torch.rand(R, generator=g, device=DEV)
        words = torch.randint(-2 ** 31, 2 ** 31, (R, _ceil(V, 32)), generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
        s["mask"] = torch.where(_ints(g, 0, 1, R)[:, None] > 0, words, torch.full_like(words, -1))
        if R > 2:
            s["mask"][R // 2] = 0                      # a grammar that allows nothing
        nb = case["bias"]
        s["bias_ids"] = torch.arange(R, device=DEV, dtype=torch.int32)[:, None] * 3 + \
            (torch.randperm(V, generator=g, device=DEV)[:nb]).to(torch.int32)[None, :]
        s["bias_ids"] = (s["bias_ids"] % V).to(torch.int32).contiguous()
        s["bias_values"] = torch.randn((R, nb), generator=g, device=DEV) * 4
        s["out"] = torch.empty((R, V), device=DEV, dtype=DTYPES[case["out"]])
    elif op == "attend":
        R, N, ps, hi = case["rows"], case["group"], case["page"], case["hi"]
        own_len = _ragged(g, case["lo"], hi, R)
        s["len"] = own_len + case["shared"]
        groups, common = R // N, case["shared"] // ps
        counts = _ceil(own_len, ps)
        width = common + _ceil(hi, ps)
        total = int(counts.sum()) + groups * common
        n_pages = total + max(2, total // 16)
        perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
        first = perm[: groups * common].view(groups, 1, common).expand(groups, N, common).reshape(R, common)
        rest = _shuffled_table(g, n_pages - groups * common, counts, width - common)
        rest = torch.where(rest >= 0, perm[groups * common + rest.clamp(min=0).long()], rest)
        s["table"] = torch.cat([first, rest], 1).contiguous()
        s["shared"] = torch.full((groups,), case["shared"], device=DEV, dtype=torch.int32)
        s["k"], s["v"] = _pool(g, case, 1, n_pages)
        sharp = 0.5 + 2 * torch.rand((1, case["q_heads"], 1), generator=g, device=DEV)
        s["q"] = (torch.randn((R, case["q_heads"], case["dim"]), generator=g, device=DEV) * sharp).to(dt)
        if case["new"]:
            s["k_new"] = _normal(g, (R, case["kv_heads"], case["dim"]), dt)
            s["v_new"] = _normal(g, (R, case["kv_heads"], case["dim"]), dt)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((R, case["q_heads"]), device=DEV)
    elif op in ("expand", "prune"):
        G, N, ps = case["groups"], case["fan"], case["page"]
        if op == "expand":
            s["len"] = _ragged(g, case["lo"], case["hi"], G)
            counts = _ceil(s["len"], ps)
            width = _ceil(case["hi"], ps)
            total = int(counts.sum())
            n_pages = total + G * N + 64
            s["table"] = _shuffled_table(g, n_pages, counts, width)
            s["src"] = torch.arange(G, device=DEV, dtype=torch.int32).repeat_interleave(N)
        else:
            R, common = G * N, case["shared"] // ps
            own_len = _ragged(g, case["lo"], case["hi"], R)
            s["len"] = own_len + common * ps
            counts = _ceil(own_len, ps)
            width = common + _ceil(case["hi"], ps)
            total = int(counts.sum()) + G * common
            n_pages = total + 64
            rest = _shuffled_table(g, n_pages - G * common, counts, width - common)
            first = torch.arange(n_pages - G * common, n_pages, device=DEV, dtype=torch.int32)
            first = first.view(G, 1, common).expand(G, N, common).reshape(R, common)
            s["table"] = torch.cat([first, rest], 1).contiguous()
            keep = torch.rand((G, N), generator=g, device=DEV).argsort(1)[:, : case["keep"]].sort(1).values
            s["src"] = (keep + torch.arange(G, device=DEV)[:, None] * N).reshape(-1).to(torch.int32)
        s["refs"] = _refs(s["table"], n_pages)
        s["k"], s["v"] = _pool(g, case, case["layers"], n_pages)
        n_out = s["src"].numel()
        s["table_out"] = torch.empty((n_out, width), device=DEV, dtype=torch.int32)
        s["len_out"] = torch.empty(n_out, device=DEV, dtype=torch.int32)
        s["refs_out"] = torch.empty_like(s["refs"])
    elif op == "pack":
        R, P, ps = case["rows"], case["pages"], case["page"]
        total = max(R, int(P * case["live"]))
        counts = torch.full((R,), total // R, device=DEV, dtype=torch.int32)
        counts[: total % R] += 1
        width = total // R + 1
        s["table"] = _shuffled_table(g, P, counts, width)
        s["len"] = counts * ps - _ints(g, 0, ps - 1, R)
        s["refs"] = _refs(s["table"], P)
        s["k"], s["v"] = _pool(g, case, case["layers"], P)
        s["table_out"] = torch.empty_like(s["table"])
        s["refs_out"] = torch.empty_like(s["refs"])
    else:
        R, ps = case["rows"], case["page"]
        s["len"] = _ragged(g, case["lo"], case["hi"], R, log=False)
        s["n_new"] = _ragged(g, case["new_lo"], case["new_hi"], R)
        s["tokens"] = int(s["n_new"].sum())
        s["start"] = torch.cat([torch.zeros(1, device=DEV, dtype=torch.int32), torch.cumsum(s["n_new"], 0).to(torch.int32)])
        counts = _ceil(s["len"], ps)
        width = _ceil(case["hi"] + case["new_hi"], ps)
        n_pages = int((counts + _ceil(s["n_new"], ps)).sum()) + 16
        s["table"] = _shuffled_table(g, n_pages, counts, width)
        s["refs"] = _refs(s["table"], n_pages)
        s["k"], s["v"] = _pool(g, case, 1, n_pages)
        s["k_new"] = _normal(g, (s["tokens"], case["kv_heads"], case["dim"]), dt)
        s["v_new"] = _normal(g, (s["tokens"], case["kv_heads"], case["dim"]), dt)
        s["len_out"] = torch.empty_like(s["len"])
        s["refs_out"] = torch.empty_like(s["refs"])
    if own:
        _handles(s)
    return s


def _handles(s):
    """Descriptors, rules and workspace that a program keeps next to its buffers."""
    from paper_2512_15347_b200 import binding as B
    op = s["case"]["op"]
    s["status"] = torch.zeros(1, device=DEV, dtype=torch.int32)
    if op == "logits":
        s["rules"] = B.make_logits_rules(tokens=s["tokens"], n_tokens=s["n_tokens"], n_prompt=s["n_prompt"],
                                         repetition=s["repetition"], presence=s["presence"], frequency=s["frequency"],
                                         bias_ids=s["bias_ids"], bias_values=s["bias_values"], mask=s["mask"],
                                         temperature=s["temperature"])
        return
    s["kv"] = B.make_kv(s["k"], s["v"], s["table"], s["len"])
    if op == "append":
        s["kv_grown"] = B.make_kv(s["k"], s["v"], s["table"], s["len_out"])
        return
    need = {"attend": lambda: B.kv_attend_workspace_bytes(s["kv"], s["case"].get("q_heads"), s["case"].get("group")),
            "expand": lambda: B.kv_fork_workspace_bytes(s["kv"], s["src"].numel()),
            "prune": lambda: B.kv_fork_workspace_bytes(s["kv"], s["src"].numel()),
            "pack": lambda: B.kv_pack_workspace_bytes(s["kv"])}[op]()
    s["workspace"] = torch.zeros(need, device=DEV, dtype=torch.uint8)


# -------------------------------------------------------------------------------- one pass

def run(s):
    op = s["case"]["op"]
    if own:
        return _own(s, op)
    return {"attend": _attend, "expand": _fork, "prune": _fork, "pack": _pack, "append": _append, "logits": _logits}[op](s)


def _own(s, op):
    from paper_2512_15347_b200 import binding as B
    if op == "attend":
        c = s["case"]
        B.kv_attend(s["kv"], 0, s["q"], s["out"], s["workspace"], k_new=s.get("k_new"), v_new=s.get("v_new"), lse=s["lse"],
                    scale=c["dim"] ** -0.5, group=c["group"], shared=s["shared"] if c["group"] > 1 else None, status=s["status"])
        return _attend_result(s, s["out"], s["lse"])
    if op in ("expand", "prune"):
        B.kv_fork(s["kv"], s["src"], s["table_out"], s["len_out"], s["refs"], s["refs_out"], s["workspace"], status=s["status"])
        return dict(table=s["table_out"], len=s["len_out"], refs=s["refs_out"], k=s["k"], v=s["v"])
    if op == "pack":
        B.kv_pack(s["kv"], s["refs"], s["refs_out"], s["table_out"], s["workspace"], status=s["status"])
        return dict(table=s["table_out"], refs=s["refs_out"], k=s["k"], v=s["v"])
    if op == "append":
        B.kv_extend(s["kv"], s["n_new"], s["len_out"], s["refs"], s["refs_out"], status=s["status"])
        B.kv_append(s["kv_grown"], 0, s["k_new"], s["v_new"], s["start"], status=s["status"])
        return dict(table=s["table"], len=s["len_out"], refs=s["refs_out"], k=s["k"], v=s["v"])
    B.logits_process(s["logits"], s["out"], s["rules"])
    return s["out"]


def _attend_result(s, out, lse):
    if s["case"]["new"]:
        return dict(out=out, lse=lse, k=s["k"], v=s["v"])
    return dict(out=out, lse=lse)


def _attend(s):
    c = s["case"]
    k, v, table, length, q = s["k"][0], s["v"][0], s["table"], s["len"].long(), s["q"]
    R, H, D, ps = c["rows"], c["kv_heads"], c["dim"], c["page"]
    if c["new"]:
        some = length > 0
        pos = (length - 1).clamp(min=0)
        page = table.gather(1, (pos // ps)[:, None])[:, 0].long().clamp(min=0)
        keep = some[:, None, None]
        k[page, :, pos % ps] = torch.where(keep, s["k_new"], k[page, :, pos % ps])
        v[page, :, pos % ps] = torch.where(keep, s["v_new"], v[page, :, pos % ps])
    at = table.clamp(min=0).long()
    T = table.shape[1] * ps
    there = (torch.arange(T, device=DEV)[None, :] < length[:, None])[:, None, None, :]
    qf = q.float().view(R, H, -1, D) * D ** -0.5
    score = torch.matmul(qf, k[at].float().permute(0, 2, 4, 1, 3).reshape(R, H, D, T))
    score = torch.where(there, score, torch.full_like(score, -math.inf))
    top = score.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v[at].float().permute(0, 2, 1, 3, 4).reshape(R, H, T, D)) / total.clamp(min=1e-38)
    lse = (torch.log(total) + top).view(R, -1)
    return _attend_result(s, out.view(R, -1, D).to(q.dtype), lse)


def _fork(s):
    table, length, src, refs = s["table"], s["len"], s["src"].long(), s["refs"]
    R, M = table.shape
    ps, n = s["case"]["page"], src.numel()
    col = torch.arange(M, device=DEV)
    order = torch.arange(n, device=DEV)
    children = torch.zeros(R, device=DEV, dtype=torch.int32).scatter_add_(0, src, torch.ones_like(src, dtype=torch.int32))
    first = torch.full((R,), n, device=DEV, dtype=torch.int64).scatter_reduce_(0, src, order, "amin")
    pages, part = _ceil(length, ps), length % ps != 0
    is_last = (col[None, :] == pages[:, None] - 1) & part[:, None]
    delta = torch.where(is_last, children.clamp(max=1)[:, None], children[:, None]) - 1
    used = col[None, :] < pages[:, None]
    new_refs = refs.clone().scatter_add_(0, table.clamp(min=0).long().view(-1), torch.where(used, delta, 0).int().view(-1))
    new_len = length[src]
    new_table = torch.where(used[src], table[src], -1)
    copied = part[src] & (first[src] != order)
    rows = torch.nonzero(copied)[:, 0]
    dst = torch.nonzero(new_refs == 0)[: rows.numel(), 0]
    last = pages[src][rows].long() - 1
    origin = new_table[rows, last].long()
    new_table[rows, last] = dst.int()
    new_refs[dst] = 1
    s["k"][:, dst] = s["k"][:, origin]
    s["v"][:, dst] = s["v"][:, origin]
    return dict(table=new_table, len=new_len, refs=new_refs, k=s["k"], v=s["v"])


def _pack(s):
    table, refs = s["table"], s["refs"]
    P = refs.numel()
    live = refs > 0
    n_live = live.sum()
    index = torch.arange(P, device=DEV)
    movers = torch.nonzero(live & (index >= n_live))[:, 0]
    holes = torch.nonzero(~live & (index < n_live))[:, 0]
    to = index.clone()
    to[movers] = holes
    new_refs = refs.clone()
    new_refs[holes] = refs[movers]
    new_refs[movers] = 0
    s["k"][:, holes] = s["k"][:, movers]
    s["v"][:, holes] = s["v"][:, movers]
    used = torch.arange(table.shape[1], device=DEV)[None, :] < _ceil(s["len"], s["case"]["page"])[:, None]
    new_table = torch.where(used, to[table.clamp(min=0).long()].int(), -1)
    return dict(table=new_table, refs=new_refs, k=s["k"], v=s["v"])


def _append(s):
    table, length, n_new, refs = s["table"], s["len"].long(), s["n_new"].long(), s["refs"]
    ps = s["case"]["page"]
    have, want = _ceil(length, ps), _ceil(length + n_new, ps)
    col = torch.arange(table.shape[1], device=DEV)[None, :]
    opened = (col >= have[:, None]) & (col < want[:, None])
    free = torch.nonzero(refs == 0)[:, 0].int()
    rank = (torch.cumsum(opened.view(-1).int(), 0) - 1).view_as(opened).clamp(min=0)
    table.copy_(torch.where(opened, free[rank.clamp(max=free.numel() - 1)], table))
    new_refs = refs.clone()
    new_refs[free[: opened.sum()].long()] = 1
    new_len = (length + n_new).int()
    token = torch.arange(s["tokens"], device=DEV)
    row = torch.searchsorted(s["start"][1:].long(), token, right=True)
    pos = length[row] + token - s["start"][row].long()
    page = table[row, pos // ps].long()
    s["k"][0][page, :, pos % ps] = s["k_new"]
    s["v"][0][page, :, pos % ps] = s["v_new"]
    return dict(table=table, len=new_len, refs=new_refs, k=s["k"], v=s["v"])


def _logits(s):
    x = s["logits"].float()
    R, V = x.shape
    tokens = s["tokens"].long()
    at = torch.arange(tokens.shape[1], device=DEV)[None, :]
    there = at < s["n_tokens"][:, None]
    made = there & (at >= s["n_prompt"][:, None])
    seen = torch.zeros((R, V), device=DEV).scatter_add_(1, tokens, there.float())
    count = torch.zeros((R, V), device=DEV).scatter_add_(1, tokens, made.float())
    rho = s["repetition"][:, None]
    x = torch.where(seen > 0, torch.where(x > 0, x / rho, x * rho), x)
    x = x - (s["frequency"][:, None] * count + s["presence"][:, None] * (count > 0))
    x = x.scatter_add(1, s["bias_ids"].long(), s["bias_values"])
    x = x / s["temperature"][:, None]
    token = torch.arange(V, device=DEV)
    allowed = (s["mask"][:, token // 32] >> (token % 32)[None, :]) & 1
    return torch.where(allowed > 0, x, -math.inf).to(s["out"].dtype)


# ------------------------------------------------------------------------------- the work

def work(case):
    op, b = case["op"], {"f32": 4, "bf16": 2, "f16": 2}[case["dtype"]]
    if op == "logits":
        out = {"f32": 4, "bf16": 2, "f16": 2}[case["out"]]
        R, V = case["rows"], case["vocab"]
        return dict(bytes=R * (V * (b + out) + V / 8 + 2 * case["hist"] + 8 * case["bias"]), flops=R * V * 4)
    token = 2 * case["kv_heads"] * case["dim"] * b                  # K and V of one token in one layer
    lo, hi = max(1, case.get("lo", 1)), max(1, case.get("hi", 1))
    mean = (hi - lo) / math.log(hi / lo) if hi > lo else hi         # of lengths spread over the logarithm
    if op == "attend":
        R, groups = case["rows"], case["rows"] // case["group"]
        mean = hi if R == 1 else mean
        read = (R * mean + groups * case["shared"]) * token
        io = R * case["q_heads"] * (2 * case["dim"] * b + 4) + (2 * R * token if case["new"] else 0)
        return dict(bytes=read + io, flops=4 * R * (mean + case["shared"]) * case["q_heads"] * case["dim"])
    page = token * case["page"] * case.get("layers", 1)
    if op == "expand":
        G, N = case["groups"], case["fan"]
        return dict(bytes=2 * page * G * (N - 1) * (1 - 1 / case["page"]) + 4 * G * (N + 1) * mean / case["page"], flops=0)
    if op == "prune":
        G, common = case["groups"], case["shared"] / case["page"]
        return dict(bytes=4 * G * (case["fan"] + case["keep"]) * (mean / case["page"] + common), flops=0)
    if op == "pack":
        return dict(bytes=2 * page * case["pages"] * case["live"] * (1 - case["live"]) + 16 * case["pages"], flops=0)
    lo, hi = max(1, case["new_lo"]), max(1, case["new_hi"])
    return dict(bytes=2 * token * case["rows"] * ((hi - lo) / math.log(hi / lo) if hi > lo else hi), flops=0)


# ----------------------------------------------------------------------- the definition, 64 bits

def exact(case, seed):
    """What run() returns, row by row from the operator's definition."""
    s = prepare(case, seed)
    return {"attend": _exact_attend, "logits": _exact_logits}.get(case["op"], _exact_pages)(s)


def _exact_attend(s):
    c = s["case"]
    per, ps = c["q_heads"] // c["kv_heads"], c["page"]
    k, v = s["k"][0], s["v"][0]
    lens, table = s["len"].tolist(), s["table"].long()
    if c["new"]:
        for r, n in enumerate(lens):
            if n:
                k[table[r, (n - 1) // ps], :, (n - 1) % ps] = s["k_new"][r]
                v[table[r, (n - 1) // ps], :, (n - 1) % ps] = s["v_new"][r]
    out = torch.zeros(s["q"].shape, device=DEV, dtype=torch.float64)
    lse = torch.full(s["lse"].shape, -math.inf, device=DEV, dtype=torch.float64)
    for r, n in enumerate(lens):
        if not n:
            continue
        pages = table[r, : _ceil(n, ps)]
        kr = k[pages].double().transpose(0, 1).flatten(1, 2)[:, :n]
        vr = v[pages].double().transpose(0, 1).flatten(1, 2)[:, :n]
        qr = s["q"][r].double().view(c["kv_heads"], per, -1)
        logit = torch.einsum("hgd,htd->hgt", qr, kr) / math.sqrt(c["dim"])
        lse[r] = torch.logsumexp(logit, -1).view(-1)
        out[r] = torch.einsum("hgt,htd->hgd", torch.softmax(logit, -1), vr).reshape(c["q_heads"], -1)
    return dict(out=out, lse=lse, k=s["k"], v=s["v"]) if c["new"] else dict(out=out, lse=lse)


def _exact_logits(s):
    R, V = s["logits"].shape
    out = torch.empty((R, V), device=DEV, dtype=torch.float64)
    bits = torch.arange(32, device=DEV, dtype=torch.int32)
    for r in range(R):
        x = s["logits"][r].double()
        n, n0 = int(s["n_tokens"][r]), int(s["n_prompt"][r])
        seen = torch.bincount(s["tokens"][r, :n].long(), minlength=V) > 0
        count = torch.bincount(s["tokens"][r, n0:n].long(), minlength=V).double()
        rho = s["repetition"][r].double()
        x[seen] = torch.maximum(x[seen], x.new_zeros(())) / rho + torch.minimum(x[seen], x.new_zeros(())) * rho
        x -= s["frequency"][r].double() * count + s["presence"][r].double() * (count > 0)
        x[s["bias_ids"][r].long()] += s["bias_values"][r].double()
        x /= s["temperature"][r].double()
        allowed = ((s["mask"][r][:, None] >> bits[None, :]) & 1).view(-1)[:V].bool()
        out[r] = torch.where(allowed, x, -math.inf)
    return out


def _exact_pages(s):
    """Page operations copy values: the pools are followed page by page on the host's lists."""
    c, ps = s["case"], s["case"]["page"]
    table, lens, refs = s["table"].tolist(), s["len"].tolist(), s["refs"].tolist()
    k, v = s["k"], s["v"]
    if c["op"] == "pack":
        n_live = sum(x > 0 for x in refs)
        holes = [p for p in range(n_live) if refs[p] == 0]
        movers = [p for p in range(n_live, len(refs)) if refs[p] > 0]
        moves = list(zip(movers, holes))
        to = dict(moves)
        table = [[to.get(p, p) if j < _ceil(n, ps) else -1 for j, p in enumerate(t)] for t, n in zip(table, lens)]
        for a, b in moves:
            refs[b], refs[a] = refs[a], 0
        new = dict(table=table, refs=refs)
    elif c["op"] == "append":
        free = iter([p for p, x in enumerate(refs) if x == 0])
        moves, t = [], 0
        kn, vn = s["k_new"], s["v_new"]
        for r, n in enumerate(s["n_new"].tolist()):
            for j in range(_ceil(lens[r], ps), _ceil(lens[r] + n, ps)):
                table[r][j] = next(free)
                refs[table[r][j]] = 1
            done = 0
            while done < n:
                pos = lens[r] + done
                m = min(ps - pos % ps, n - done)
                k[0, table[r][pos // ps], :, pos % ps: pos % ps + m] = kn[t: t + m].transpose(0, 1)
                v[0, table[r][pos // ps], :, pos % ps: pos % ps + m] = vn[t: t + m].transpose(0, 1)
                done, t = done + m, t + m
            lens[r] += n
        new = dict(table=table, len=lens, refs=refs)
    else:
        src = s["src"].tolist()
        taken, rows, wanted = set(), [], []
        for r, n in enumerate(lens):
            for j in range(_ceil(n, ps)):
                refs[table[r][j]] -= 1
        for i, r in enumerate(src):
            n, last = lens[r], _ceil(lens[r], ps) - 1
            row = [p if j <= last else -1 for j, p in enumerate(table[r])]
            for p in row[: last + 1]:
                refs[p] += 1
            if n % ps and r in taken:
                refs[row[last]] -= 1
                wanted.append((i, last))
            taken.add(r)
            rows.append(row)
        free = iter([p for p, x in enumerate(refs) if x == 0])
        moves = []
        for i, j in wanted:
            p = next(free)
            moves.append((rows[i][j], p))
            rows[i][j], refs[p] = p, 1
        new = dict(table=rows, len=[lens[r] for r in src], refs=refs)
    if moves:
        a, b = torch.tensor(moves, device=DEV).unbind(1)
        k[:, b], v[:, b] = k[:, a], v[:, a]
    return dict({name: torch.tensor(x, device=DEV, dtype=torch.int32) for name, x in new.items()}, k=k, v=v)
