"""The token-rollout calls against plain 64-bit forms: single-token attention over the paged cache,
forking / dropping / packing pages, growing the cache, rules on logits; their refusals."""
import math

import pytest
import torch

from paper_2512_15347_b200 import binding as B
from tests import kv_reference as ref

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {name: torch.finfo(dt).eps / 2 for name, dt in DT.items()}     # relative error of one rounding to the type


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def status_word():
    return torch.zeros(1, device="cuda", dtype=torch.int32)


class Cache:
    """Rows of the given lengths over randomly numbered pages.  Whatever no row owns (free pages, slots
    past a row's length, table entries past its last page) holds NaN, infinities or wild numbers."""

    def __init__(self, lens, heads, dim, page, dtype="bf16", layers=1, spare=3, seed=0, width=None, k=None, v=None):
        g = gen(seed)
        self.lens, self.page = list(lens), page
        need = [ref.ceil(n, page) for n in lens]
        self.n_pages = sum(need) + spare
        self.width = width or max(need + [1])
        if k is None:
            shape = (layers, self.n_pages, heads, page, dim)
            k, v = (torch.full(shape, float("nan"), device="cuda", dtype=DT[dtype]) for _ in range(2))
            v[:, ::2] = float("inf")
        self.k, self.v = k, v
        order = torch.randperm(self.n_pages, generator=g, device="cuda").tolist()
        self.rows, at = [], 0
        for r, n in enumerate(lens):
            own = order[at: at + need[r]]
            at += need[r]
            self.rows.append(own + [2 ** 31 - 1 if j % 2 else -7 for j in range(self.width - need[r])])
            for j, p in enumerate(own):
                m = min(page, n - j * page)
                for pool in (self.k, self.v):
                    pool[:, p, :, :m] = torch.randn((layers, heads, m, dim), generator=g, device="cuda").to(DT[dtype])
        self.table = torch.tensor(self.rows, device="cuda", dtype=torch.int32).view(len(self.lens), self.width)
        self.len = torch.tensor(self.lens, device="cuda", dtype=torch.int32)
        self.refs = torch.zeros(self.n_pages, device="cuda", dtype=torch.int32)
        for row, n in zip(self.rows, lens):
            for p in row[: ref.ceil(n, page)]:
                self.refs[p] += 1
        self.kv = B.make_kv(self.k, self.v, self.table, self.len)


def check_attention(c, q, out, lse, scale, dtype, layer=0):
    """|out - exact| against what the arithmetic can lose, element by element.

    One rounding of the result (u |o|); in 16 bits the weights p are rounded too, and the sum l may be
    that of the rounded ones (2 u sum p|v|).  A score is a sum of D products in fp32: at most D + 2
    roundings of sum |q||k| scale (2^-24 each), and the hardware's exponential is good to 2^-22 of its result plus
    2^-23 of its argument's size, all of which move p relative to l twice; the join over the row's
    parts rounds a handful of times."""
    want, want_lse, spread, mass = ref.attend(q, c.k[layer], c.v[layer], c.table, c.len, scale)
    u = UNIT[dtype]
    D = q.shape[-1]
    moved = (D + 4) * 2.0 ** -24 * mass + 2.0 ** -22 + 64 * 2.0 ** -24
    bound = u * want.abs() + (2 * moved[..., None] + (2 * u if dtype != "f32" else 0)) * spread + 1e-30
    if dtype == "f16":
        bound = bound + 2.0 ** -24          # subnormal results
    assert torch.isfinite(out.double()).all()
    off = (out.double() - want).abs()
    assert (off <= bound).all(), (off / bound).max().item()
    if lse is not None:
        empty = c.len == 0
        assert torch.equal(torch.isinf(lse).all(1), empty) and (lse[empty] < 0).all()
        d = (lse.double() - want_lse).abs()[~empty]
        lim = (moved + 2.0 ** -23 * (1 + want_lse.abs()))[~empty]
        assert (d <= lim).all(), (d / lim).max().item()


def run_attention(c, q, dtype, scale=None, layer=0, group=1, shared=None, new=None, lse=True, ws=None, out=None, stream=None):
    R, Hq, D = q.shape
    out = torch.full_like(q, float("nan")) if out is None else out
    l = torch.full((R, Hq), float("nan"), device="cuda") if lse else None
    st = status_word()
    ws = torch.zeros(B.kv_attend_workspace_bytes(c.kv, Hq, group), device="cuda", dtype=torch.uint8) if ws is None else ws
    kn, vn = new if new else (None, None)
    B.kv_attend(c.kv, layer, q, out, ws, k_new=kn, v_new=vn, lse=l, scale=scale, group=group, shared=shared, status=st, stream=stream)
    B.kv_status(st, stream)
    return out, l


def queries(R, Hq, D, dtype, seed=1, sharp=1.0):
    return (torch.randn((R, Hq, D), generator=gen(seed), device="cuda") * sharp).to(DT[dtype])


# ------------------------------------------------------------------------------ attention

@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 8), (8, 1), (32, 8), (14, 2), (20, 1), (9, 3), (48, 1)])
@pytest.mark.parametrize("dim", [64, 128])
def test_attention_head_layouts(dtype, heads, kv_heads, dim):
    c = Cache([37, 0, 1, 200, 64, 129], kv_heads, dim, 16, dtype)
    q = queries(6, heads, dim, dtype, sharp=2.0)
    out, lse = run_attention(c, q, dtype)
    check_attention(c, q, out, lse, dim ** -0.5, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim", [8, 16, 24, 40, 72, 80, 96, 112, 136, 192, 248, 256])
def test_attention_head_dims(dtype, dim):
    c = Cache([0, 1, 15, 70, 331], 2, dim, 16, dtype, seed=dim)
    for heads in (2, 24):
        q = queries(5, heads, dim, dtype, sharp=1.5)
        out, lse = run_attention(c, q, dtype)
        check_attention(c, q, out, lse, dim ** -0.5, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page", [1, 3, 5, 8, 12, 16, 24, 32, 100, 256])
def test_attention_page_sizes(dtype, page):
    """Pages that end inside any tile, lengths around their ends."""
    lens = [1, 2, page, page + 1, max(page - 1, 0), 3 * page, 3 * page + 1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 500]
    c = Cache(lens, 2, 64, page, dtype, seed=page)
    q = queries(len(lens), 8, 64, dtype)
    out, lse = run_attention(c, q, dtype)
    check_attention(c, q, out, lse, 0.125, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("lens", [[70001], [40000, 3, 0, 9000], [1] * 700, [0] * 9 + [777] + [0] * 30, [0, 0],
                                  [5000 - 37 * i for i in range(130)]])
def test_attention_split_over_long_and_many_rows(dtype, lens):
    c = Cache(lens, 2, 64, 16, dtype, seed=3)
    q = queries(len(lens), 8, 64, dtype, sharp=3.0)
    out, lse = run_attention(c, q, dtype)
    check_attention(c, q, out, lse, 0.125, dtype)
    again, lse2 = run_attention(c, q, dtype)
    assert torch.equal(out, again) and torch.equal(lse, lse2)       # the same bits on every run


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("scale", [0.0, -0.3, 0.05, 8.0])
def test_attention_scales(dtype, scale):
    """Uniform weights, a negative scale, weights that fall on one token."""
    c = Cache([300, 17, 1000], 2, 64, 16, dtype, seed=5)
    q = queries(3, 4, 64, dtype)
    out, lse = run_attention(c, q, dtype, scale=scale)
    check_attention(c, q, out, lse, scale, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_attention_largest_score_last_and_scores_far_below(dtype):
    """The running maximum rises at every token; then tokens whose weights vanish."""
    c = Cache([900, 900], 1, 64, 16, dtype, seed=6)
    ramp = torch.linspace(0, 1, 900, device="cuda")
    for r, f in ((0, ramp), (1, ramp.flip(0))):
        for t in range(900):
            c.k[0, c.rows[r][t // 16], 0, t % 16] = (f[t] * 4).to(DT[dtype])
    q = torch.full((2, 2, 64), 1.0, device="cuda", dtype=DT[dtype])
    q[:, 1] = -1.0
    out, lse = run_attention(c, q, dtype, scale=1.0)
    check_attention(c, q, out, lse, 1.0, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_attention_infinite_scores(dtype):
    """A key of -inf against a positive query takes no weight; a row whose every score is -inf is left
    empty (zeros, lse -inf); NaN stays NaN."""
    c = Cache([40, 20, 33], 1, 64, 16, dtype, seed=8)
    q = queries(3, 3, 64, dtype).abs() + 0.1
    def key(r, t):
        return c.k[0, c.rows[r][t // 16], 0, t % 16]
    for t in (0, 7, 16, 39):
        key(0, t)[:] = -math.inf
    for t in range(20):
        key(1, t)[5] = -math.inf
    key(2, 32)[3] = math.nan
    R, Hq, D = q.shape
    out, lse = run_attention(c, q, dtype)
    keep = [t for t in range(40) if t not in (0, 7, 16, 39)]
    d = Cache([36], 1, 64, 16, dtype, seed=9)
    for i, t in enumerate(keep):
        for a, b in ((c.k, d.k), (c.v, d.v)):
            b[0, d.rows[0][i // 16], 0, i % 16] = a[0, c.rows[0][t // 16], 0, t % 16]
    check_attention(d, q[:1], out[:1], lse[:1], 0.125, dtype)
    assert (out[1] == 0).all() and (lse[1] == -math.inf).all()
    assert torch.isnan(out[2]).all() and torch.isnan(lse[2]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("heads,kv_heads,dim,page", [(8, 2, 64, 16), (40, 2, 128, 8), (4, 4, 256, 24), (6, 1, 72, 3)])
def test_attention_stores_the_new_token(dtype, heads, kv_heads, dim, page):
    """k_new / v_new: token len-1 comes from them and lands in its page; nothing else changes.  The
    new tokens and the queries are slices of one projection's output (strided rows)."""
    lens = [1, page, page + 1, 0, 400, 33]
    R = len(lens)
    c = Cache(lens, kv_heads, dim, page, dtype, layers=2, seed=11)
    for r, n in enumerate(lens):                       # the last token's slot is not written yet
        if n:
            for pool in (c.k, c.v):
                pool[1, c.rows[r][(n - 1) // page], :, (n - 1) % page] = math.nan
    fused = torch.randn((R, heads + 2 * kv_heads, dim), generator=gen(12), device="cuda").to(DT[dtype])
    q, kn, vn = fused[:, :heads], fused[:, heads: heads + kv_heads], fused[:, heads + kv_heads:]
    wide = torch.full((R, heads + 5, dim), -1.0, device="cuda", dtype=DT[dtype])
    want_k, want_v = c.k.clone(), c.v.clone()
    for r, n in enumerate(lens):
        if n:
            want_k[1, c.rows[r][(n - 1) // page], :, (n - 1) % page] = kn[r]
            want_v[1, c.rows[r][(n - 1) // page], :, (n - 1) % page] = vn[r]
    out, lse = run_attention(c, q, dtype, layer=1, new=(kn, vn), out=wide[:, :heads])
    assert torch.equal(c.k.nan_to_num(7.0), want_k.nan_to_num(7.0)) and torch.equal(c.v.nan_to_num(7.0), want_v.nan_to_num(7.0))
    check_attention(c, q, out, lse, dim ** -0.5, dtype, layer=1)
    assert (wide[:, heads:] == -1.0).all()


def shared_cache(groups, n, shared, tails, heads, dim, page, dtype, seed=0):
    """Rows of group-shared first pages and tails of their own."""
    heads_c = Cache([shared] * groups, heads, dim, page, dtype, seed=seed)
    c = Cache(tails, heads, dim, page, dtype, seed=seed + 1, spare=heads_c.n_pages)
    free = [p for p in range(c.n_pages) if int(c.refs[p]) == 0]
    full = shared // page
    rows = []
    for g in range(groups):
        mine = [free.pop() for _ in range(full)]
        for j, p in enumerate(mine):
            c.k[:, p], c.v[:, p] = heads_c.k[:, heads_c.rows[g][j]], heads_c.v[:, heads_c.rows[g][j]]
        for i in range(n):
            rows.append(mine + c.rows[g * n + i])
    c.rows, c.lens = rows, [shared + t for t in tails]
    c.table = torch.tensor(rows, device="cuda", dtype=torch.int32)
    c.len = torch.tensor(c.lens, device="cuda", dtype=torch.int32)
    c.kv = B.make_kv(c.k, c.v, c.table, c.len)
    return c


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("groups,n,shared,heads,kv_heads,dim,page", [
    (2, 16, 64, 8, 2, 64, 16), (1, 64, 1024, 8, 1, 128, 16), (3, 5, 320, 4, 4, 128, 8), (2, 24, 48, 16, 1, 64, 24),
    (1, 2, 4096, 2, 2, 64, 32), (2, 48, 528, 28, 4, 256, 16), (2, 3, 33, 5, 1, 40, 3)])
def test_attention_over_pages_shared_by_a_group(dtype, groups, n, shared, heads, kv_heads, dim, page):
    """After an expansion; also with the shared count below the pages in common, of zero, and on rows
    that end before it."""
    tails = [(7 * i) % 90 + 1 for i in range(groups * n)]
    c = shared_cache(groups, n, shared, tails, kv_heads, dim, page, dtype, seed=20)
    q = queries(groups * n, heads, dim, dtype, sharp=2.0)
    kn, vn = (torch.randn((groups * n, kv_heads, dim), generator=gen(s), device="cuda").to(DT[dtype]) for s in (1, 2))
    for count in (shared, shared // 2 + 1, 0):
        sh = torch.full((groups,), count, device="cuda", dtype=torch.int32)
        out, lse = run_attention(c, q, dtype, group=n, shared=sh)
        check_attention(c, q, out, lse, dim ** -0.5, dtype)
    sh = torch.full((groups,), shared, device="cuda", dtype=torch.int32)
    out, lse = run_attention(c, q, dtype, group=n, shared=sh, new=(kn, vn))
    check_attention(c, q, out, lse, dim ** -0.5, dtype)
    # rows cut back to inside the shared tokens, to one token, to nothing - the first of a group among them
    c.len[1] = 1
    c.len[n - 1] = max(shared // 3, 1)
    c.len[(groups - 1) * n] = 0
    sh[0] = 10 ** 6                                            # more than any row has
    out, lse = run_attention(c, q, dtype, group=n, shared=sh)
    check_attention(c, q, out, lse, dim ** -0.5, dtype)


def test_attention_bad_indices_are_reported_not_followed():
    c = Cache([40, 40, 40], 2, 64, 16, "bf16", seed=30)
    q = queries(3, 4, 64, "bf16")
    good, _ = run_attention(c, q, "bf16")
    for bad in (-1, c.n_pages, 2 ** 31 - 1, -2 ** 31):
        c.table[1, 1] = bad
        st = status_word()
        out = torch.empty_like(q)
        ws = torch.zeros(B.kv_attend_workspace_bytes(c.kv, 4), device="cuda", dtype=torch.uint8)
        B.kv_attend(c.kv, 0, q, out, ws, status=st)
        with pytest.raises(B.PgError) as e:
            B.kv_status(st)
        assert e.value.code == B.EINDEX
        assert torch.equal(out[[0, 2]], good[[0, 2]])
    c.table[1, 1] = c.rows[1][1]
    for n in (-5, 3 * 16 + 1, 2 ** 31 - 1):
        c.len[2] = n
        c.table[2] = torch.tensor(c.rows[2][:3], device="cuda", dtype=torch.int32)
        st = status_word()
        ws = torch.zeros(B.kv_attend_workspace_bytes(c.kv, 4), device="cuda", dtype=torch.uint8)
        out = torch.empty_like(q)
        B.kv_attend(c.kv, 0, q, out, ws, status=st)
        with pytest.raises(B.PgError) as e:
            B.kv_status(st)
        assert e.value.code == B.EINDEX and torch.equal(out[:2], good[:2])


def test_attention_offsets_past_32_bits():
    """Pools of more than 2^32 elements: pages 2^21 elements apart, k and v interleaved, two layers."""
    stride, n_pages = 1 << 21, 2100
    flat = torch.zeros(n_pages * stride, device="cuda", dtype=torch.bfloat16)
    size = (2, n_pages, 2, 16, 64)
    st = (1 << 20, stride, 16 * 64, 64, 1)
    k = flat.as_strided(size, st)
    v = flat.as_strided(size, st, 1 << 12)
    c = Cache([16 * 100, 500, 20000], 2, 64, 16, "bf16", layers=2, seed=31, spare=n_pages - (100 + 32 + 1250), k=k, v=v)
    q = queries(3, 8, 64, "bf16")
    out, lse = run_attention(c, q, "bf16", layer=1)
    check_attention(c, q, out, lse, 0.125, "bf16", layer=1)
    src = torch.tensor([1, 1, 1, 2, 2], device="cuda", dtype=torch.int32)
    check_fork(c, src)


def test_attention_on_another_stream_and_in_a_graph():
    c = Cache([3000, 10, 500], 2, 128, 16, "bf16", seed=33)
    q = queries(3, 8, 128, "bf16")
    good, good_lse = run_attention(c, q, "bf16")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out, lse = run_attention(c, q, "bf16")
    torch.cuda.synchronize()
    assert torch.equal(out, good) and torch.equal(lse, good_lse)
    out2 = torch.empty_like(q)
    ws = torch.zeros(B.kv_attend_workspace_bytes(c.kv, 8), device="cuda", dtype=torch.uint8)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.kv_attend(c.kv, 0, q, out2, ws)
    for _ in range(3):
        out2.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out2, good)
    c.len[0] = 77                                              # lengths are read at replay
    graph.replay()
    torch.cuda.synchronize()
    check_attention(c, q, out2, None, 128 ** -0.5, "bf16")


def test_attention_workspace_is_reusable_across_shapes():
    """One workspace, calls of different lengths in a row: every call leaves its counters at zero."""
    c = Cache([9000, 1200, 7, 0, 64], 2, 64, 16, "f16", seed=34)
    q = queries(5, 16, 64, "f16")
    ws = torch.zeros(B.kv_attend_workspace_bytes(c.kv, 16), device="cuda", dtype=torch.uint8)
    for lens in ([9000, 1200, 7, 0, 64], [1, 1, 1, 1, 1], [5000, 0, 0, 0, 64], [9000, 1200, 7, 0, 64]):
        lens[3] = 0
        c.len.copy_(torch.tensor(lens, dtype=torch.int32))
        out, lse = run_attention(c, q, "f16", ws=ws)
        check_attention(c, q, out, lse, 0.125, "f16")


def test_attention_refusals():
    c = Cache([40, 40], 2, 64, 16, "bf16", seed=35)
    q = queries(2, 4, 64, "bf16")
    out = torch.empty_like(q)
    ws = torch.zeros(B.kv_attend_workspace_bytes(c.kv, 4), device="cuda", dtype=torch.uint8)

    def refused(code=B.EINVAL, kv=c.kv, **kw):
        a = dict(layer=0, q=q, out=out, workspace=ws)
        more = {k: kw.pop(k) for k in list(kw) if k not in a}
        a.update(kw)
        with pytest.raises(B.PgError) as e:
            B.kv_attend(kv, a["layer"], a["q"], a["out"], a["workspace"], **more)
        assert e.value.code == code

    refused(layer=1)
    refused(layer=-1)
    refused(scale=math.nan)
    refused(group=3)
    refused(group=0)
    refused(q=queries(2, 3, 64, "bf16"), out=queries(2, 3, 64, "bf16"))      # 3 query heads over 2
    refused(workspace=ws[: ws.numel() - 16])
    refused(workspace=torch.zeros(ws.numel() + 16, device="cuda", dtype=torch.uint8)[8:])
    flat = torch.zeros(2 * 2 * 64 + 8, device="cuda", dtype=torch.bfloat16)
    new = flat[1: 1 + 256].view(2, 2, 64)                                     # not on 16 bytes
    refused(k_new=new, v_new=new)
    for bad in (dict(q=q.float()), dict(out=out[:1]), dict(q=q[:, :, :32]), dict(lse=torch.zeros(3, device="cuda")),
                dict(k_new=torch.zeros(2, 2, 64, device="cuda", dtype=torch.bfloat16)), dict(q=q.transpose(0, 1).contiguous().transpose(0, 1)),
                dict(q=q[:1].expand(2, 4, 64)), dict(shared=torch.zeros(2, device="cuda", dtype=torch.int64))):
        a = dict(q=q, out=out)
        more = {k: bad.pop(k) for k in list(bad) if k not in a}
        a.update(bad)
        with pytest.raises((ValueError, AttributeError)):
            B.kv_attend(c.kv, 0, a["q"], a["out"], ws, **more)
    for field, value in (("head_dim", 60), ("head_dim", 264), ("page_size", 0), ("n_pages", 0), ("dtype", 3), ("page_stride", 8),
                         ("page_stride", 2052), ("k", None), ("table", None), ("max_pages", 0), ("n_kv_heads", 0), ("n_rows", -1)):
        kv = B.make_kv(c.k, c.v, c.table, c.len)
        setattr(kv, field, value)
        assert B.lib().pg_kv_attend_workspace_bytes(kv._ref, 4, 1) == 0
        rc = B.lib().pg_kv_attend(kv._ref, 0, 4, q.data_ptr(), 0, None, None, 0, 0.1, 1, None, out.data_ptr(), 0, None, ws.data_ptr(),
                                  ws.numel(), None, None)
        assert rc == B.EINVAL, field
    with pytest.raises(ValueError):
        B.make_kv(c.k, c.v.float(), c.table, c.len)
    with pytest.raises(ValueError):
        B.make_kv(c.k.transpose(2, 3), c.v.transpose(2, 3), c.table, c.len)
    with pytest.raises(ValueError):
        B.make_kv(c.k, c.v, c.table.long(), c.len)


# ------------------------------------------------------------------------------ pages

def pools_after(c, copies):
    k, v = c.k.clone(), c.v.clone()
    for a, b in copies:
        k[:, b], v[:, b] = c.k[:, a], c.v[:, a]
    return k, v


def same_bits(a, b):
    kind = torch.int32 if a.dtype == torch.float32 else torch.int16
    return torch.equal(a.contiguous().view(kind), b.contiguous().view(kind))


def clean_rows(c):
    return [t[: ref.ceil(n, c.page)] + [-1] * (c.width - ref.ceil(n, c.page)) for t, n in zip(c.rows, c.lens)]


def check_fork(c, src, in_place=False, short=False):
    n = src.numel()
    width = c.table.shape[1]
    table, lens, refs, copies, ran_out = ref.fork(c.rows, c.lens, c.refs.tolist(), src.tolist(), c.page, c.n_pages)
    assert ran_out == short
    strided = not c.k.is_contiguous()
    want_k, want_v = (None, None) if strided else pools_after(c, copies)
    t_out = torch.full((n, width), 77, device="cuda", dtype=torch.int32)
    l_out = torch.full((n,), 77, device="cuda", dtype=torch.int32)
    r_out = c.refs if in_place else torch.full_like(c.refs, 77)
    ws = torch.zeros(B.kv_fork_workspace_bytes(c.kv, n), device="cuda", dtype=torch.uint8)
    st = status_word()
    B.kv_fork(c.kv, src, t_out, l_out, c.refs, r_out, ws, status=st)
    if short:
        with pytest.raises(B.PgError) as e:
            B.kv_status(st)
        assert e.value.code == B.ENOPAGES
    else:
        B.kv_status(st)
    assert t_out.tolist() == table and l_out.tolist() == lens and r_out.tolist() == refs
    if strided:
        for a, b in copies:
            assert same_bits(c.k[:, a], c.k[:, b]) and same_bits(c.v[:, a], c.v[:, b])
    else:
        assert same_bits(c.k, want_k) and same_bits(c.v, want_v)
    return t_out, l_out, r_out


@pytest.mark.parametrize("dtype,heads,dim,page,layers", [("bf16", 2, 64, 16, 1), ("f32", 1, 8, 3, 3), ("f16", 8, 128, 32, 2),
                                                         ("bf16", 1, 24, 1, 2), ("f32", 4, 256, 16, 1)])
@pytest.mark.parametrize("src", [[0, 0, 0, 1, 1, 1, 2, 2, 2], [3, 1], [], [5, 4, 3, 2, 1, 0], [2, 0, 2, -1, 5, 2, 0, -1, 4],
                                 [4] * 40, [0, 1, 2, 3, 4, 5], [-1, -1]])
def test_fork_against_plain_form(dtype, heads, dim, page, layers, src):
    c = Cache([2 * page + 1 if page > 1 else 2, page, 0, 1, 5 * page - 1 if page > 1 else 4, 40], heads, dim, page, dtype,
              layers=layers, spare=45, seed=41)
    check_fork(c, torch.tensor(src, device="cuda", dtype=torch.int32))
    check_fork(c, torch.tensor(src, device="cuda", dtype=torch.int32), in_place=True)


def test_fork_chain_expand_prune_release():
    """Expansion, growth, a prune through pg_prune_ovf's src_rows, another expansion, release: counts
    return to zero, every row's tokens stay what they were."""
    G, N, K, page = 3, 8, 4, 8
    c = Cache([20, 8, 33], 2, 64, page, "bf16", spare=120, seed=42, width=12)
    src = torch.arange(G, device="cuda", dtype=torch.int32).repeat_interleave(N)
    t, l, r = check_fork(c, src)
    c.table, c.len, c.refs, c.rows, c.lens = t, l, r, t.tolist(), l.tolist()
    c.kv = B.make_kv(c.k, c.v, c.table, c.len)
    h = B.rollout_init(B.make_config(G, N, 4, 4, [(1, K)], 0, B.VEL_F32))
    try:
        x = torch.zeros(G * N, 4, device="cuda")
        lp = torch.empty(G * N, device="cuda")
        B.step(h, 0, (1.0, 0.0, 1.0), x, x.clone(), None, x, lp)
        keep, rows = (torch.empty(G * K, device="cuda", dtype=torch.int32) for _ in range(2))
        B.prune_ovf(h, 0, torch.randn(G * N, generator=gen(1), device="cuda"), keep, rows)
        t, l, r = check_fork(c, rows)
    finally:
        torch.cuda.synchronize()
        B.rollout_destroy(h)
    assert int((r > 0).sum()) < int((c.refs > 0).sum())
    c.table, c.len, c.refs, c.rows, c.lens = t, l, r, t.tolist(), l.tolist()
    c.kv = B.make_kv(c.k, c.v, c.table, c.len)
    ws = torch.zeros(B.kv_fork_workspace_bytes(c.kv, 0), device="cuda", dtype=torch.uint8)
    B.kv_fork(c.kv, None, None, None, c.refs, c.refs, ws)
    torch.cuda.synchronize()
    assert (c.refs == 0).all()


def test_fork_out_of_pages_and_bad_rows():
    c = Cache([20, 20], 1, 8, 16, "f32", spare=2, seed=43)
    check_fork(c, torch.tensor([0, 0, 1, 0, 1, 1], device="cuda", dtype=torch.int32), short=True)
    src = torch.tensor([0, 2, -2, 2 ** 31 - 1], device="cuda", dtype=torch.int32)
    t, l = torch.empty((4, c.width), device="cuda", dtype=torch.int32), torch.empty(4, device="cuda", dtype=torch.int32)
    st, out = status_word(), torch.empty_like(c.refs)
    ws = torch.zeros(B.kv_fork_workspace_bytes(c.kv, 4), device="cuda", dtype=torch.uint8)
    B.kv_fork(c.kv, src, t, l, c.refs, out, ws, status=st)
    with pytest.raises(B.PgError) as e:
        B.kv_status(st)
    assert e.value.code == B.EINDEX
    assert l.tolist() == [20, 0, 0, 0] and (t[1:] == -1).all()


@pytest.mark.parametrize("rows,fan", [(64, 64), (3, 700), (2000, 1)])
def test_fork_many_rows(rows, fan):
    lens = [(13 * i) % 40 for i in range(rows)]
    c = Cache(lens, 1, 8, 4, "bf16", spare=rows * fan + 5, seed=44)
    src = torch.arange(rows, device="cuda", dtype=torch.int32).repeat_interleave(fan)
    check_fork(c, src)
    check_fork(c, src.flip(0).contiguous())


@pytest.mark.parametrize("dtype,heads,dim,page,layers", [("bf16", 2, 64, 16, 2), ("f32", 1, 8, 3, 1), ("f16", 8, 256, 16, 1)])
@pytest.mark.parametrize("lens,spare", [([100, 0, 37, 260], 60), ([1], 0), ([5, 5, 5], 1500), ([0, 0], 4), ([3000], 3000)])
def test_pack_against_plain_form(dtype, heads, dim, page, layers, lens, spare):
    for in_place in (False, True):
        c = Cache(lens, heads, dim, page, dtype, layers=layers, spare=spare + (sum(lens) == 0), seed=50)
        table, refs, moves, to = ref.pack(clean_rows(c), c.lens, c.refs.tolist(), page)
        want_k, want_v = pools_after(c, moves)
        t_out = c.table if in_place else torch.empty_like(c.table)
        r_out = c.refs if in_place else torch.empty_like(c.refs)
        page_map = torch.empty_like(c.refs)
        ws = torch.zeros(B.kv_pack_workspace_bytes(c.kv), device="cuda", dtype=torch.uint8)
        st = status_word()
        B.kv_pack(c.kv, c.refs, r_out, t_out, ws, page_map=page_map, status=st)
        B.kv_status(st)
        assert t_out.tolist() == table and r_out.tolist() == refs and page_map.tolist() == to
        assert same_bits(c.k, want_k) and same_bits(c.v, want_v)


@pytest.mark.parametrize("n_new", [1, 0, 7, [3, 0, 40, 1, 16, 100], [0] * 6, [1000, 1, 1, 1, 1, 1], [5, 5, 190, 5, 5, 5]])
@pytest.mark.parametrize("page", [1, 5, 16])
@pytest.mark.parametrize("spare", [0, 3, 400])
def test_extend_against_plain_form(n_new, page, spare):
    lens = [16, 0, 3, 31, 32, 1]
    c = Cache(lens, 1, 8, page, "f32", spare=spare + 1, seed=60, width=200)
    add = [n_new] * 6 if isinstance(n_new, int) else n_new
    table, length, refs, short = ref.extend(clean_rows(c), c.lens, c.refs.tolist(), add, page)
    before = c.table.clone()
    l_out, r_out, st = torch.empty_like(c.len), torch.empty_like(c.refs), status_word()
    arg = n_new if isinstance(n_new, int) else torch.tensor(n_new, device="cuda", dtype=torch.int32)
    B.kv_extend(c.kv, arg, l_out, c.refs, r_out, status=st)
    assert (int(st) != 0) == short and (not short or int(st) == 8)
    assert l_out.tolist() == length and r_out.tolist() == refs
    got = c.table.tolist()
    for r in range(6):
        used = ref.ceil(length[r], page)
        assert got[r][:used] == table[r][:used]
    # in place
    c.table.copy_(before)
    B.kv_extend(c.kv, arg, c.len, c.refs, c.refs)
    torch.cuda.synchronize()
    assert c.len.tolist() == length and c.refs.tolist() == refs


def test_extend_many_rows():
    lens = [(7 * i) % 50 for i in range(2500)]
    c = Cache(lens, 1, 8, 16, "f32", spare=2600, seed=61, width=5)
    table, length, refs, short = ref.extend(clean_rows(c), c.lens, c.refs.tolist(), [9] * 2500, 16)
    assert not short
    B.kv_extend(c.kv, 9, c.len, c.refs, c.refs)
    torch.cuda.synchronize()
    assert c.len.tolist() == length and c.refs.tolist() == refs
    got = c.table.tolist()
    assert all(got[r][: ref.ceil(n, 16)] == table[r][: ref.ceil(n, 16)] for r, n in enumerate(length))
    bad = torch.full((2500,), -1, device="cuda", dtype=torch.int32)
    st = status_word()
    B.kv_extend(c.kv, bad, c.len, c.refs, c.refs, status=st)
    assert int(st) == 4 and c.len.tolist() == length


@pytest.mark.parametrize("dtype,heads,dim,page", [("bf16", 2, 64, 16), ("f32", 3, 40, 5), ("f16", 1, 8, 1), ("bf16", 8, 256, 24)])
def test_append_against_plain_form(dtype, heads, dim, page):
    new = [3, 0, 40, 1, 0, 17]
    lens = [16, 5, 3, 31, 0, 32]
    grown = [a + b for a, b in zip(lens, new)]
    c = Cache(grown, heads, dim, page, dtype, layers=3, seed=70)
    n = sum(new)
    fused = torch.randn((n, 3 * heads, dim), generator=gen(71), device="cuda").to(DT[dtype])
    kn, vn = fused[:, heads: 2 * heads], fused[:, 2 * heads:]
    want_k, want_v = c.k.clone(), c.v.clone()
    t = 0
    for r in range(6):
        for j in range(new[r]):
            pos = lens[r] + j
            want_k[1, c.rows[r][pos // page], :, pos % page] = kn[t]
            want_v[1, c.rows[r][pos // page], :, pos % page] = vn[t]
            t += 1
    start = torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), device="cuda", dtype=torch.int32)
    st = status_word()
    B.kv_append(c.kv, 1, kn, vn, start, status=st)
    B.kv_status(st)
    assert same_bits(c.k, want_k) and same_bits(c.v, want_v)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_append_one_token_per_row(dtype):
    lens = [16, 5, 3, 31, 1, 32] * 50
    c = Cache(lens, 4, 64, 16, dtype, seed=72)
    kn, vn = (torch.randn((300, 4, 64), generator=gen(s), device="cuda").to(DT[dtype]) for s in (1, 2))
    want_k, want_v = c.k.clone(), c.v.clone()
    for r, n in enumerate(lens):
        want_k[0, c.rows[r][(n - 1) // 16], :, (n - 1) % 16] = kn[r]
        want_v[0, c.rows[r][(n - 1) // 16], :, (n - 1) % 16] = vn[r]
    B.kv_append(c.kv, 0, kn, vn)
    torch.cuda.synchronize()
    assert same_bits(c.k, want_k) and same_bits(c.v, want_v)
    c.len[7] = 0                                               # a row without room for its token
    c.table[9, 0] = 10 ** 6
    st = status_word()
    B.kv_append(c.kv, 0, kn, vn, status=st)
    with pytest.raises(B.PgError) as e:
        B.kv_status(st)
    assert e.value.code == B.EINDEX


def test_page_call_refusals():
    c = Cache([20, 20], 1, 8, 16, "f32", seed=80)
    i32 = dict(device="cuda", dtype=torch.int32)
    src = torch.zeros(3, **i32)
    t, l, r = torch.empty((3, c.width), **i32), torch.empty(3, **i32), torch.empty_like(c.refs)
    ws = torch.zeros(B.kv_fork_workspace_bytes(c.kv, 3), device="cuda", dtype=torch.uint8)
    for args in ((src, c.table.view(-1)[: 2 * c.width], l, c.refs, r, ws), (src, t, l, c.refs, r, ws[:-16]),):
        with pytest.raises((B.PgError, ValueError)):
            B.kv_fork(c.kv, *args)
    two = torch.zeros(2, **i32)
    with pytest.raises(B.PgError) as e:
        B.kv_fork(c.kv, two, c.table, torch.empty(2, **i32), c.refs, r, ws)      # onto its own table
    assert e.value.code == B.EINVAL
    with pytest.raises(B.PgError):
        B.kv_fork(c.kv, two, torch.empty_like(c.table), c.len, c.refs, r, ws)
    with pytest.raises(ValueError):
        B.kv_fork(c.kv, src.long(), t, l, c.refs, r, ws)
    with pytest.raises(B.PgError):
        B.kv_extend(c.kv, -1, c.len, c.refs, c.refs)
    with pytest.raises(ValueError):
        B.kv_extend(c.kv, torch.zeros(3, **i32), c.len, c.refs, c.refs)
    new = torch.zeros(2, 1, 8, device="cuda")
    with pytest.raises(B.PgError):
        B.kv_append(c.kv, 2, new, new)
    with pytest.raises(B.PgError):
        B.kv_append(c.kv, 0, new[:1], new[:1])                                  # one token for two rows
    with pytest.raises(ValueError):
        B.kv_append(c.kv, 0, new.half(), new.half())
    with pytest.raises(B.PgError):
        B.kv_pack(c.kv, c.refs, c.refs, c.table, torch.zeros(16, device="cuda", dtype=torch.uint8))
    assert B.lib().pg_kv_status(None, None) == B.EINVAL
    kv = B.make_kv(c.k, c.v, c.table, c.len)
    kv.max_pages = 2 ** 30
    assert B.lib().pg_kv_pack_workspace_bytes(kv._ref) == 0


# ------------------------------------------------------------------------------ logits

def logits_case(R, V, H, n_bias, dtype, seed):
    g = gen(seed)
    c = dict(x=(torch.randn((R, V), generator=g, device="cuda") * 3).to(DT[dtype]))
    c["tokens"] = torch.randint(-2, V + 2, (R, H), generator=g, device="cuda", dtype=torch.int32)
    c["tokens"][:, ::3] = V // 2                                 # one token over and over
    c["n_tokens"] = torch.randint(0, H + 1, (R,), generator=g, device="cuda", dtype=torch.int32)
    c["n_prompt"] = torch.randint(0, H + 1, (R,), generator=g, device="cuda", dtype=torch.int32)
    c["rho"], c["pi"], c["phi"] = 1 + torch.rand(R, generator=g, device="cuda"), torch.randn(R, generator=g, device="cuda"), \
        torch.randn(R, generator=g, device="cuda")
    c["tau"] = 0.3 + torch.rand(R, generator=g, device="cuda")
    c["bias_ids"] = torch.randint(-1, V + 1, (R, n_bias), generator=g, device="cuda", dtype=torch.int32)
    c["bias_values"] = torch.randn((R, n_bias), generator=g, device="cuda") * 5
    c["mask"] = torch.randint(-2 ** 31, 2 ** 31, (R, ref.ceil(V, 32)), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    if R > 2:
        c["mask"][1] = 0
        c["mask"][2] = -1
    return c


RULES = ("tokens", "n_tokens", "n_prompt", "rho", "pi", "phi", "tau", "bias_ids", "bias_values", "mask")


def make_rules(c):
    return B.make_logits_rules(tokens=c.get("tokens"), n_tokens=c.get("n_tokens"), n_prompt=c.get("n_prompt"),
                               repetition=c.get("rho"), presence=c.get("pi"), frequency=c.get("phi"), temperature=c.get("tau"),
                               bias_ids=c.get("bias_ids"), bias_values=c.get("bias_values"), mask=c.get("mask"))


def check_logits(c, got, out_dtype):
    """Seven roundings in fp32 of terms no larger than the sum of their sizes, then one of the result."""
    want = ref.logits(c["x"], *(c.get(k) for k in RULES))
    size = c["x"].double().abs()
    big = torch.ones(got.shape[0], device="cuda", dtype=torch.float64)
    H = 0 if c.get("tokens") is None else c["tokens"].shape[1]
    if c.get("rho") is not None:
        size = size * torch.maximum(c["rho"].double(), 1 / c["rho"].double())[:, None]
    for key, f in (("phi", H), ("pi", 1)):
        if c.get(key) is not None:
            big = big + c[key].double().abs() * f
    if c.get("bias_values") is not None and c["bias_values"].numel():
        big = big + c["bias_values"].double().abs().amax(1)
    size = size + big[:, None]
    if c.get("tau") is not None:
        size = size / c["tau"].double()[:, None]
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got.double()), fine)
    assert torch.equal(got.double()[~fine], want[~fine])
    off = (got.double() - want).abs()[fine]
    lim = (7 * 2.0 ** -24 * size + UNIT[out_dtype] * want.abs() + (2.0 ** -24 if out_dtype == "f16" else 0))[fine]
    assert (off <= lim).all(), (off / lim).max().item()


@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("R,V,H,n_bias", [(1, 1, 1, 1), (3, 31, 5, 2), (4, 8192, 100, 7), (5, 8193, 2000, 40), (3, 50001, 3000, 2046),
                                          (2, 131072, 20000, 300)])
def test_logits_rules_together(dtype, out, R, V, H, n_bias):
    c = logits_case(R, V, H, n_bias, dtype, R + V)
    got = torch.full((R, V), float("nan"), device="cuda", dtype=DT[out])
    B.logits_process(c["x"], got, make_rules(c))
    torch.cuda.synchronize()
    check_logits(c, got, out)


@pytest.mark.parametrize("keep", [(), ("mask",), ("tau",), ("bias_ids", "bias_values"), ("tokens", "rho"), ("tokens", "n_tokens", "pi"),
                                  ("tokens", "n_prompt", "phi"), ("tokens",), ("tokens", "n_tokens", "n_prompt", "rho", "mask"),
                                  ("rho", "pi", "phi")])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logits_rules_one_by_one(keep, dtype):
    c = logits_case(3, 10007, 333, 9, dtype, 7)
    c = {k: v for k, v in c.items() if k == "x" or k in keep}
    got = torch.empty_like(c["x"])
    B.logits_process(c["x"], got, make_rules(c))
    torch.cuda.synchronize()
    check_logits(c, got, dtype)
    if not keep:
        assert torch.equal(got, c["x"])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_logits_strides_and_in_place(dtype, shift):
    """Rows inside a wider tensor, starting at any element; in place; one row of bits for all rows."""
    c = logits_case(4, 9001, 64, 5, dtype, 9)
    c["mask"] = c["mask"][:1].contiguous()
    wide = torch.full((4, 9001 + 7), 3.0, device="cuda", dtype=DT[dtype])
    x = wide[:, shift: shift + 9001]
    x.copy_(c["x"])
    hist = torch.zeros((4, 100), device="cuda", dtype=torch.int32)
    hist[:, 11: 75] = c["tokens"]
    rules = make_rules(dict(c, tokens=hist[:, 11: 75]))
    out = torch.full((4, 9001 + 2), 5.0, device="cuda", dtype=DT[dtype])
    B.logits_process(x, out[:, 1: 9002], rules)
    torch.cuda.synchronize()
    check_logits(c, out[:, 1: 9002], dtype)
    assert (out[:, 0] == 5.0).all() and (out[:, 9002] == 5.0).all()
    B.logits_process(x, x, rules)
    torch.cuda.synchronize()
    assert torch.equal(x, out[:, 1: 9002])
    rest = torch.cat([wide[:, :shift], wide[:, shift + 9001:]], 1)
    assert (rest == 3.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_logits_extreme_values(dtype):
    """Lowest values, infinities and NaN: where the mask forbids they become -inf, elsewhere they go
    through the formula."""
    lowest = torch.finfo(DT[dtype]).min
    x = torch.tensor([[lowest, -math.inf, math.inf, math.nan, 0.0, -0.0, -lowest, 1.0] * 2], device="cuda", dtype=DT[dtype])
    mask = torch.tensor([[0xFF]], device="cuda", dtype=torch.int32)
    out = torch.empty_like(x, dtype=torch.float32)
    B.logits_process(x, out, B.make_logits_rules(mask=mask))
    torch.cuda.synchronize()
    assert (out[0, 8:] == -math.inf).all()
    assert torch.equal(out[0, :8].nan_to_num(nan=123.0, posinf=3e38, neginf=-3e38),
                       x[0, :8].float().nan_to_num(nan=123.0, posinf=3e38, neginf=-3e38))
    tokens = torch.arange(8, device="cuda", dtype=torch.int32)[None]
    rho, tau = torch.tensor([1.25], device="cuda"), torch.tensor([0.5], device="cuda")
    B.logits_process(x, out, B.make_logits_rules(tokens=tokens, repetition=rho, temperature=tau, mask=mask))
    torch.cuda.synchronize()
    y = x.float()
    want = torch.where(y > 0, y / 1.25, y * 1.25) / 0.5
    assert torch.equal(out[0, :8].nan_to_num(nan=123.0, posinf=3e38, neginf=-3e38),
                       want[0, :8].nan_to_num(nan=123.0, posinf=3e38, neginf=-3e38))


def test_logits_repeated_bias_ids_take_the_last():
    x = torch.zeros((1, 100), device="cuda")
    ids = torch.tensor([[5, 7, 5, -1, 100, 5, 7]], device="cuda", dtype=torch.int32)
    val = torch.tensor([[1.0, 2.0, 3.0, 9.0, 9.0, 4.0, 6.0]], device="cuda")
    for _ in range(5):
        out = torch.empty_like(x)
        B.logits_process(x, out, B.make_logits_rules(bias_ids=ids, bias_values=val))
        torch.cuda.synchronize()
        want = torch.zeros(100)
        want[5], want[7] = 4.0, 6.0
        assert torch.equal(out[0].cpu(), want)


def test_logits_refusals():
    x = torch.zeros((2, 100), device="cuda")
    out = torch.empty_like(x)
    none = B.make_logits_rules()
    for bad in (dict(logits=x.double()), dict(out=out[:, :50]), dict(logits=x.t().contiguous().t()), dict(logits=x[:1].expand(2, 100))):
        a = dict(logits=x, out=out, rules=none)
        a.update(bad)
        with pytest.raises(ValueError):
            B.logits_process(**a)
    with pytest.raises(B.PgError):
        B.logits_process(x, out, _bad_rules())
    with pytest.raises(ValueError):
        B.logits_process(x, out, B.make_logits_rules(temperature=torch.ones(3, device="cuda")))
    with pytest.raises(ValueError):
        B.logits_process(x, out, B.make_logits_rules(mask=torch.zeros((2, 3), device="cuda", dtype=torch.int32)))
    with pytest.raises(ValueError):
        B.make_logits_rules(tokens=torch.zeros((2, 5), device="cuda"))
    with pytest.raises(ValueError):
        B.make_logits_rules(bias_ids=torch.zeros((2, 5), device="cuda", dtype=torch.int32))
    L = B.lib()
    args = (x.data_ptr(), 0, B.F32, out.data_ptr(), 0, none._ref, None)
    assert L.pg_logits_process(2, 0, B.F32, *args) == B.EINVAL
    assert L.pg_logits_process(-1, 100, B.F32, *args) == B.EINVAL
    assert L.pg_logits_process(2, 100, 5, *args) == B.EINVAL
    assert L.pg_logits_process(2, 100, B.F32, None, *args[1:]) == B.EINVAL
    assert L.pg_logits_process(2, 100, B.F32, x.data_ptr(), 99, *args[2:]) == B.EINVAL
    assert L.pg_logits_process(2, 100, B.F32, x.data_ptr() + 2, *args[1:]) == B.EINVAL
    assert L.pg_logits_process(2, 100, B.F32, x.data_ptr(), 0, B.BF16, x.data_ptr(), 0, none._ref, None) == B.EINVAL
    assert L.pg_logits_process(0, 100, B.F32, *args) == B.OK


def _bad_rules():
    r = B.make_logits_rules(tokens=torch.zeros((2, 5), device="cuda", dtype=torch.int32))
    r.max_tokens = B.LOGITS_MAX_TOKENS + 1
    return r
