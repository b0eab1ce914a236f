"""The token-rollout calls where something has gone wrong before them: waits that ran out, rows that found no
page, workspaces that other calls have used, sizes near the ends of their types."""
import math

import pytest
import torch

from paper_2512_15347_b200 import binding as B
from tests import kv_reference as ref
from tests import test_gpu_kv as T

pytestmark = pytest.mark.gpu


def lost(*kinds):
    """Waits of these kinds run out at once inside the block."""
    class Lost:
        def __enter__(self):
            B.selftest_token_waits(*kinds)

        def __exit__(self, *a):
            torch.cuda.synchronize()
            B.selftest_token_waits()
    return Lost()


def attend_status(c, q, ws, **kw):
    """The status code of one call, whose outputs are not looked at."""
    st, out = T.status_word(), torch.empty_like(q)
    B.kv_attend(c.kv, 0, q, out, ws, lse=torch.empty(q.shape[:2], device="cuda"), status=st, **kw)
    try:
        B.kv_status(st)
    except B.PgError as e:
        return e.code
    return B.OK


# ------------------------------------------------------------------------------ waits that run out

def group_case(dim, dtype, seed=0):
    """Two groups of 48 rows, 1024 tokens in common: several tiles a CTA, two products of queries at once up to dim 128."""
    c = T.shared_cache(2, 48, 1024, [1 + i % 37 for i in range(96)], 2, dim, 16, dtype, seed=seed)
    q = T.queries(96, 8, dim, dtype, sharp=2.0)
    sh = torch.full((2,), 1024, device="cuda", dtype=torch.int32)
    return c, q, dict(group=48, shared=sh)


@pytest.mark.parametrize("kind", ["tiles", "stages", "queries", "scores", "weights", "products"])
@pytest.mark.parametrize("dim,dtype", [(64, "f16"), (128, "bf16"), (256, "bf16")])
def test_a_wait_of_the_shared_part_that_runs_out_is_reported(kind, dim, dtype):
    c, q, kw = group_case(dim, dtype)
    ws = torch.zeros(B.kv_attend_workspace_bytes(c.kv, 8, 48), device="cuda", dtype=torch.uint8)
    with lost(kind):
        assert attend_status(c, q, ws, **kw) == B.ETIMEOUT
    out, lse = T.run_attention(c, q, dtype, ws=ws, **kw)
    T.check_attention(c, q, out, lse, dim ** -0.5, dtype)


@pytest.mark.parametrize("dim,dtype", [(64, "f16"), (64, "f32"), (128, "bf16"), (256, "bf16"), (256, "f32")])
@pytest.mark.parametrize("lens", [[5000, 300, 0, 77], [17], [40] * 200])
def test_a_wait_for_a_rows_own_chunks_that_runs_out_is_reported(dim, dtype, lens):
    """Bulk copies that are under way when their warp gives up: in long pieces that are dumped into the ring and joined, and in
    short ones; the calls after it find their counters at zero."""
    c = T.Cache(lens, 2, dim, 16, dtype, seed=3)
    q = T.queries(len(lens), 8, dim, dtype)
    ws = torch.zeros(B.kv_attend_workspace_bytes(c.kv, 8, 1), device="cuda", dtype=torch.uint8)
    with lost("chunks"):
        for _ in range(3):
            assert attend_status(c, q, ws) == B.ETIMEOUT
    out, lse = T.run_attention(c, q, dtype, ws=ws)
    T.check_attention(c, q, out, lse, dim ** -0.5, dtype)


@pytest.mark.parametrize("dim,dtype", [(64, "f16"), (128, "bf16"), (256, "bf16")])
@pytest.mark.parametrize("fill", [0x7F, 0x3F, 0xBF, 0xFF])
def test_shared_part_that_gave_up_over_a_used_workspace(dim, dtype, fill):
    """Behind its counters a workspace holds anything (another shape's partial results): the units that the shared part has
    not come to are followed through none of it.  Many units a CTA, so that most are not come to."""
    c = T.shared_cache(40, 3, 64, [1 + i % 20 for i in range(120)], 8, dim, 16, dtype)
    q = T.queries(120, 8, dim, dtype)
    kw = dict(group=3, shared=torch.full((40,), 64, device="cuda", dtype=torch.int32))
    ws = torch.zeros(B.kv_attend_workspace_bytes(c.kv, 8, 3), device="cuda", dtype=torch.uint8)
    for kind in ("tiles", "weights"):
        ws[4096:] = fill
        with lost(kind):
            assert attend_status(c, q, ws, **kw) == B.ETIMEOUT
    out, lse = T.run_attention(c, q, dtype, ws=ws, **kw)
    T.check_attention(c, q, out, lse, dim ** -0.5, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_one_attention_workspace_over_group_sizes(dtype):
    """The counters' place depends on nothing; what lies behind them moves with the group size and is written before it is read."""
    cases = [(2, 48, 1024), (12, 2, 64), (1, 200, 128), (2, 16, 320)]
    made = []
    for groups, n, shared in cases:
        c = T.shared_cache(groups, n, shared, [1 + 5 * i % 61 for i in range(groups * n)], 2, 64, 16, dtype, seed=n)
        made.append((c, T.queries(groups * n, 8, 64, dtype), n, torch.full((groups,), shared, device="cuda", dtype=torch.int32)))
    ws = torch.zeros(max(B.kv_attend_workspace_bytes(c.kv, 8, n) for c, _, n, _ in made), device="cuda", dtype=torch.uint8)
    for c, q, n, sh in made + made[::-1]:
        out, lse = T.run_attention(c, q, dtype, group=n, shared=sh, ws=ws)
        T.check_attention(c, q, out, lse, 0.125, dtype)


def test_waits_are_named_or_refused():
    assert B.lib().pg_selftest_token_waits(1 << 31) == B.EINVAL
    with pytest.raises(ValueError):
        B.selftest_token_waits("nothing")
    B.selftest_token_waits()


@pytest.mark.parametrize("src", [[0, 1, 2], [2, 1], [1, 1, 0], [0, 2], []])
@pytest.mark.parametrize("bad", [-1, 10 ** 6, 2 ** 31 - 1])
def test_fork_reports_a_bad_page_whatever_becomes_of_its_row(src, bad):
    """Kept by one fork (its counts do not change), by several, or dropped; also in the partly filled last page."""
    for at in (0, 2):
        c = T.Cache([40, 40, 16], 1, 8, 16, "f32", spare=9, seed=45)
        c.table[1, at] = bad
        st, n = T.status_word(), len(src)
        ws = torch.zeros(B.kv_fork_workspace_bytes(c.kv, n), device="cuda", dtype=torch.uint8)
        t, l = torch.empty((n, c.width), device="cuda", dtype=torch.int32), torch.empty(n, device="cuda", dtype=torch.int32)
        B.kv_fork(c.kv, torch.tensor(src, device="cuda", dtype=torch.int32), t, l, c.refs, c.refs, ws, status=st)
        with pytest.raises(B.PgError) as e:
            B.kv_status(st)
        assert e.value.code == B.EINDEX


# ------------------------------------------------------------------------------ one buffer for all calls

def test_one_workspace_for_calls_of_every_kind():
    """Packing, forking and attention in turn over one buffer: none finds its counters at what another has left."""
    def cache(seed):
        return T.Cache([77, 5, 130, 64], 2, 64, 16, "bf16", spare=90, seed=seed)
    need = lambda c: max(B.kv_pack_workspace_bytes(c.kv), B.kv_fork_workspace_bytes(c.kv, 12), B.kv_attend_workspace_bytes(c.kv, 8, 1))
    ws = torch.zeros(need(cache(1)), device="cuda", dtype=torch.uint8)
    long = T.Cache([9000, 41], 2, 64, 16, "bf16", seed=9)                 # pieces that several CTAs share
    ql = T.queries(2, 8, 64, "bf16")
    for seed in range(1, 4):
        c = cache(seed)
        table, refs, moves, _ = ref.pack(T.clean_rows(c), c.lens, c.refs.tolist(), c.page)
        assert moves
        want_k, want_v = T.pools_after(c, moves)
        st = T.status_word()
        B.kv_pack(c.kv, c.refs, c.refs, c.table, ws, status=st)
        B.kv_status(st)
        assert c.table.tolist() == table and c.refs.tolist() == refs and T.same_bits(c.k, want_k) and T.same_bits(c.v, want_v)
        out, lse = T.run_attention(long, ql, "bf16", ws=ws)
        T.check_attention(long, ql, out, lse, 0.125, "bf16")
        c.rows = table
        src = [0, 0, 0, 1, 1, 2, 2, 3, 2]
        want_t, want_l, want_r, copies, _ = ref.fork(c.rows, c.lens, refs, src, c.page, c.n_pages)
        want_k, want_v = T.pools_after(c, copies)
        t, n = torch.empty((9, c.width), device="cuda", dtype=torch.int32), torch.empty(9, device="cuda", dtype=torch.int32)
        B.kv_fork(c.kv, torch.tensor(src, device="cuda", dtype=torch.int32), t, n, c.refs, c.refs, ws, status=st)
        B.kv_status(st)
        assert t.tolist() == want_t and n.tolist() == want_l and c.refs.tolist() == want_r
        assert T.same_bits(c.k, want_k) and T.same_bits(c.v, want_v)
        assert int(ws[:4096].sum()) == 0
        out, lse = T.run_attention(long, ql, "bf16", ws=ws)
        T.check_attention(long, ql, out, lse, 0.125, "bf16")


# ------------------------------------------------------------------------------ tensors that are not the device's

def test_host_tensors_are_refused_before_any_launch(monkeypatch):
    """A host address in a kernel is a fault: every tensor of every call is looked at."""
    c = T.Cache([20, 20], 1, 64, 16, "bf16", seed=1)
    q = T.queries(2, 2, 64, "bf16")
    kn = torch.zeros((2, 1, 64), device="cuda", dtype=torch.bfloat16)
    i32 = dict(device="cuda", dtype=torch.int32)
    ws = torch.zeros(1 << 24, device="cuda", dtype=torch.uint8)
    attend = dict(q=q, out=torch.empty_like(q), workspace=ws, k_new=kn, v_new=kn, lse=torch.zeros((2, 2), device="cuda"),
                  shared=torch.zeros(1, **i32), status=T.status_word())
    extend = dict(n_new=torch.ones(2, **i32), len_out=c.len, refs=c.refs, refs_out=c.refs, status=T.status_word())
    append = dict(k_new=kn, v_new=kn, start=torch.zeros(3, **i32), status=T.status_word())
    fork = dict(src_rows=torch.zeros(2, **i32), table_out=torch.zeros_like(c.table), len_out=torch.zeros(2, **i32), refs=c.refs, refs_out=c.refs,
                workspace=ws, status=T.status_word())
    pack = dict(refs=c.refs, refs_out=c.refs, table_out=c.table, workspace=ws, page_map=torch.zeros_like(c.refs), status=T.status_word())
    x = torch.zeros((2, 64), device="cuda")
    logits = dict(logits=x, out=torch.zeros_like(x))
    rules = dict(tokens=torch.zeros((2, 4), **i32), n_tokens=torch.zeros(2, **i32), n_prompt=torch.zeros(2, **i32), repetition=torch.ones(2, device="cuda"),
                 presence=torch.ones(2, device="cuda"), frequency=torch.ones(2, device="cuda"), temperature=torch.ones(2, device="cuda"),
                 bias_ids=torch.zeros((2, 1), **i32), bias_values=torch.zeros((2, 1), device="cuda"), mask=torch.zeros((2, 2), **i32))
    calls = [(lambda **a: B.kv_attend(c.kv, 0, group=2, **a), attend), (lambda **a: B.kv_extend(c.kv, **a), extend),
             (lambda **a: B.kv_append(c.kv, 0, **a), append), (lambda **a: B.kv_fork(c.kv, **a), fork),
             (lambda **a: B.kv_pack(c.kv, **a), pack), (lambda **a: B.logits_process(rules=B.make_logits_rules(), **a), logits),
             (B.make_logits_rules, rules), (lambda **a: B.make_kv(a["k"], a["v"], a["table"], a["length"]),
                                            dict(k=c.k, v=c.v, table=c.table, length=c.len))]
    before = B.launch_count()
    for call, args in calls:
        for name in args:
            with pytest.raises(ValueError):
                call(**{**args, name: args[name].cpu()})
        with pytest.raises(ValueError):
            call(**{name: t.cpu() for name, t in args.items()})
    with pytest.raises(ValueError):
        B.kv_status(torch.zeros(1, dtype=torch.int32))
    monkeypatch.setattr(B, "_device", lambda: 1)                # another device is current
    for call, args in calls[:6]:
        with pytest.raises(ValueError):
            call(**args)
    assert B.launch_count() == before


def test_driver_refuses_host_tensors():
    from paper_2512_15347_b200.kvcache import PagedCache
    c = PagedCache(32, 16, 1, 1, 64, 8, 64)
    c.admit(2)
    with pytest.raises(ValueError):
        c.extend(torch.tensor([3, 4], dtype=torch.int32))
    c.extend(torch.tensor([3, 4], device="cuda", dtype=torch.int32))
    with pytest.raises(ValueError):
        c.prune(torch.zeros(2, dtype=torch.int32), 1)
    assert c.n_rows == 2 and c.len.tolist() == [3, 4]
    c.check()


def test_new_values_without_keys_are_refused():
    c = T.Cache([20, 20], 1, 64, 16, "bf16", seed=1)
    q = T.queries(2, 2, 64, "bf16")
    new = torch.zeros((2, 1, 64), device="cuda", dtype=torch.bfloat16)
    ws = torch.zeros(B.kv_attend_workspace_bytes(c.kv, 2), device="cuda", dtype=torch.uint8)
    for kw in (dict(v_new=new), dict(k_new=new)):
        with pytest.raises(ValueError):
            B.kv_attend(c.kv, 0, q, torch.empty_like(q), ws, **kw)


# ------------------------------------------------------------------------------ rows that found no page

def look(cache):
    """What check_attention needs of a driver's cache, as it is now."""
    from types import SimpleNamespace
    return SimpleNamespace(k=cache.k, v=cache.v, table=cache.table.clone(), len=cache.len.clone())


@pytest.mark.parametrize("dtype,dim,page,prompt", [("bf16", 64, 16, 64), ("f16", 128, 16, 128), ("f32", 64, 16, 32), ("bf16", 72, 8, 64), ("f32", 40, 3, 9)])
def test_rows_without_a_page_take_no_new_token(dtype, dim, page, prompt):
    """A prompt of whole pages is expanded, the pool has pages for some of the rows only: the others' new tokens must not
    land in the prompt's last page, which all of them share.  Once by the decoding step, once by the appending call."""
    from paper_2512_15347_b200.kvcache import PagedCache
    G, N, heads, layers = 2, 6, 2, 2
    c = PagedCache(G * prompt // page + 5, page, layers, heads, dim, G * N, prompt + 4 * page, T.DT[dtype])
    c.admit(G)
    c.extend(prompt)
    new = lambda n, seed: torch.randn((n, heads, dim), generator=T.gen(seed), device="cuda").to(T.DT[dtype])
    start = torch.tensor([0, prompt, 2 * prompt], device="cuda", dtype=torch.int32)
    for layer in range(layers):
        c.append(layer, new(2 * prompt, layer), new(2 * prompt, 10 + layer), start)
    c.expand(N)
    c.check()
    c.extend(1)                                                 # pages for the first five rows
    with pytest.raises(B.PgError) as e:
        c.check()
    assert e.value.code == B.ENOPAGES
    assert c.len.tolist() == [prompt + 1] * 5 + [prompt] * 7
    q, kn, vn = T.queries(G * N, 4, dim, dtype), new(G * N, 20), new(G * N, 21)
    want_k, want_v = c.k.clone(), c.v.clone()
    for r in range(5):
        at = int(c.table[r, prompt // page])
        want_k[0, at, :, 0], want_v[0, at, :, 0] = kn[r], vn[r]
        want_k[1, at, :, 0], want_v[1, at, :, 0] = kn[r], vn[r]
    lse = torch.empty((G * N, 4), device="cuda")
    out = c.attend(0, q, kn, vn, lse=lse)
    T.check_attention(look(c), q, out, lse, dim ** -0.5, dtype)
    c.append(1, kn, vn)                                         # one token a row
    assert T.same_bits(c.k, want_k) and T.same_bits(c.v, want_v)
    c.status.zero_()
    c.append(1, kn, vn, torch.arange(G * N + 1, device="cuda", dtype=torch.int32))
    assert T.same_bits(c.k, want_k) and T.same_bits(c.v, want_v)
    c.check()
    # pruned to the rows that grew and one that did not, there are pages again
    c.prune(torch.tensor([0, 4, 6, 7], device="cuda", dtype=torch.int32), 2)
    c.extend(torch.tensor([1, 0, 1, 1], device="cuda", dtype=torch.int32))
    c.check()
    q, kn, vn = T.queries(4, 4, dim, dtype, seed=5), new(4, 22), new(4, 23)
    want_k, want_v = c.k.clone(), c.v.clone()
    for r in (0, 2, 3):
        n = int(c.len[r]) - 1
        want_k[1, c.table[r, n // page], :, n % page], want_v[1, c.table[r, n // page], :, n % page] = kn[r], vn[r]
    lse = torch.empty((4, 4), device="cuda")
    out = c.attend(1, q, kn, vn, lse=lse)
    assert T.same_bits(c.k, want_k) and T.same_bits(c.v, want_v)
    T.check_attention(look(c), q, out, lse, dim ** -0.5, dtype, layer=1)


def test_appended_tokens_beyond_what_a_row_has_grown_by_are_left_out():
    c = T.Cache([10, 20, 30], 1, 8, 8, "f32", seed=4)
    grown = torch.tensor([3, 2, 0], device="cuda", dtype=torch.int32)
    kv = B.make_kv(c.k, c.v, c.table, c.len, grown)
    new = torch.randn((9, 1, 8), generator=T.gen(5), device="cuda")
    want = c.k.clone()
    for r, t, pos in ((0, 0, 7), (0, 1, 8), (0, 2, 9), (1, 4, 18), (1, 5, 19)):
        want[0, c.rows[r][pos // 8], :, pos % 8] = new[t]
    st = T.status_word()
    B.kv_append(kv, 0, new, new, torch.tensor([0, 3, 6, 9], device="cuda", dtype=torch.int32), status=st)
    B.kv_status(st)
    assert T.same_bits(c.k, want)


def test_driver_wants_room_before_new_tokens():
    from paper_2512_15347_b200.kvcache import PagedCache
    c = PagedCache(32, 16, 1, 1, 64, 8, 64)
    q, new = (torch.zeros((2, 1, 64), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    c.admit(1)
    with pytest.raises(ValueError):
        c.append(0, new[:1], new[:1])
    c.extend(16)
    c.append(0, new[:1], new[:1])
    c.expand(2)
    with pytest.raises(ValueError):
        c.attend(0, q, new, new)                                # would overwrite the prompt's last token
    c.attend(0, q)
    c.extend(1)
    c.attend(0, q, new, new)
    c.check()


# ------------------------------------------------------------------------------ sizes near the ends of their types

@pytest.mark.parametrize("first", [0, 5])
def test_extend_by_more_pages_than_32_bits_count(first):
    """1024 rows that want 2^21 pages each, all at once, from a pool of a few: a row that fits, the rest refused, nothing handed out twice."""
    rows, width, pages = 1024, 1 << 21, 64
    k = torch.zeros((1, pages, 1, 1, 8), device="cuda", dtype=torch.bfloat16)
    table = torch.full((rows, width), -1, device="cuda", dtype=torch.int32)          # 8 GB
    length, refs, st = torch.zeros(rows, device="cuda", dtype=torch.int32), torch.zeros(pages, device="cuda", dtype=torch.int32), T.status_word()
    n_new = torch.full((rows,), width, device="cuda", dtype=torch.int32)
    n_new[0] = first
    grown = torch.full((rows,), 77, device="cuda", dtype=torch.int32)
    kv = B.make_kv(k, k.clone(), table, length, grown)
    B.kv_extend(kv, n_new, length, refs, refs, status=st)
    assert int(st) == 8
    assert length.tolist() == [first] + [0] * (rows - 1) and grown.tolist() == length.tolist()
    assert refs.tolist() == [1] * first + [0] * (pages - first)
    assert table[0, :first].tolist() == list(range(first))


def test_logits_of_the_longest_row():
    """The end of the last part passes 2^31."""
    x = torch.ones((1, 0x7FFF0000), device="cuda", dtype=torch.bfloat16)
    x[0, -1] = 3.0
    B.logits_process(x, x, B.make_logits_rules(temperature=torch.full((1,), 0.5, device="cuda")))
    assert x[0, -1] == 6.0 and bool((x[0, :-1] == 2.0).all())


# ------------------------------------------------------------------------------ scores far from zero

@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("size", [2.0 ** 6, 2.0 ** 9, 2.0 ** 11, 2.0 ** 13, 2.0 ** 15])
@pytest.mark.parametrize("scale", [0.125, 0.1, -0.1])
def test_scores_far_from_zero_take_the_largest(dtype, size, scale):
    """Queries and keys up to half the range of the smallest type: the largest score is apart from the rest by more than any weight
    spans, and the result is its token's value - in the tokens that a group shares and in the rows' own."""
    n, dim, tokens = 16, 64, 320
    c = T.shared_cache(2, n, 256, [64] * 2 * n, 1, dim, 16, dtype, seed=2)
    q = torch.full((2 * n, 4, dim), size, device="cuda", dtype=T.DT[dtype])
    q *= torch.linspace(0.5, 1, 2 * n, device="cuda").to(T.DT[dtype])[:, None, None]
    sign = 1 if scale > 0 else -1
    for g, best in ((0, 200), (1, 100)):
        for t in range(256):                                       # shared tokens: levels below the best one, rising and falling
            level = size if t == best else size * (0.25 + 0.125 * (t % 5))
            c.k[0, c.rows[g * n][t // 16], 0, t % 16] = sign * level
    own = {}
    for r in range(2 * n):
        for t in range(256, tokens):
            c.k[0, c.rows[r][t // 16], 0, t % 16] = sign * size * 0.5
        if r % 2:                                                  # every other row has its largest score in a token of its own
            own[r] = 256 + r
            c.k[0, c.rows[r][own[r] // 16], 0, own[r] % 16] = sign * size * 1.5
    sh = torch.full((2,), 256, device="cuda", dtype=torch.int32)
    for kw in (dict(group=n, shared=sh), dict()):
        out, lse = T.run_attention(c, q, dtype, scale=scale, **kw)
        assert torch.isfinite(lse).all()
        for r in range(2 * n):
            t = own.get(r, (200, 100)[r // n])
            v = c.v[0, c.rows[r][t // 16], 0, t % 16].double()
            # the one weight is rounded to the type, and the result: u each, and fp32's roundings beside them
            assert ((out[r].double() - v).abs() <= 2.1 * T.UNIT[dtype] * v.abs() + 2.0 ** -22 * v.abs() + 2.0 ** -24).all(), (r, t)


# ------------------------------------------------------------------------------ many small weights beside a large one

@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("nats", [10.0, 14.0, 16.0, 17.0, 17.5])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 16), (72, 5)])
def test_small_weights_beside_a_token_of_value_zero(dtype, nats, dim, page):
    """One token far above the others that carries no value (an attention sink): the result is the others' share, whose weights
    are below what the type resolves near 1.  In the rows' own tokens, in tokens that a group shares, and with the sink in one and
    the others in the other."""
    tokens = 16384
    c = T.Cache([tokens + 1, tokens, 300], 1, dim, page, dtype, seed=40)
    q = torch.zeros((3, 2, dim), device="cuda", dtype=T.DT[dtype])
    q[:, :, 0] = 4.0
    c.k[:, :, :, :, :] = torch.where(torch.isnan(c.k), c.k, torch.zeros_like(c.k))
    c.v.abs_()
    for r, t in ((0, 5000), (1, 0), (2, 299)):
        c.k[0, c.rows[r][t // page], 0, t % page, 0] = nats / 4
        c.v[0, c.rows[r][t // page], 0, t % page] = 0
    out, lse = T.run_attention(c, q, dtype, scale=1.0)
    T.check_attention(c, q, out, lse, 1.0, dtype)
    if dtype == "f32":
        return
    n, shared = 8, 4096 // page // 64 * 64 * page              # whole tiles of whole pages
    g = T.shared_cache(3, n, shared, [200] * 3 * n, 1, dim, page, dtype, seed=41)
    q = torch.zeros((3 * n, 2, dim), device="cuda", dtype=T.DT[dtype])
    q[:, :, 0] = 4.0
    g.k[:, :, :, :, :] = torch.where(torch.isnan(g.k), g.k, torch.zeros_like(g.k))
    g.v.abs_()
    for r in range(3 * n):
        t = (1000, shared - 1, shared + 77)[r // n]            # early and late in the shared tokens; in each row's own
        g.k[0, g.rows[r][t // page], 0, t % page, 0] = nats / 4
        g.v[0, g.rows[r][t // page], 0, t % page] = 0
    sh = torch.full((3,), shared, device="cuda", dtype=torch.int32)
    out, lse = T.run_attention(g, q, dtype, scale=1.0, group=n, shared=sh)
    T.check_attention(g, q, out, lse, 1.0, dtype)


# ------------------------------------------------------------------------------ the driver's streams

def driver(tokens, rows=3):
    from paper_2512_15347_b200.kvcache import PagedCache
    c = PagedCache(rows * -(-tokens // 16) + 4, 16, 1, 2, 64, rows, tokens + 40)
    c.admit(rows)
    c.extend(tokens)
    kn = torch.randn((rows * tokens, 2, 64), generator=T.gen(8), device="cuda").bfloat16()
    c.append(0, kn, kn.flip(0).contiguous(), torch.arange(rows + 1, device="cuda", dtype=torch.int32) * tokens)
    return c


def test_driver_calls_on_two_streams_share_no_workspace():
    c = driver(5000)
    qs = [T.queries(3, 8, 64, "bf16", seed=s) for s in range(6)]
    good = [c.attend(0, q) for q in qs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    here = c._space(1)
    with torch.cuda.stream(side):
        c.attend(0, qs[0])
        there = c._space(1)
    assert here.data_ptr() != there.data_ptr()
    torch.cuda.synchronize()
    outs = [torch.empty_like(q) for q in qs]
    for _ in range(5):
        for i, q in enumerate(qs):                             # calls that overlap
            with torch.cuda.stream(side if i % 2 else torch.cuda.current_stream()):
                c.attend(0, q, out=outs[i])
        torch.cuda.synchronize()
        for a, b in zip(outs, good):
            assert torch.equal(a, b)


def test_driver_workspace_made_under_capture_stays_with_the_graph():
    """What zeroes it runs at the replay, not when it is made: a call outside the graph must not find it."""
    c = driver(5000)
    q = T.queries(3, 8, 64, "bf16")
    good = c.attend(0, q)
    c._spaces.clear()                                          # as before any call
    side, out = torch.cuda.Stream(), torch.empty_like(q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.attend(0, q, out=out)
    assert not c._spaces
    with torch.cuda.stream(side):
        again = c.attend(0, q)
    torch.cuda.synchronize()
    assert torch.equal(again, good)
    for _ in range(2):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, good)


def test_driver_workspace_that_a_graph_uses_outlives_growth():
    c = driver(5000)
    q = T.queries(3, 8, 64, "bf16")
    side, out = torch.cuda.Stream(), torch.empty_like(q)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        good = c.attend(0, q)
        used = c._space(1).data_ptr()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.attend(0, q, out=out)
    with torch.cuda.stream(side):
        grown = c._space(1 << 30)
        assert grown.data_ptr() != used and c._space(1) is grown
        taken = [torch.full((1 << 20,), 255, device="cuda", dtype=torch.uint8) for _ in range(64)]
        assert all(not t.data_ptr() <= used < t.data_ptr() + t.nbytes for t in taken)
    torch.cuda.synchronize()
    for _ in range(2):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, good)


def test_driver_refuses_before_it_changes_anything():
    c = driver(100)
    q = T.queries(3, 8, 64, "bf16")
    good, refs = c.attend(0, q), c.refs.clone()
    for refused in (lambda: c.admit(4), lambda: c.admit(-1), lambda: c.expand(0), lambda: c.expand(-2), lambda: c.expand(2),
                    lambda: c.prune(torch.zeros(0, device="cuda", dtype=torch.int32), 0)):
        with pytest.raises(ValueError):
            refused()
        assert c.n_rows == 3 and c.group == 1 and c.len.tolist() == [100] * 3 and torch.equal(c.refs, refs)
        assert torch.equal(c.attend(0, q), good)
    c.check()


def test_rules_of_another_shape_are_refused():
    i32 = dict(device="cuda", dtype=torch.int32)
    for rules in (dict(n_tokens=torch.zeros((2, 3), **i32)), dict(n_prompt=torch.zeros((2, 2), **i32)), dict(n_tokens=torch.zeros((), **i32)),
                  dict(bias_ids=torch.zeros(2, **i32), bias_values=torch.zeros(2, device="cuda")),
                  dict(bias_ids=torch.zeros((2, 1, 1), **i32), bias_values=torch.zeros((2, 1, 1), device="cuda"))):
        with pytest.raises(ValueError):
            B.make_logits_rules(tokens=torch.zeros((2, 4), **i32), **rules)
    B.make_logits_rules(tokens=torch.zeros((2, 4), **i32), n_tokens=torch.zeros((2, 1), **i32))
