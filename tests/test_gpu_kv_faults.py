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
