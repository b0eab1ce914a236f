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
