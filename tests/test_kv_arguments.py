"""Argument checks of the token-rollout calls that come before any CUDA call, without a GPU."""
import pytest
import torch

from paper_2512_15347_b200 import binding as B


def pools(**kw):
    a = dict(n_layers=1, n_pages=4, n_kv_heads=1, page_size=16, head_dim=64)
    a.update(kw)
    return torch.zeros(a["n_layers"], a["n_pages"], a["n_kv_heads"], a["page_size"], a["head_dim"], dtype=torch.bfloat16)


def test_host_tensors_do_not_make_a_cache():
    k = pools()
    with pytest.raises(ValueError):
        B.make_kv(k, k.clone(), torch.zeros((2, 2), dtype=torch.int32), torch.zeros(2, dtype=torch.int32))


def test_host_tensors_do_not_make_rules():
    for rules in (dict(temperature=torch.ones(2)), dict(tokens=torch.zeros((2, 3), dtype=torch.int32)), dict(mask=torch.zeros((1, 3), dtype=torch.int32))):
        with pytest.raises(ValueError):
            B.make_logits_rules(**rules)


def test_host_logits_and_status_are_refused():
    x = torch.zeros((2, 64))
    with pytest.raises(ValueError):
        B.logits_process(x, x.clone(), B.make_logits_rules())
    with pytest.raises(ValueError):
        B.kv_status(torch.zeros(1, dtype=torch.int32))


def described(**kw):
    """A descriptor with addresses that nothing follows."""
    a = dict(k=1 << 20, v=1 << 21, dtype=B.BF16, n_layers=1, n_pages=64, n_kv_heads=1, page_size=16, head_dim=8, page_stride=128, layer_stride=0,
             table=1 << 22, len=1 << 23, n_rows=4, max_pages=8, grown=None)
    a.update(kw)
    return B.Kv(*(a[name] for name, _ in B.Kv._fields_))


@pytest.mark.parametrize("kw,good", [
    (dict(), True),
    (dict(n_pages=2 ** 31 - 2 ** 20), True), (dict(n_pages=2 ** 31 - 2 ** 20 + 1), False), (dict(n_pages=2 ** 31 - 1), False),
    (dict(n_rows=2 ** 31 - 2 ** 20), True), (dict(n_rows=2 ** 31 - 1), False),
    (dict(page_size=1, page_stride=8, max_pages=2 ** 31 - 4097), True), (dict(page_size=1, page_stride=8, max_pages=2 ** 31 - 4096), False),
    # a length near the row's end, rounded up to whole pages, would pass 31 bits
    (dict(page_size=1 << 20, page_stride=1 << 23, max_pages=2046), True), (dict(page_size=1 << 20, page_stride=1 << 23, max_pages=2047), False),
])
def test_counts_that_pass_32_bits_on_the_way_are_refused(kw, good):
    import ctypes
    kv = described(**kw)
    L, at = B.lib(), ctypes.byref(kv)
    for need in (L.pg_kv_attend_workspace_bytes(at, 1, 1), L.pg_kv_fork_workspace_bytes(at, 1), L.pg_kv_pack_workspace_bytes(at)):
        assert (need > 0) == good
    if not good:
        some = 1 << 24
        assert L.pg_kv_extend(at, None, 1, some, some, some, None, None) == B.EINVAL
        assert L.pg_kv_append(at, 0, kv.n_rows, some, some, 0, None, None, None) == B.EINVAL


def test_forks_that_pass_32_bits_are_refused_before_any_launch():
    import ctypes
    L, kv, some = B.lib(), described(), 1 << 24
    assert L.pg_kv_fork_workspace_bytes(ctypes.byref(kv), 2 ** 31 - 1) == 0
    assert L.pg_kv_fork(ctypes.byref(kv), 2 ** 31 - 1, some, some, some, some, some, some, 1 << 40, None, None) == B.EINVAL
    # more pieces of pages over all layers than 32 bits count: known before the counts are touched
    kv = described(n_layers=2 ** 31 - 1, layer_stride=128)
    assert L.pg_kv_fork_workspace_bytes(ctypes.byref(kv), 4) == 0 and L.pg_kv_pack_workspace_bytes(ctypes.byref(kv)) == 0
    assert L.pg_kv_fork(ctypes.byref(kv), 4, some, some, some, some, some, some, 1 << 40, None, None) == B.EINVAL
    assert L.pg_kv_pack(ctypes.byref(kv), some, some, some, None, some, 1 << 40, None, None) == B.EINVAL
