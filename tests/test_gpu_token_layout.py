"""Logits that are not one block of memory: slices of a padded vocabulary, rows that begin off 16 bytes, through the update driver; what it allocates."""
import pytest
import torch

from tests.test_gpu_token_update import ALL, check_gradient, make, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("V,pitch,first", [(5003, 5056, 0), (5003, 5003, 0), (5000, 5001, 3), (9, 64, 1), (7, 7, 0), (1, 5, 2), (5003, 20000, 7)])
def test_the_gradient_lies_on_its_logits_offsets(dtype, V, pitch, first):
    """A gradient whose rows lie on the 16-byte offsets of the logits' rows is written by whole units."""
    from paper_2512_15347_b200.token_update import TokenUpdate
    n = 6
    c = make(n, V, dtype, V, masks=False)
    room = torch.randn((n, first + pitch), device="cuda").to(dtype)
    x = room[:, first: first + V]
    x.copy_(c["x"])
    c["x"] = x
    start, adv = torch.tensor([0, 2, n], device="cuda", dtype=torch.int32), torch.tensor([0.5, -1.0], device="cuda")
    u = TokenUpdate(norm="sum").step(x, c["ids"].view(-1), start, adv, temperature=c["tau"])
    g = u.dlogits
    assert g.shape == x.shape and g.dtype == dtype and g.stride(1) == 1
    for r in range(n):
        assert (g[r].data_ptr() - x[r].data_ptr()) % 16 == 0
    # no more room than the rows need
    assert g.untyped_storage().nbytes() <= (n * (V + 16) + 16) * x.element_size()
    w = dict(c, dlogp=torch.tensor([0.5] * 2 + [-1.0] * 4, device="cuda")[:, None], dentropy=torch.zeros(n, device="cuda"))
    check_gradient(w, g, reference(w, entropy=False))


def test_a_contiguous_batch_gets_a_contiguous_gradient():
    from paper_2512_15347_b200.token_update import TokenUpdate
    x = torch.randn((4, 1000), device="cuda").to(torch.bfloat16)
    u = TokenUpdate().step(x, torch.zeros(4, device="cuda", dtype=torch.int32), torch.tensor([0, 4], device="cuda", dtype=torch.int32), torch.ones(1, device="cuda"))
    assert u.dlogits.is_contiguous()


@pytest.mark.parametrize("default", [torch.bfloat16, torch.float64])
def test_the_driver_does_not_depend_on_torchs_default_type(default):
    """Training programs set it to their weights' type; the calls' outputs are fp32 all the same."""
    from paper_2512_15347_b200.token_update import TokenUpdate, score
    x = torch.randn((5, 1000), device="cuda", dtype=torch.bfloat16)
    start, adv = torch.tensor([0, 2, 5], device="cuda", dtype=torch.int32), torch.tensor([0.5, -1.0], device="cuda")

    def steps():
        lists = score(x, torch.arange(5, device="cuda", dtype=torch.int32), n_top=8)
        u = TokenUpdate(entropy_coef=0.1, distill_coef=0.5, kind="reverse_rest").step(x, lists.top_ids[:, 1].contiguous(), start, adv, lists.logp[:, 0].contiguous(),
                                                                                     teacher=(lists.top_ids, lists.top_logp))
        return list(lists) + list(u)

    want = steps()
    before = torch.get_default_dtype()
    torch.set_default_dtype(default)
    try:
        got = steps()
    finally:
        torch.set_default_dtype(before)
    for a, b in zip(got, want):
        assert a.dtype == b.dtype and torch.equal(a, b)
