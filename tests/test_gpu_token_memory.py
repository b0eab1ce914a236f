"""Tensors that a token call was given are free when the caller lets go of them, not when the garbage collector next runs."""
import gc
import weakref

import pytest
import torch

from paper_2512_15347_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture
def no_collector():
    gc.collect()
    gc.disable()
    yield
    gc.enable()


def test_terms_and_rules_let_go_of_their_tensors(no_collector):
    ids = torch.zeros((4, 8), device="cuda", dtype=torch.int32)
    logp, x, tau = torch.zeros((4, 8), device="cuda"), torch.zeros((4, 100), device="cuda"), torch.ones(4, device="cuda")
    terms = B.make_token_terms(ids=ids, teacher_ids=ids, teacher_logp=logp, temperature=tau)
    B.token_forward(x, terms, lse=torch.empty(4, device="cuda"))
    rules = B.make_logits_rules(temperature=tau)
    B.logits_process(x, torch.empty_like(x), rules)
    seen = [weakref.ref(t) for t in (ids, logp, tau)]
    del ids, logp, tau, terms, rules
    assert [s() for s in seen] == [None] * 3


def test_update_steps_hold_no_memory(no_collector):
    from paper_2512_15347_b200.token_update import TokenUpdate, score
    n, V = 64, 1000
    x = torch.randn((n, V), device="cuda")
    start, adv = torch.tensor([0, n], device="cuda", dtype=torch.int32), torch.ones(1, device="cuda")
    rule = TokenUpdate(distill_coef=0.5, kind="reverse_rest")

    def step():
        lists = score(x, n_top=64)
        rule.step(x, lists.top_ids[:, 0].contiguous(), start, adv, teacher=(lists.top_ids, lists.top_logp))

    step()
    held = torch.cuda.memory_allocated()
    for _ in range(5):
        step()
    assert torch.cuda.memory_allocated() == held


def test_a_cache_lets_go_of_its_pool(no_collector):
    from paper_2512_15347_b200.kvcache import PagedCache
    before = torch.cuda.memory_allocated()
    cache = PagedCache(n_pages=64, page_size=16, n_layers=2, n_kv_heads=2, head_dim=64, max_rows=8, max_tokens=128)
    cache.admit(2)
    cache.extend(3)
    cache.expand(4)
    cache.check()
    del cache
    assert torch.cuda.memory_allocated() == before


def test_counts_beyond_32_bits_are_refused():
    """They would be cut to 32 bits on the way to the library: a batch of 2^32 + 5 tokens to one of five."""
    n = 2 ** 32 + 5
    logits = torch.empty(n, device="cuda", dtype=torch.bfloat16)
    one = torch.full((1,), 7.0, device="cuda")
    for shape in ((1, n), (n, 1)):
        with pytest.raises(ValueError):
            B.token_forward(logits.view(shape), B.make_token_terms(), lse=one)
    del logits
    lp = torch.empty(n, device="cuda")
    ws = torch.zeros(B.token_objective_workspace_bytes(5), device="cuda", dtype=torch.uint8)
    with pytest.raises(ValueError):
        B.token_objective(torch.tensor([0, 5], device="cuda", dtype=torch.int32), lp, one, one.clone(), lp, ws)
    with pytest.raises(ValueError):
        B.token_objective_workspace_bytes(n)
    assert float(one) == 7.0
    del lp
    torch.cuda.empty_cache()
