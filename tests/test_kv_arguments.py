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
