"""Teachers' lists whose log-probabilities lie far from 0: raw logits, lists of tokens that the teacher masks by a finite value."""
import math

import pytest
import torch

from paper_2512_15347_b200 import binding as B
from tests.test_gpu_token_update import check_forward, check_gradient, make, outputs, reference, terms_of

pytestmark = pytest.mark.gpu

GRADS = ("dlogp", "dentropy", "ddistill")


def check_kind(c, kind):
    R = c["x"].shape[0]
    rows = reference(c, kind)
    for w in rows:
        if w["distill"] > 3.4028235e38:                             # no number of 32 bits
            w["distill"] = math.inf
    o, one, two = outputs(R, c, 0, True), torch.empty_like(c["x"]), torch.empty_like(c["x"])
    B.token_forward_backward(c["x"], terms_of(c, kind), one, **o, **{k: c[k] for k in GRADS})
    check_forward(c, o, rows)
    check_gradient(c, one, rows)
    o = outputs(R, c, 0, True)
    B.token_forward(c["x"], terms_of(c, kind), **o)
    check_forward(c, o, rows)
    B.token_backward(c["x"], terms_of(c, kind), o["saved"], two, **{k: c[k] for k in GRADS})
    check_gradient(c, two, rows)


@pytest.mark.parametrize("k", [1, 7, 40, 256])
@pytest.mark.parametrize("at", [-1e9, -3e38, -1e5, 3000.0, 1e6, 3e38])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_renormalised_list_of_any_logits(dtype, at, k):
    """t is the softmax over the list: only differences count."""
    c = make(6, 5003, dtype, 17, n_list=k, masks=False)
    c["list_logp"] = c["list_logp"] + at
    c["list_logp"][1] = at
    c["list_ids"][4] = -1
    check_kind(c, "forward")


@pytest.mark.parametrize("k", [2, 40, 256])
@pytest.mark.parametrize("kind", ["forward_rest", "reverse_rest"])
@pytest.mark.parametrize("far", [-200.0, -1e9, -3e38])
def test_lists_with_tokens_that_the_teacher_masks(far, kind, k):
    """As a teacher's alternatives are where its mask leaves fewer tokens than the list has places.  In the reverse kind what the policy gives
    such a token costs p_i |tl_i|: with a p_i of 1e-6 a number of 32 bits."""
    c = make(6, 5003, torch.float32, 18, n_list=k, masks=False, peaks=0.0)
    c["x"] *= 0.1
    c["list_logp"][:, 1:] = far
    c["list_logp"][0, : k // 2] = -3.0
    c["ddistill"] = c["ddistill"].sign() * 0.25
    check_kind(c, kind)


@pytest.mark.parametrize("k", [33, 64, 200])
@pytest.mark.parametrize("low,high", [(-65504.0, 0.0), (-1e9, 0.0), (-3e38, 3e38)])
def test_entries_of_no_weight_whose_tokens_the_policy_masks(low, high, k):
    """Teacher and policy under one grammar: the tail of the teacher's list has t_i = 0, and its tokens are not allowed."""
    c = make(6, 5003, torch.bfloat16, 19, n_list=k, masks=False)
    c["list_logp"] += high
    c["list_ids"][0, k // 2:] = c["list_ids"][1, k // 2: 2 * (k // 2) + k % 2]      # make leaves them out
    for r in (0, 2, 5):
        tail = c["list_ids"][r, 20:].long()
        keep = ~torch.isin(tail, c["ids"][r].long()) & ~torch.isin(tail, c["list_ids"][r, :20].long())
        c["list_logp"][r, 20:] = low
        c["x"][r, tail[keep]] = -math.inf
    rows = reference(c, "forward")
    assert all(math.isfinite(w["distill"]) for w in rows)
    check_kind(c, "forward")


@pytest.mark.parametrize("kind", ["forward", "forward_rest"])
@pytest.mark.parametrize("low", [-86.0, -90.0, -99.0, -102.5])
def test_entries_of_next_to_no_weight_whose_tokens_the_policy_masks(low, kind):
    """t_i is next to 0, below the smallest normal number, but not 0: the divergence is infinite."""
    c = make(3, 5003, torch.float32, 23, n_list=12, masks=False)
    c["list_logp"][:, 0], c["list_logp"][:, 9:] = -0.01, low
    tail = c["list_ids"][:, 10].long()
    c["x"][torch.arange(3), tail] = -math.inf
    rows = reference(c, kind)
    o = outputs(3, c, 0, True)
    B.token_forward(c["x"], terms_of(c, kind), **o)
    assert [w["distill"] for w in rows] == [math.inf] * 3
    assert o["distill"].tolist() == [math.inf] * 3
