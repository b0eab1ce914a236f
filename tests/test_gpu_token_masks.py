"""Rows of logits masked by finite values far below the others (-1e9, -1e10, -1e20, ... of a grammar, a padded vocabulary), and small
temperatures, which put logits as far apart: log-probs, entropy, divergences and gradients against 64 bits."""
import math

import pytest
import torch

from paper_2512_15347_b200 import binding as B
from tests import token_reference as ref
from tests.test_gpu_token_update import check_forward, check_gradient, close, make, outputs, reference, terms_of, tiles_of, tol_logp

pytestmark = pytest.mark.gpu

MASKS = [-1e4, -1e9, -5e9, -1e10, -1e15, -1e20, -1e30, -3e38]
GRADS = ("dlogp", "dentropy", "ddistill")


def masked(V, dtype, mask, seed, n_list=6, whole=False):
    """Rows of which few tokens are allowed, a half, all but one, one alone, none of a run; whole: rows masked throughout, and rows whose
    list has all allowed tokens."""
    R = 5
    c = make(R, V, dtype, seed, n_ids=2, n_list=n_list, masks=False)
    x = c["x"]
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    if not whole:
        x[0, torch.rand(V, generator=g, device="cuda") > 8 / V] = mask
        x[0, V // 2] = 1.5
        x[1, V // 2:] = mask
        x[2, V // 3] = mask
        x[3, 1:] = mask
        x[4, V // 4: V // 2] = mask
        return c
    x[0] = mask
    x[1] = (mask + 3 * torch.randn(V, generator=g, device="cuda")).to(dtype)
    for r in (2, 3):                                        # allowed: the listed ones
        on = c["list_ids"][r].long()
        kept = x[r, on].clone()
        x[r] = mask if r == 2 else (mask * (0.5 + 0.5 * torch.rand(V, generator=g, device="cuda"))).to(dtype)
        x[r, on] = kept
    c["list_ids"][3, 3:] = -1                               # all but three
    x[4] = mask
    x[4, V // 2:] = mask * 0.9375
    return c


def check(c, o, rows, n_top):
    """check_forward, where logits lie far from 0.  A divergence's size is that of all its terms t_i ln p_i: the reference counts an ln p_i below
    -1e4 as -1e4; such terms are of one sign (t_i |ln p_i|), so all of them are no more than the divergence and what is counted.  Log-probs of
    alternatives by differences from the largest logit: at 1e20 a difference of two 64-bit numbers next to each other is 16384."""
    for w in rows:
        if w["distill"] > 3.4028235e38:                     # no number of 32 bits
            w["distill"] = math.inf
        if math.isfinite(w["distill"]):
            w["size_distill"] += abs(w["distill"])
    check_forward(c, {k: v for k, v in o.items() if not k.startswith("top")}, rows)
    for r in range(len(rows)):
        x, tau = c["x"][r].double(), float(c["tau"][r])
        at = ref.alternatives(c["x"][r], n_top)
        assert o["top_ids"][r].tolist() == at.tolist(), ("top_ids", r)
        lp = (x[at] - x.max()) / tau - torch.logsumexp((x - x.max()) / tau, -1)
        for j in range(n_top):
            tol = tol_logp(tiles_of(x.numel(), c["x"].dtype), float(x.max() - x[at[j]]) / tau, float(lp[j]))
            close(o["top_logp"][r, j], lp[j], tol, ("top", r, j))


@pytest.mark.parametrize("whole", [False, True])
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [9, 20011, 140000])
def test_masked_tokens_do_not_disturb_their_row(V, dtype, mask, whole):
    c = masked(V, dtype, mask, V, whole=whole)
    for kind in B.DISTILL_KINDS:
        rows = reference(c, kind)
        o = outputs(5, c, 3, True)
        B.token_forward(c["x"], terms_of(c, kind, n_top=3), **o)
        check(c, o, rows, 3)
        o, g = outputs(5, c, 3, True), torch.empty_like(c["x"])
        B.token_forward_backward(c["x"], terms_of(c, kind, n_top=3), g, **o, **{k: c[k] for k in GRADS})
        check(c, o, rows, 3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tau", [1e-6, 1e-9, 1e-20])
def test_log_probs_at_small_temperatures(dtype, tau):
    c = make(5, 9001, dtype, 3, n_ids=2, masks=False)
    c["x"][1:3] = -20 - c["x"][1:3].abs()
    c["tau"].fill_(tau)
    o = outputs(5, c, 3)
    B.token_forward(c["x"], terms_of(c, n_top=3), **o)
    check(c, o, reference(c), 3)


@pytest.mark.parametrize("whole", [False, True])
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [9, 20011, 140000])
def test_gradients_of_masked_rows(V, dtype, mask, whole):
    """Where nothing else is left - in the row, or outside the teacher's list - masked tokens are what the gradient's slope refers to."""
    c = masked(V, dtype, mask, V + 1, whole=whole)
    for kind in B.DISTILL_KINDS:
        rows = reference(c, kind)
        grads = {k: c[k] for k in GRADS}
        o, one, two = outputs(5, c, 0, True), torch.full_like(c["x"], 7), torch.full_like(c["x"], 7)
        B.token_forward_backward(c["x"], terms_of(c, kind), one, **o, **grads)
        check_gradient(c, one, rows)
        B.token_backward(c["x"], terms_of(c, kind), o["saved"], two, **grads)
        check_gradient(c, two, rows)
        # without entropy
        plain = dict(c, dentropy=torch.zeros(5, device="cuda"))
        rows = reference(plain, kind)
        B.token_forward_backward(c["x"], terms_of(c, kind), one, dlogp=c["dlogp"], ddistill=c["ddistill"])
        check_gradient(c, one, rows)
        B.token_backward(c["x"], terms_of(c, kind), o["saved"], two, dlogp=c["dlogp"], ddistill=c["ddistill"])
        check_gradient(c, two, rows)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tau", [1e-6, 1e-9])
def test_gradients_at_small_temperatures(dtype, tau):
    """With weights as small as T, so that gradients are of ordinary size."""
    c = make(5, 9001, dtype, 3, n_ids=2, n_list=6, masks=False)
    c["x"][1:3] = -20 - c["x"][1:3].abs()
    c["tau"].fill_(tau)
    for k in GRADS:
        c[k] *= tau
    for kind in B.DISTILL_KINDS:
        rows = reference(c, kind)
        o, one, two = outputs(5, c, 0, True), torch.full_like(c["x"], 7), torch.full_like(c["x"], 7)
        B.token_forward_backward(c["x"], terms_of(c, kind), one, **o, **{k: c[k] for k in GRADS})
        check_gradient(c, one, rows)
        B.token_backward(c["x"], terms_of(c, kind), o["saved"], two, **{k: c[k] for k in GRADS})
        check_gradient(c, two, rows)
