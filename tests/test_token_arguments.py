"""Argument checks of the policy-update calls on token trajectories that come before any CUDA call, and the plain forms that the
calls are tested against, without a GPU."""
import ctypes
import math

import pytest
import torch

from paper_2512_15347_b200 import binding as B
from tests import token_reference as ref

SOME = 1 << 24


def forward(rows=4, vocab=100, dtype=B.F32, logits=SOME, stride=0, terms=None, **out):
    t = B.TokenTerms(**(terms or {}))
    return B.lib().pg_token_forward(rows, vocab, dtype, logits, stride, t, B.TokenOut(**out), None)


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(vocab=0), dict(vocab=B.TOKEN_MAX_VOCAB + 1), dict(dtype=3), dict(dtype=-1), dict(logits=None), dict(logits=SOME + 2),
    dict(stride=99), dict(stride=2 ** 60), dict(saved=SOME + 4), dict(top_logp=SOME),
    dict(terms=dict(n_top=B.TOKEN_MAX_TOP + 1)), dict(terms=dict(n_top=-1)), dict(vocab=5, terms=dict(n_top=6)),
    dict(terms=dict(ids=SOME, n_ids=B.TOKEN_MAX_LIST + 1)), dict(terms=dict(ids=SOME, n_ids=-1)), dict(terms=dict(kind=3)), dict(terms=dict(kind=-1)),
    dict(terms=dict(teacher_ids=SOME, n_teacher=4)), dict(terms=dict(teacher_ids=SOME, teacher_logp=SOME, n_teacher=B.TOKEN_MAX_LIST + 1)),
])
def test_forward_refuses(kw):
    assert forward(**kw) == B.EINVAL


def test_no_rows_and_null_descriptors():
    L = B.lib()
    assert forward(rows=0, logits=None) == B.OK
    assert L.pg_token_forward(4, 100, B.F32, SOME, 0, None, B.TokenOut(), None) == B.EINVAL
    assert L.pg_token_forward(4, 100, B.F32, SOME, 0, B.TokenTerms(), None, None) == B.EINVAL
    assert L.pg_token_backward(4, 100, B.F32, SOME, 0, B.TokenTerms(), SOME, None, SOME, 0, None) == B.EINVAL
    assert L.pg_token_forward_backward(4, 100, B.F32, SOME, 0, B.TokenTerms(), None, B.TokenGrads(), SOME, 0, None) == B.EINVAL


@pytest.mark.parametrize("kw", [
    dict(saved=None), dict(saved=SOME + 8), dict(dl=None), dict(dl=SOME + 2), dict(dl_stride=50), dict(dl=SOME, dl_stride=128),
    dict(grads=dict(dlogp=SOME)), dict(grads=dict(ddistill=SOME)),
])
def test_backward_refuses(kw):
    a = dict(saved=SOME, dl=2 * SOME, dl_stride=0, grads={})
    a.update(kw)
    L, t, g = B.lib(), B.TokenTerms(), B.TokenGrads(**a["grads"])
    assert L.pg_token_backward(4, 100, B.F32, SOME, 0, t, a["saved"], g, a["dl"], a["dl_stride"], None) == B.EINVAL
    if "saved" not in kw:
        assert L.pg_token_forward_backward(4, 100, B.F32, SOME, 0, t, B.TokenOut(), g, a["dl"], a["dl_stride"], None) == B.EINVAL


@pytest.mark.parametrize("kw", [
    dict(n_rows=-1), dict(n_rows=2 ** 31 - 1), dict(n_tokens=-1), dict(n_tokens=2 ** 31 - 1), dict(start=None), dict(adv=None), dict(logp_new=None),
    dict(objective=None), dict(dlogp=None), dict(ws=None), dict(ws=SOME + 8), dict(size=4096), dict(norm=3), dict(norm=-1), dict(clip_low=1.01),
    dict(clip_low=-0.1), dict(clip_high=-0.1), dict(clip_high=math.nan),
])
def test_objective_refuses(kw):
    a = dict(n_rows=3, n_tokens=50, start=SOME, adv=SOME, logp_new=SOME, objective=SOME, dlogp=SOME, ws=SOME, size=1 << 20, norm=0, clip_low=0.2, clip_high=0.2)
    a.update(kw)
    b = B.TokenBatch(start=a["start"], logp_new=a["logp_new"], adv=a["adv"], clip_low=a["clip_low"], clip_high=a["clip_high"], scale=1.0, norm=a["norm"])
    assert B.lib().pg_token_objective(a["n_rows"], a["n_tokens"], b, a["objective"], a["dlogp"], None, None, None, a["ws"], a["size"], None, None) == B.EINVAL


def test_workspace_grows_with_tokens_and_stops():
    sizes = [B.token_objective_workspace_bytes(n) for n in (0, 1, 1024, 1025, 10 ** 6, 2 ** 31 - 2 ** 20)]
    assert sizes == sorted(sizes) and sizes[0] > 4096 and sizes[-1] < 1 << 20
    assert B.token_objective_workspace_bytes(-1) == 0


def test_host_tensors_are_refused():
    with pytest.raises(ValueError):
        B.make_token_terms(ids=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        B.token_forward(torch.zeros(3, 5), B.make_token_terms())
    with pytest.raises(ValueError):
        B.token_objective(torch.zeros(2, dtype=torch.int32), torch.zeros(3), torch.zeros(1), torch.zeros(1), torch.zeros(3), torch.zeros(8192, dtype=torch.uint8))


def test_the_plain_gradient_is_the_one_of_differences():
    """In 64 bits, h = 1e-5: off by h^2 times a third derivative below 100 and by 1e-15 / h."""
    g = torch.Generator().manual_seed(1)
    for kind in B.DISTILL_KINDS:
        x = 2 * torch.randn(12, generator=g, dtype=torch.float64)
        x[5] = -math.inf
        kw = dict(tau=0.7, ids=[3, 3, 8, -1], list_ids=[1, 8, 2, -1], list_logp=[-1.0, -0.9, -2.0, 0.0], kind=kind)
        w = dict(dlogp=[0.5, -1.0, 2.0, 9.0], dentropy=0.3, ddistill=-0.8)
        out = ref.row_terms(x, **kw, **w)

        def value(y):
            o = ref.row_terms(y, **kw)
            return sum(a * b for a, b in zip(o["logp"].tolist(), w["dlogp"])) + w["dentropy"] * o["entropy"] + w["ddistill"] * o["distill"]

        for v in range(12):
            up, down = x.clone(), x.clone()
            up[v] += 1e-5
            down[v] -= 1e-5
            d = 0.0 if v == 5 else (value(up) - value(down)) / 2e-5
            assert abs(d - float(out["gradient"][v])) <= 1e-8, (kind, v)
        assert (out["size_gradient"] + 1e-12 >= out["gradient"].abs()).all()


def test_the_plain_objective_moves_as_its_derivative_says():
    start = torch.tensor([0, 3, 3, 7])
    g = torch.Generator().manual_seed(2)
    new = -torch.rand(7, generator=g, dtype=torch.float64)
    kw = dict(adv=torch.tensor([1.0, 2.0, -0.5]), old=new + 0.1 * torch.randn(7, generator=g, dtype=torch.float64),
              ref=new + 0.1 * torch.randn(7, generator=g, dtype=torch.float64), beta=0.3, norm="rows")
    dlogp = ref.objective(start, new, **kw)[1]
    for j in range(7):
        up, down = new.clone(), new.clone()
        up[j] += 1e-6
        down[j] -= 1e-6
        d = (ref.objective(start, up, **kw)[0] - ref.objective(start, down, **kw)[0]) / 2e-6
        assert abs(d - dlogp[j]) <= 1e-8
