"""The policy update on token trajectories against 64 bits: log-probs, entropy, alternatives, divergences from a teacher's list, their
gradient, the objective of ragged rows; where masks, ties, strides and sizes can go wrong; refusals."""
import ctypes
import math

import pytest
import torch

from paper_2512_15347_b200 import binding as B
from tests import token_reference as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}     # results below: flushed, or a step of it
ALL = [torch.float32, torch.bfloat16, torch.float16]

# Errors in units of 2^-24, relative to the sums of absolute values that a result is made of.  A term 2^y: the argument is off by four
# roundings of y (difference, 1/T, c, product), which the sum sees weighted by p, so by at most 4 ln 2 (log2 V <= 20) = 56; the
# exponential itself by 4; additions in a thread by 16 a tile of at most 16 tiles where logits are not kept, 16 in all others
# here, and 14 in the trees.  So a sum is off by at most 56 + 4 + 16 * tiles + 14, its logarithm by as much in absolute terms.
SUM = 56 + 4 + 14


def tol_logp(tiles, spread, value):
    return U * (SUM + 16 * tiles + 4 * spread + 4 * abs(value) + 4)


def tiles_of(V, dtype):
    return -(-V // (8 * 512 * (4 if dtype == torch.float32 else 8))) + 1      # with one part, the worst


def make(R, V, dtype, seed, n_ids=1, n_list=0, masks=True, peaks=6.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn((R, V), generator=g, device="cuda") * (1 + 2 * torch.rand((R, 1), generator=g, device="cuda"))).to(dtype)
    c = dict(tau=0.5 + torch.rand(R, generator=g, device="cuda"), ids=torch.randint(0, V, (R, n_ids), generator=g, device="cuda", dtype=torch.int32))
    for j in range(n_ids):
        x.scatter_(1, c["ids"][:, j: j + 1].long(), (peaks * torch.rand((R, 1), generator=g, device="cuda")).to(dtype))
    if masks and R > 4:
        off = torch.rand(V, generator=g, device="cuda") < 0.7
        off[c["ids"][1].long()] = False
        x[1].masked_fill_(off, -math.inf)
        x[2].masked_fill_(off, torch.finfo(dtype).min)
        x[3] = -math.inf
        c["ids"][4, -1] = -1
    c["x"] = x
    if n_list:
        y = x.float() + torch.randn((R, V), generator=g, device="cuda")
        k = min(n_list, V)
        top = torch.log_softmax(torch.nan_to_num(y, neginf=-1e30), -1).topk(k, -1)
        ids = torch.full((R, n_list), -1, device="cuda", dtype=torch.int32)
        tl = torch.zeros((R, n_list), device="cuda")
        ids[:, :k], tl[:, :k] = top.indices.int(), top.values
        ids.masked_fill_(tl < -1e20, -1)
        if R > 4:
            ids[0, k // 2:] = -1
            ids[4] = -1                                            # an empty list
        c["list_ids"], c["list_logp"] = ids, tl
    c["dlogp"] = torch.randn((R, n_ids), generator=g, device="cuda")
    c["dentropy"] = torch.randn(R, generator=g, device="cuda")
    c["ddistill"] = torch.randn(R, generator=g, device="cuda")
    return c


def terms_of(c, kind="forward", n_top=0, ids=True, lists=True):
    return B.make_token_terms(temperature=c.get("tau"), ids=c["ids"] if ids else None, n_top=n_top, kind=kind,
                              teacher_ids=c.get("list_ids") if lists else None, teacher_logp=c.get("list_logp") if lists else None)


def reference(c, kind="forward", entropy=True, ids=True, lists=True):
    rows = []
    for r in range(c["x"].shape[0]):
        has = lists and "list_ids" in c
        rows.append(ref.row_terms(c["x"][r], float(c["tau"][r]) if c.get("tau") is not None else 1.0, c["ids"][r].tolist() if ids else (),
                                  c["list_ids"][r].tolist() if has else (), c["list_logp"][r].tolist() if has else (), kind,
                                  c["dlogp"][r].tolist() if ids else None, float(c["dentropy"][r]) if entropy else 0.0,
                                  float(c["ddistill"][r]) if has else 0.0))
    return rows


def outputs(R, c, n_top=0, lists=False):
    new = lambda *s: torch.full(s, math.nan, device="cuda")
    o = dict(logp=new(R, c["ids"].shape[1]), lse=new(R), entropy=new(R), saved=new(R, B.TOKEN_SAVED))
    if n_top:
        o.update(top_ids=torch.full((R, n_top), -7, device="cuda", dtype=torch.int32), top_logp=new(R, n_top))
    if lists:
        o["distill"] = new(R)
    return o


def close(got, want, tol, what):
    got, want = float(got), float(want)
    if want < -3.4028235e38:                        # the type's lowest logit over a temperature below 1: no number of 32 bits
        want = -math.inf
    if math.isinf(want) or math.isnan(want):
        assert got == want or (math.isnan(got) and math.isnan(want)), (what, got, want)
    else:
        assert abs(got - want) <= tol, (what, got, want, tol)


def check_forward(c, o, rows, n_top=0):
    V = c["x"].shape[1]
    tiles = tiles_of(V, c["x"].dtype)
    host = {k: v.cpu() for k, v in o.items()}
    for r, w in enumerate(rows):
        for j, lp in enumerate(w["logp"].tolist()):
            close(host["logp"][r, j], lp, tol_logp(tiles, float(w["spread"][j]), lp), ("logp", r, j))
        tau = float(c["tau"][r]) if c.get("tau") is not None else 1.0
        top = float(c["x"][r].double().max()) / tau
        if abs(w["lse"]) < 3e38:
            close(host["lse"][r], w["lse"], tol_logp(tiles, 0, abs(w["lse"]) + (abs(top) if math.isfinite(top) else 0)), ("lse", r))
        # ln 2 (log2 s0 - s1 / s0): each quotient's sums are off by SUM + 16 tiles, s1 once more by the product with y
        close(host["entropy"][r], w["entropy"], U * (SUM + 16 * tiles) * (1 + 3 * w["entropy"]) + 4 * U, ("entropy", r))
        if "distill" in host:
            close(host["distill"][r], w["distill"], U * (SUM + 16 * tiles + 40) * (w["size_distill"] + 1), ("distill", r))
        if n_top:
            at = ref.alternatives(c["x"][r], n_top).cpu()
            assert host["top_ids"][r].tolist() == at.tolist(), ("top_ids", r)
            for j, i in enumerate(at.tolist()):
                lp = -math.inf
                if i >= 0:
                    lp = float(c["x"][r, i].double()) / tau - w["lse"]
                close(host["top_logp"][r, j], lp, tol_logp(tiles, top - lp - w["lse"] if i >= 0 else 0, lp if i >= 0 else 0), ("top", r, j))


def check_gradient(c, got, rows):
    dtype, V = c["x"].dtype, c["x"].shape[1]
    tiles = tiles_of(V, dtype)
    for r, w in enumerate(rows):
        g = got[r].double()
        # a factor p_v is off by its own argument's roundings (4 |ln p|, at most 4 * 104 before it is 0) and by those of the sums
        tol = U * (2 * (SUM + 16 * tiles) + 4 * 104 + 40) * w["size_gradient"] + HALF_STEP[dtype] * w["gradient"].abs() * 1.01 + TINY[dtype]
        bad = ~((g - w["gradient"]).abs() <= tol)
        assert not bool(bad.any()), ("gradient", r, [(int(i), float(g[i]), float(w["gradient"][i]), float(tol[i])) for i in torch.nonzero(bad)[:4, 0]])


SIZES = [(1, 1), (5, 2), (6, 7), (6, 8), (6, 9), (7, 1000), (6, 4099), (40, 9001), (1, 32000), (6, 50001), (6, 131072)]


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("R,V", SIZES)
def test_forward_with_alternatives(dtype, R, V):
    n_top = min(V, 20)
    c = make(R, V, dtype, R + V, n_ids=3)
    o = outputs(R, c, n_top)
    B.token_forward(c["x"], terms_of(c, n_top=n_top), **o)
    check_forward(c, o, reference(c), n_top)


@pytest.mark.parametrize("kind", B.DISTILL_KINDS)
@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("R,V,k", [(1, 1, 1), (5, 3, 3), (6, 9, 4), (6, 1000, 10), (7, 5003, 64), (5, 33000, 256), (5, 131075, 100)])
def test_all_terms_in_one_pass_and_in_two(dtype, R, V, k, kind):
    c = make(R, V, dtype, 3 * R + V, n_ids=2, n_list=k)
    rows = reference(c, kind)
    t = terms_of(c, kind, n_top=min(V, 5))
    a, b = outputs(R, c, min(V, 5), True), outputs(R, c, min(V, 5), True)
    one, two = (torch.full_like(c["x"], 7) for _ in range(2))
    grads = {k: c[k] for k in ("dlogp", "dentropy", "ddistill")}
    B.token_forward_backward(c["x"], t, one, **a, **grads)
    check_forward(c, a, rows, min(V, 5))
    check_gradient(c, one, rows)
    B.token_forward(c["x"], t, **b)
    B.token_backward(c["x"], t, b["saved"], two, **grads)
    check_forward(c, b, rows, min(V, 5))
    check_gradient(c, two, rows)


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("V", [262147, 524288, 1048576])
def test_vocabularies_that_do_not_stay_in_registers(dtype, V):
    for kind in ("forward", "reverse_rest"):
        c = make(2, V, dtype, V, n_ids=1, n_list=30)
        rows = reference(c, kind)
        o, g = outputs(2, c, 40, True), torch.empty_like(c["x"])
        grads = {k: c[k] for k in ("dlogp", "dentropy", "ddistill")}
        B.token_forward_backward(c["x"], terms_of(c, kind, n_top=40), g, **o, **grads)
        check_forward(c, o, rows, 40)
        check_gradient(c, g, rows)
        g.zero_()
        B.token_backward(c["x"], terms_of(c, kind), o["saved"], g, **grads)
        check_gradient(c, g, rows)


@pytest.mark.parametrize("R", [2, 30, 80, 160, 400, 700])
def test_rows_are_cut_by_how_many_there_are(R):
    """The same rows, alone and among others, give the same results up to the order of additions, and bit for bit in a second call."""
    V = 20011
    c = make(R, V, torch.bfloat16, R, n_list=16)
    t = terms_of(c, "forward_rest", n_top=8)
    o, again = outputs(R, c, 8, True), outputs(R, c, 8, True)
    B.token_forward(c["x"], t, **o)
    B.token_forward(c["x"], t, **again)
    for k in o:
        assert torch.equal(o[k], again[k]) or k == "saved"
    few = {k: v[:6] for k, v in c.items()}
    check_forward(few, {k: v[:6] for k, v in o.items()}, reference(few, "forward_rest"), 8)


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("off,pitch", [(0, 9008), (1, 9001), (3, 9013), (5, 9002), (8, 9016)])
def test_strides_and_in_place(dtype, off, pitch):
    R, V = 6, 9001
    c = make(R, V, dtype, off + pitch, n_ids=2, n_list=20)
    for kind in ("forward", "reverse_rest"):
        rows = reference(c, kind)
        grads = {k: c[k] for k in ("dlogp", "dentropy", "ddistill")}
        room = torch.full((R * pitch + 16,), 5.0, device="cuda", dtype=dtype)
        x = room[off: off + R * pitch].view(R, pitch)[:, :V]
        x.copy_(c["x"])
        t, o = terms_of(c, kind, n_top=9), outputs(R, c, 9, True)
        out = torch.full((R, V + 2), 3.0, device="cuda", dtype=dtype)           # another alignment than the logits'
        B.token_forward_backward(x, t, out[:, 1: V + 1], **o, **grads)
        check_forward(c, o, rows, 9)
        check_gradient(c, out[:, 1: V + 1], rows)
        assert (out[:, 0] == 3).all() and (out[:, V + 1] == 3).all()
        B.token_backward(x, t, o["saved"], out[:, 1: V + 1], **grads)
        check_gradient(c, out[:, 1: V + 1], rows)
        B.token_backward(x, t, o["saved"], x, **grads)
        check_gradient(c, x, rows)
        x.copy_(c["x"])
        B.token_forward_backward(x, t, x, **o, **grads)
        check_gradient(c, x, rows)
        rest = torch.ones(room.numel(), dtype=torch.bool, device="cuda")
        for r in range(R):
            rest[off + r * pitch: off + r * pitch + V] = False
        assert (room[rest] == 5).all()


@pytest.mark.parametrize("parts", [1, 4])
def test_in_place_with_rows_that_are_cut(parts):
    R, V = (400, 1000) if parts == 1 else (3, 131072)
    c = make(R, V, torch.bfloat16, parts, n_ids=3, n_list=50)
    few = {k: v[:6] for k, v in c.items()}
    rows = reference(few, "forward_rest")
    grads = {k: c[k] for k in ("dlogp", "dentropy", "ddistill")}
    x = c["x"].clone()
    o = outputs(R, c, 0, True)
    B.token_forward_backward(x, terms_of(c, "forward_rest"), x, **o, **grads)
    check_gradient(few, x[:6], rows)
    x = c["x"].clone()
    B.token_backward(x, terms_of(c, "forward_rest"), o["saved"], x, **grads)
    check_gradient(few, x[:6], rows)


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("V", [100, 1000, 5000, 40000, 140000])
def test_alternatives_of_rows_full_of_ties(dtype, V):
    """Equal logits throughout, two values, ascending, descending, few allowed, none but zeros of both signs."""
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.zeros((8, V), device="cuda", dtype=dtype)
    x[1] = (torch.rand(V, generator=g, device="cuda") < 0.4).to(dtype)
    x[2] = torch.linspace(-4, 4, V, device="cuda").to(dtype)
    x[3] = torch.linspace(4, -4, V, device="cuda").to(dtype)
    x[4] = -math.inf
    x[4, torch.randperm(V, generator=g, device="cuda")[:11]] = 1.5
    x[5] = torch.where(torch.rand(V, generator=g, device="cuda") < 0.5, -0.0, 0.0).to(dtype)
    x[6] = torch.finfo(dtype).min
    x[7] = torch.randint(-3, 4, (V,), generator=g, device="cuda").to(dtype)
    for n in (1, 7, 100, 128):
        n = min(n, V)
        for lists in (False, True):
            ids, lp = torch.empty((8, n), device="cuda", dtype=torch.int32), torch.empty((8, n), device="cuda")
            more = dict(teacher_ids=torch.arange(0, 32, device="cuda", dtype=torch.int32).repeat(8, 1),
                        teacher_logp=torch.full((8, 32), -4.0, device="cuda"), kind="forward_rest") if lists else {}
            B.token_forward(x, B.make_token_terms(n_top=n, **more), top_ids=ids, top_logp=lp)
            for r in range(8):
                assert ids[r].tolist() == ref.alternatives(x[r], n).tolist(), (r, n, lists)
            # equal logits: -ln V, off by a sum of V equal terms
            assert (lp[0] + math.log(V)).abs().max() <= U * (SUM + 16 * tiles_of(V, dtype) + 8 * math.log(V))
            assert (lp[6] + math.log(V)).abs().max() <= U * (SUM + 16 * tiles_of(V, dtype) + 8 * math.log(V))


@pytest.mark.parametrize("dtype", ALL)
def test_nan_and_infinity_stay_in_their_rows(dtype):
    R, V = 6, 3001
    c = make(R, V, dtype, 4, n_list=8, masks=False)
    c["x"][1, 7] = math.nan
    c["x"][2, 2999] = math.inf
    c["x"][4] = math.nan
    for kind in B.DISTILL_KINDS:
        o, g = outputs(R, c, 5, True), torch.empty_like(c["x"])
        grads = {k: c[k] for k in ("dlogp", "dentropy", "ddistill")}
        t = terms_of(c, kind, n_top=5)
        B.token_forward_backward(c["x"], t, g, **o, **grads)
        for r in (1, 2, 4):
            assert all(torch.isnan(o[k][r]).all() for k in ("logp", "lse", "entropy", "distill")) and torch.isnan(g[r]).all()
            assert ((o["top_ids"][r] >= -1) & (o["top_ids"][r] < V)).all()
        good = [0, 3, 5]
        few = {k: v[good] for k, v in c.items()}
        rows = reference(few, kind)
        check_forward(few, {k: v[good] for k, v in o.items()}, rows, 5)
        check_gradient(few, g[good], rows)
        B.token_backward(c["x"], t, o["saved"], g, **grads)
        check_gradient(few, g[good], rows)
        assert torch.isnan(g[1]).all()


def test_given_tokens_twice_beside_and_on_the_list():
    R, V, dtype = 5, 700, torch.float32
    c = make(R, V, dtype, 5, n_ids=7, n_list=12, masks=False)
    c["ids"][:, 1] = c["ids"][:, 0]
    c["ids"][:, 2] = c["ids"][:, 0]
    c["ids"][:, 4] = c["list_ids"][:, 3].clamp(min=0)
    c["ids"][:, 5] = c["list_ids"][:, 3].clamp(min=0)
    c["ids"][2, 6] = V                                             # outside
    c["ids"][3, 6] = -2 ** 31
    c["list_ids"][1, 5] = c["list_ids"][1, 2]                      # the last one counts
    c["list_logp"][1, 5] = -1.25
    c["list_logp"][2, 4] = -math.inf
    c["list_ids"][2, 6] = V + 5
    for kind in B.DISTILL_KINDS:
        rows = reference(c, kind)
        o, g, h = outputs(R, c, 0, True), torch.empty_like(c["x"]), torch.empty_like(c["x"])
        grads = {k: c[k] for k in ("dlogp", "dentropy", "ddistill")}
        B.token_forward_backward(c["x"], terms_of(c, kind), g, **o, **grads)
        check_forward(c, o, rows)
        check_gradient(c, g, rows)
        B.token_backward(c["x"], terms_of(c, kind), o["saved"], h, **grads)
        check_gradient(c, h, rows)


@pytest.mark.parametrize("kind", B.DISTILL_KINDS)
@pytest.mark.parametrize("n_list,different", [(30, 9), (64, 40), (201, 70), (256, 3)])
def test_lists_with_the_same_ids_again(kind, n_list, different):
    R, V = 4, 5003
    c = make(R, V, torch.float32, 14, n_list=n_list, masks=False)
    g = torch.Generator(device="cuda").manual_seed(n_list)
    some = torch.randint(0, V, (different,), generator=g, device="cuda", dtype=torch.int32)
    c["list_ids"] = some[torch.randint(0, different, (R, n_list), generator=g, device="cuda")].contiguous()
    c["list_ids"][1, ::3] = -1
    c["list_logp"] = -math.log(n_list) - torch.rand((R, n_list), generator=g, device="cuda")
    rows = reference(c, kind)
    o, both, back = outputs(R, c, 0, True), torch.empty_like(c["x"]), torch.empty_like(c["x"])
    t, grads = terms_of(c, kind), {k: c[k] for k in ("dlogp", "dentropy", "ddistill")}
    B.token_forward_backward(c["x"], t, both, **o, **grads)
    check_forward(c, o, rows)
    check_gradient(c, both, rows)
    o = outputs(R, c, 0, True)
    B.token_forward(c["x"], t, **o)
    check_forward(c, o, rows)
    B.token_backward(c["x"], t, o["saved"], back, **grads)
    check_gradient(c, back, rows)


def test_256_given_tokens_and_256_listed():
    R, V = 5, 2000
    c = make(R, V, torch.float32, 6, n_ids=256, n_list=256)
    for kind in B.DISTILL_KINDS:
        rows = reference(c, kind)
        o, g = outputs(R, c, 128, True), torch.empty_like(c["x"])
        B.token_forward_backward(c["x"], terms_of(c, kind, n_top=128), g, **o, **{k: c[k] for k in ("dlogp", "dentropy", "ddistill")})
        check_forward(c, o, rows, 128)
        check_gradient(c, g, rows)


@pytest.mark.parametrize("gap", [20.0, 60.0, 110.0, 300.0])
@pytest.mark.parametrize("kind", ["forward_rest", "reverse_rest"])
def test_mass_outside_the_list_far_below_it(kind, gap):
    """The list holds all but exp(-gap): 1 - (its mass) is 0 in 32 bits, the bucket's logarithm is not."""
    V = 4000
    x = torch.randn(1, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    x[0, :5] += gap
    c = dict(x=x, ids=torch.tensor([[17]], device="cuda", dtype=torch.int32), list_ids=torch.arange(5, device="cuda", dtype=torch.int32)[None],
             list_logp=torch.full((1, 5), math.log(0.19), device="cuda"), dlogp=torch.ones(1, 1, device="cuda"), dentropy=torch.ones(1, device="cuda"),
             ddistill=torch.ones(1, device="cuda"))
    rows = reference(c, kind)
    o, g = outputs(1, c, 0, True), torch.empty_like(x)
    B.token_forward_backward(x, terms_of(c, kind), g, **o, **{k: c[k] for k in ("dlogp", "dentropy", "ddistill")})
    check_forward(c, o, rows)
    check_gradient(c, g, rows)


def test_list_that_covers_everything_and_a_mask_that_does():
    c = dict(x=torch.tensor([[0.5, -1.0, 2.0], [0.5, -math.inf, -math.inf]], device="cuda"),
             ids=torch.tensor([[0], [0]], device="cuda", dtype=torch.int32),
             list_ids=torch.tensor([[0, 1, 2], [0, -1, -1]], device="cuda", dtype=torch.int32),
             list_logp=torch.tensor([[-1.0, -1.5, -0.9], [-0.1, 0, 0]], device="cuda"), dlogp=torch.zeros(2, 1, device="cuda"),
             dentropy=torch.zeros(2, device="cuda"), ddistill=torch.tensor([1.0, -2.0], device="cuda"))
    for kind in B.DISTILL_KINDS:
        rows = reference(c, kind)
        o, g = outputs(2, c, 0, True), torch.empty_like(c["x"])
        B.token_forward_backward(c["x"], terms_of(c, kind), g, **o, **{k: c[k] for k in ("dlogp", "dentropy", "ddistill")})
        check_forward(c, o, rows)
        check_gradient(c, g, rows)


def test_listed_token_that_the_policy_masks():
    c = make(2, 600, torch.float32, 9, n_list=6, masks=False)
    c["x"][0, int(c["list_ids"][0, 2])] = -math.inf
    for kind in B.DISTILL_KINDS:
        rows = reference(c, kind)
        assert (rows[0]["distill"] == math.inf) == (kind != "reverse_rest")
        o, g = outputs(2, c, 0, True), torch.empty_like(c["x"])
        B.token_forward_backward(c["x"], terms_of(c, kind), g, **o, **{k: c[k] for k in ("dlogp", "dentropy", "ddistill")})
        check_forward(c, o, rows)
        check_gradient(c, g, rows)


@pytest.mark.parametrize("only", ["logp", "entropy", "distill", "top"])
def test_terms_one_by_one(only):
    R, V = 5, 10007
    c = make(R, V, torch.bfloat16, 11, n_list=20)
    ids, lists, ent = only == "logp", only == "distill", only == "entropy"
    rows = reference(c, "reverse_rest", entropy=ent, ids=ids, lists=lists)
    t = terms_of(c, "reverse_rest", n_top=6 if only == "top" else 0, ids=ids, lists=lists)
    grads = dict(dlogp=c["dlogp"]) if ids else dict(dentropy=c["dentropy"]) if ent else dict(ddistill=c["ddistill"]) if lists else {}
    saved, g, h = torch.empty(R, B.TOKEN_SAVED, device="cuda"), torch.empty_like(c["x"]), torch.empty_like(c["x"])
    more = {}
    if only == "top":
        more = dict(top_ids=torch.empty((R, 6), device="cuda", dtype=torch.int32))
    B.token_forward_backward(c["x"], t, g, saved=saved, **grads, **more)
    check_gradient(c, g, rows)
    B.token_backward(c["x"], t, saved, h, **grads)
    check_gradient(c, h, rows)
    B.token_forward_backward(c["x"], t, g, **grads)                # without anything of the forward pass
    check_gradient(c, g, rows)


def test_gradient_against_differences():
    """Central differences of the forward pass's own results.  With a step h = 2^-5 they are off by h^2 / 6 times the third derivative
    (of ln p, the entropy and the divergences: below 6 times 1 + their largest logarithm, 12 here) and by twice the results' error over 2 h."""
    V, h = 50, 2.0 ** -5
    for kind in B.DISTILL_KINDS:
        c = make(1, V, torch.float32, 21, n_ids=2, n_list=6, masks=False, peaks=2.0)
        c["tau"] = torch.ones(1, device="cuda")
        g = torch.empty_like(c["x"])
        B.token_forward_backward(c["x"], terms_of(c, kind), g, **{k: c[k] for k in ("dlogp", "dentropy", "ddistill")})
        x = c["x"].repeat(2 * V, 1)
        i = torch.arange(V, device="cuda")
        x[i, i] += h
        x[V + i, i] -= h
        many = dict(x=x, tau=None, **{k: c[k].repeat(2 * V, 1) for k in ("ids", "list_ids", "list_logp")})
        o = outputs(2 * V, many, 0, True)
        B.token_forward(x, terms_of(many, kind), **o)
        f = (o["logp"] @ c["dlogp"][0] + o["entropy"] * c["dentropy"] + o["distill"] * c["ddistill"]).double()
        d = (f[:V] - f[V:]) / (2 * h)
        size = float(c["dlogp"].abs().sum() + c["dentropy"].abs().sum() + c["ddistill"].abs().sum())
        tol = h * h * 12 * size + 2 * 200 * U * 12 * size / (2 * h)
        assert (d - g[0]).abs().max() <= tol, (kind, float((d - g[0]).abs().max()), tol)


@pytest.mark.parametrize("V,off", [(5001, 0), (40003, 0), (40003, 1), (131072, 0)])
def test_rows_without_derivatives_are_zero_and_not_read(V, off):
    R = 6
    c = make(R, V, torch.bfloat16, 12, n_list=10, masks=False)
    t, o = terms_of(c, "forward_rest"), outputs(R, c, 0, True)
    B.token_forward(c["x"], t, **o)
    c["dlogp"][1:3] = 0
    c["dentropy"][1:3] = 0
    c["ddistill"][1:3] = 0
    rows = reference(c, "forward_rest")
    x = c["x"].clone()
    x[1] = math.nan                                                # no longer looked at
    g = torch.full((R, V + off), 9.0, device="cuda", dtype=torch.bfloat16)[:, off:]
    B.token_backward(x, t, o["saved"], g, **{k: c[k] for k in ("dlogp", "dentropy", "ddistill")})
    assert (g[1:3] == 0).all()
    check_gradient(c, g, rows)


@pytest.mark.parametrize("kind", B.DISTILL_KINDS)
@pytest.mark.parametrize("V,off", [(7, 0), (5001, 0), (40003, 1), (131072, 0)])
def test_padding_rows_of_any_content_have_no_gradient(V, off, kind):
    R = 6
    c = make(R, V, torch.bfloat16, 13, n_list=4, masks=False)
    c["x"][1], c["x"][2, -1], c["x"][3, 0] = math.nan, math.inf, math.nan
    for r in (1, 2, 3):
        c["ids"][r], c["dlogp"][r], c["dentropy"][r], c["ddistill"][r] = -1, 5.0, 0, 0       # what padding's dlogp holds plays no part
    c["list_logp"][5, 1], c["ddistill"][5] = math.nan, 0                                     # a teacher's list without weight
    t, o, grads = terms_of(c, kind), outputs(R, c, 0, True), {k: c[k] for k in ("dlogp", "dentropy", "ddistill")}
    both, back = (torch.full((R, V + off), 9.0, device="cuda", dtype=torch.bfloat16)[:, off:] for _ in range(2))
    B.token_forward_backward(c["x"], t, both, **o, **grads)
    B.token_backward(c["x"], t, o["saved"], back, **grads)
    c["list_logp"][5, 1] = -1.0
    good = [0, 4, 5]
    rows = reference({k: v[good] for k, v in c.items()}, kind)
    for g in (both, back):
        assert (g[1:4] == 0).all()
        check_gradient({k: v[good] for k, v in c.items()}, g[good], rows)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_logits_next_to_the_types_ends(dtype):
    """Logits of +-3e38, whose products with log2(e) / T have no 32-bit value: alone, beside ordinary ones, on the list."""
    R, V = 7, 20011
    c = make(R, V, dtype, 31, n_ids=2, n_list=6, masks=False)
    big = torch.finfo(dtype).max
    c["x"][0, ::3] = big
    c["x"][1] = -big
    c["x"][2, 5000:] = -big
    c["x"][3, int(c["list_ids"][3, 0])] = big
    c["x"][4] = big
    c["x"][5, 1:] = -big
    for kind in B.DISTILL_KINDS:
        rows = reference(c, kind)
        o, g, h = outputs(R, c, 3, True), torch.empty_like(c["x"]), torch.empty_like(c["x"])
        grads = {k: c[k] for k in ("dlogp", "dentropy", "ddistill")}
        B.token_forward_backward(c["x"], terms_of(c, kind, n_top=3), g, **o, **grads)
        check_gradient(c, g, rows)
        B.token_backward(c["x"], terms_of(c, kind), o["saved"], h, **grads)
        check_gradient(c, h, rows)
        for r in (1, 4):                                           # all equal
            assert abs(float(o["entropy"][r]) - math.log(V)) <= U * (SUM + 16 * tiles_of(V, dtype)) * (1 + 3 * math.log(V))
        for r in range(R):
            assert o["top_ids"][r].tolist() == ref.alternatives(c["x"][r], 3).tolist()


def test_rows_more_than_2_to_the_31_elements_apart():
    """Rows at both ends of a buffer of 8 GB."""
    V, pitch = 5003, 2 ** 31 + 24
    c = make(3, V, torch.bfloat16, 41, n_list=5, masks=False)
    room = torch.empty(2 * pitch + V, device="cuda", dtype=torch.bfloat16)
    x = room.as_strided((3, V), (pitch, 1))
    x.copy_(c["x"])
    rows = reference(c, "forward_rest")
    o, g = outputs(3, c, 4, True), torch.empty((3, V), device="cuda", dtype=torch.bfloat16)
    grads = {k: c[k] for k in ("dlogp", "dentropy", "ddistill")}
    B.token_forward_backward(x, terms_of(c, "forward_rest", n_top=4), g, **o, **grads)
    check_forward(c, o, rows, 4)
    check_gradient(c, g, rows)
    B.token_backward(x, terms_of(c, "forward_rest"), o["saved"], x, **grads)
    check_gradient(c, x, rows)
    del room, x
    torch.cuda.empty_cache()


def test_calls_on_a_stream_that_is_given():
    c = make(5, 9001, torch.float16, 42, n_list=5)
    rows = reference(c, "forward")
    side = torch.cuda.Stream()
    o, g = outputs(5, c, 4, True), torch.empty_like(c["x"])
    side.wait_stream(torch.cuda.current_stream())
    B.token_forward_backward(c["x"], terms_of(c, "forward", n_top=4), g, **o, **{k: c[k] for k in ("dlogp", "dentropy", "ddistill")}, stream=side)
    side.synchronize()
    check_forward(c, o, rows, 4)
    check_gradient(c, g, rows)


# ------------------------------------------------------------------------------------ the objective

def objective_case(lens, seed, head=0, tail=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, R = sum(lens) + head + tail, len(lens)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    start = torch.tensor([head] + [head + sum(lens[: i + 1]) for i in range(R)], device="cuda", dtype=torch.int32)
    new = -2 * torch.rand(n, generator=g, device="cuda")
    return dict(start=start, new=new, adv=rnd(R), old=new + 0.3 * rnd(n), ref=new + 0.05 * rnd(n), entropy=rnd(n).abs(), distill=rnd(n).abs())


def run_objective(c, use=("old", "ref", "entropy", "distill"), inplace=False, **kw):
    n = c["new"].numel()
    new = lambda k: torch.full((k,), math.nan, device="cuda")
    o = dict(objective=new(1), dlogp=new(n), weight=new(n), ratio=new(n), stats=new(B.TOKEN_STATS))
    ws = torch.zeros(B.token_objective_workspace_bytes(n), device="cuda", dtype=torch.uint8)
    status = torch.zeros(1, device="cuda", dtype=torch.int32)
    lp = c["new"].clone()
    if inplace:
        o["dlogp"] = lp
    names = dict(old="logp_old", ref="logp_ref", entropy="entropy", distill="distill")
    B.token_objective(c["start"], lp, c["adv"], o["objective"], o["dlogp"], ws, weight=o["weight"], ratio=o["ratio"], stats=o["stats"],
                      status=status, **{names[k]: c[k] for k in use}, **kw)
    assert int(ws[:4096].sum()) == 0
    return o, status


def check_objective(c, o, use, **kw):
    # 64 bits inside: results are off by their rounding to 32, sums relative to the sum of their terms' sizes
    kw = {k: ctypes.c_float(v).value if isinstance(v, float) else v for k, v in kw.items()}      # as the call takes them
    J, dlogp, weight, ratio, stats = ref.objective(c["start"], c["new"], c["adv"], **{k: c[k] for k in use}, **kw)
    for name, want in (("dlogp", dlogp), ("weight", weight), ("ratio", ratio), ("stats", stats)):
        got, want = o[name].double().cpu(), torch.tensor(want, dtype=torch.float64)
        assert ((got - want).abs() <= U * 1.01 * want.abs() + 1e-13).all(), (name, got, want)
    assert abs(float(o["objective"]) - J) <= U * 1.01 * abs(J) + 1e-12


KW = dict(clip_low=0.2, clip_high=0.28, beta=0.04, entropy_coef=0.01, distill_coef=0.5, scale=0.25)


@pytest.mark.parametrize("norm", B.TOKEN_NORMS)
@pytest.mark.parametrize("lens", [[1], [0, 3, 0, 0, 5], [0, 0], [700, 1, 0, 2000, 33], [5] * 400, list(range(120))])
def test_objective_of_ragged_rows(lens, norm):
    for use in (("old", "ref", "entropy", "distill"), ("old",), (), ("ref",)):
        for head, tail in ((0, 0), (3, 9)):
            c = objective_case(lens, len(lens) + head, head, tail)
            o, status = run_objective(c, use, norm=norm, **KW)
            check_objective(c, o, use, norm=norm, **KW)
            assert int(status) == 0
            again, _ = run_objective(c, use, inplace=True, norm=norm, **KW)
            assert all(torch.equal(o[k], again[k]) for k in o)


def test_objective_at_the_clip_range_and_of_no_advantage():
    c = objective_case([8], 3)
    lo, hi = 1 - 0.2, 1 + 0.28
    r = torch.tensor([lo, hi, 1.0, 0.5, 2.0, lo * 0.999, hi * 1.001, 1.0], dtype=torch.float64)
    c["new"] = torch.zeros(8, device="cuda")
    c["old"] = (-torch.log(r)).float().cuda()
    for a in (1.0, -1.0, 0.0):
        c["adv"] = torch.tensor([a], device="cuda")
        o, _ = run_objective(c, ("old",), **KW)
        check_objective(c, o, ("old",), **KW)


def test_objective_with_starts_that_do_not_ascend():
    c = objective_case([5, 6, 7], 8)
    for bad in ([0, 11, 5, 18], [-1, 5, 11, 18], [0, 5, 11, 2 ** 31 - 1], [18, 11, 5, 0]):
        c["start"] = torch.tensor(bad, device="cuda", dtype=torch.int32)
        o, status = run_objective(c, ("old",), **KW)
        assert int(status) == 4
        with pytest.raises(B.PgError) as e:
            B.kv_status(status)
        assert e.value.code == B.EINDEX
    c = objective_case([5, 6, 7], 8)
    o, status = run_objective(c, ("old",), **KW)
    check_objective(c, o, ("old",), **KW)


def test_objective_of_many_tokens():
    """More chunks than slots of the workspace: several chunks a CTA."""
    n, R = 4096 * 1024 * 2 + 77, 3
    g = torch.Generator(device="cuda").manual_seed(1)
    start = torch.tensor([0, 1000003, 1000003, n], device="cuda", dtype=torch.int32)
    new = torch.randn(n, generator=g, device="cuda")
    old = new + 0.2 * torch.randn(n, generator=g, device="cuda")
    c = dict(start=start, new=new, old=old, adv=torch.tensor([1.0, 5.0, -0.5], device="cuda"))
    o, _ = run_objective(c, ("old",), norm="tokens")
    a = torch.full((n,), -0.5, device="cuda", dtype=torch.float64)
    a[:1000003] = 1
    r = torch.exp(new.double() - old.double())
    free, held = r * a, r.clamp(1 - B.TokenBatch(clip_low=0.2).clip_low, 1 + B.TokenBatch(clip_high=0.2).clip_high) * a
    surr = torch.minimum(free, held)
    # 64-bit sums of n terms in another order
    assert abs(float(o["objective"]) - float(surr.mean())) <= U * abs(float(surr.mean())) + 1e-9
    want = torch.where(free <= held, free, torch.zeros_like(free)) / n
    assert ((o["dlogp"].double() - want).abs() <= U * 1.01 * want.abs()).all()


# ------------------------------------------------------------------------------------ together

def test_update_step_in_a_graph_and_on_two_streams():
    """Forward, objective and backward as a training step runs them: eager, captured and replayed on new inputs, and two at once on
    streams of their own."""
    V, lens = 6007, [5, 0, 11, 3]
    n = sum(lens)

    def state(seed):
        c = make(n, V, torch.bfloat16, seed, n_list=12, masks=False)
        c.update(objective_case(lens, seed))
        c["old"] = torch.full((n,), -3.0, device="cuda")
        o = outputs(n, c, 0, True)
        s = dict(c=c, o=o, t=terms_of(c, "reverse_rest"), g=torch.empty_like(c["x"]), dlogp=torch.empty(n, device="cuda"),
                 weight=torch.empty(n, device="cuda"), J=torch.empty(1, device="cuda"),
                 ws=torch.zeros(B.token_objective_workspace_bytes(n), device="cuda", dtype=torch.uint8))
        return s

    def step(s):
        c, o = s["c"], s["o"]
        B.token_forward(c["x"], s["t"], **o)
        B.token_objective(c["start"], o["logp"].view(-1), c["adv"], s["J"], s["dlogp"], s["ws"], logp_old=c["old"], entropy=o["entropy"],
                          distill=o["distill"], weight=s["weight"], entropy_coef=0.01, distill_coef=0.5)
        B.token_backward(c["x"], s["t"], o["saved"], s["g"], dlogp=s["dlogp"].view(-1, 1), dentropy=s["weight"], entropy_scale=0.01,
                         ddistill=s["weight"], distill_scale=-0.5)

    def check(s):
        c = s["c"]
        kw = dict(entropy_coef=ctypes.c_float(0.01).value, distill_coef=0.5)
        J, dlogp, weight, _, _ = ref.objective(c["start"], s["o"]["logp"].view(-1), c["adv"], old=c["old"], entropy=s["o"]["entropy"],
                                               distill=s["o"]["distill"], **kw)
        assert abs(float(s["J"]) - J) <= 2 * U * abs(J) + 1e-12
        c["dlogp"], w = torch.tensor(dlogp, device="cuda")[:, None], torch.tensor(weight, device="cuda")
        c["dentropy"], c["ddistill"] = 0.01 * w, -0.5 * w
        check_gradient(c, s["g"], reference(c, "reverse_rest"))

    a, b = state(1), state(2)
    step(a)
    check(a)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(a)
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        step(a)
    fresh = make(n, V, torch.bfloat16, 77, masks=False)
    a["c"]["x"].copy_(fresh["x"])
    a["g"].zero_()
    graph.replay()
    torch.cuda.synchronize()
    check(a)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for s, st in zip((a, b), streams):
            with torch.cuda.stream(st):
                s["g"].fill_(3)
                step(s)
    torch.cuda.synchronize()
    check(a)
    check(b)


# ------------------------------------------------------------------------------------ refusals

def test_refusals_of_the_binding():
    x = torch.zeros((4, 100), device="cuda")
    ids = torch.zeros((4, 2), device="cuda", dtype=torch.int32)
    tl = torch.zeros((4, 3), device="cuda")
    tids = torch.zeros((4, 3), device="cuda", dtype=torch.int32)
    for bad in (dict(ids=ids.long()), dict(ids=ids.cpu()), dict(ids=torch.zeros((4, 257), device="cuda", dtype=torch.int32)),
                dict(teacher_ids=tids), dict(teacher_logp=tl), dict(teacher_ids=tids, teacher_logp=tl[:, :2]),
                dict(teacher_ids=tids, teacher_logp=tl.double()), dict(n_top=129), dict(n_top=-1), dict(kind="backward"),
                dict(temperature=torch.ones(4, 1, device="cuda")), dict(temperature=torch.ones(4, device="cuda").double()),
                dict(temperature=torch.ones(3, device="cuda"), ids=ids), dict(ids=ids.t()[:, :2].t())):
        if "ids" in bad and bad["ids"].is_contiguous() and bad["ids"].dtype is torch.int32 and bad["ids"].is_cuda and len(bad) == 1 and bad["ids"].shape[1] == 2:
            continue
        with pytest.raises(ValueError):
            B.make_token_terms(**bad)
    t = B.make_token_terms(ids=ids, n_top=3, teacher_ids=tids, teacher_logp=tl)
    f = lambda *s: torch.empty(s, device="cuda")
    for bad in (dict(logp=f(4, 3)), dict(logp=f(4, 2).half()), dict(logp=f(4, 2).cpu()), dict(lse=f(5)), dict(entropy=f(8)[::2]),
                dict(top_ids=f(4, 3)), dict(top_logp=f(4, 3)), dict(distill=f(3)), dict(saved=f(4, 11))):
        with pytest.raises(ValueError):
            B.token_forward(x, t, **bad)
    none = B.make_token_terms()
    for bad in (dict(logp=f(4, 2)), dict(distill=f(4)), dict(top_ids=ids)):
        with pytest.raises(ValueError):
            B.token_forward(x, none, **bad)
    saved, g = f(4, B.TOKEN_SAVED), f(4, 100)
    for logits in (x.double(), x.cpu(), x.t(), x[:1].expand(4, 100), x[:3], x[0]):
        with pytest.raises(ValueError):
            B.token_forward(logits, t, lse=f(4))
    for out in (g.half(), g[:, :50], g.cpu(), g.t().contiguous().t()):
        with pytest.raises(ValueError):
            B.token_backward(x, t, saved, out, dlogp=f(4, 2))
        with pytest.raises(ValueError):
            B.token_forward_backward(x, t, out, dlogp=f(4, 2))
    for bad in (dict(dlogp=f(4)), dict(dentropy=f(4, 2)), dict(ddistill=f(4).double())):
        with pytest.raises(ValueError):
            B.token_backward(x, t, saved, g, **bad)
    with pytest.raises(ValueError):
        B.token_backward(x, none, saved, g, dlogp=f(4, 2))
    with pytest.raises(B.PgError):
        B.token_forward(x[:, :2], t, lse=f(4))                      # more alternatives than tokens
    start, adv, lp = torch.zeros(5, device="cuda", dtype=torch.int32), f(4), f(9)
    ws = torch.zeros(B.token_objective_workspace_bytes(9), device="cuda", dtype=torch.uint8)
    good = dict(start=start, logp_new=lp, adv=adv, objective=f(1), dlogp=f(9), workspace=ws)
    B.token_objective(**good)
    for bad in (dict(start=start.long()), dict(adv=f(3)), dict(dlogp=f(8)), dict(objective=f(2)), dict(logp_old=f(8)), dict(workspace=ws.cpu()),
                dict(norm="mean"), dict(logp_new=lp.cpu()), dict(stats=f(4)), dict(weight=f(9).half())):
        with pytest.raises(ValueError):
            B.token_objective(**{**good, **bad})
    for bad in (dict(clip_low=-0.1), dict(clip_low=1.5), dict(clip_high=-1.0), dict(clip_high=math.nan), dict(workspace=ws[:64])):
        with pytest.raises(B.PgError) as e:
            B.token_objective(**{**good, **bad})
        assert e.value.code == B.EINVAL


def test_nothing_to_do():
    x = torch.zeros((0, 100), device="cuda")
    t = B.make_token_terms()
    B.token_forward(x, t, lse=torch.empty(0, device="cuda"))
    B.token_forward_backward(x, t, x)
    y = torch.randn(3, 10, device="cuda")
    B.token_forward(y, t)
    ws = torch.zeros(B.token_objective_workspace_bytes(0), device="cuda", dtype=torch.uint8)
    for rows in (0, 2):
        J, none = torch.ones(1, device="cuda"), torch.empty(0, device="cuda")
        B.token_objective(torch.zeros(rows + 1, device="cuda", dtype=torch.int32), none, torch.ones(rows, device="cuda"), J, none, ws)
        assert float(J) == 0.0
