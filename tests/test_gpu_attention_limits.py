"""Attention where numbers, lengths and masks meet the ends of what they may be: large biases and scores, Inf and NaN beside rows that
see nothing and behind a sequence's states, numbers of unequal size in one head."""
import math

import pytest
import torch

import paper_2006_10901_amd as spdl
from tests.attention_util import Case, causal, reference, sparse_rows
from tests.gpu_util import TOL_F16, TOL_F32

pytestmark = pytest.mark.gpu

TYPES = ["f32", "f16"]


def step(case):
    case.prepare()
    case.forward()
    case.backward()
    torch.cuda.synchronize()
    return {name: t.cpu().double() for name, t in case.results().items()}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,k,span", [(1, 90, 16), (40, 70, 16), (40, 2050, 128), (130, 200, 0), (33, 40, 40)])
@pytest.mark.parametrize("lengths", [None, [35, 29]])
def test_a_large_bias_beside_rows_that_are_not_there(dtype, m, k, span, lengths):
    """exp(100) is more than fp32 holds: lanes behind the last query, whose products are 0, must not have such weights.
    Weights count to 2^-39 of a row's largest, dS to 2^-36 of a block's, so that those of exp(-100) are lost: each of the terms that a result adds up, at most
    2 max(m, k) of them (dtable: m k), may be off by 2^-36 times the most that it multiplies a weight by."""
    case = Case(dtype, batch=2, heads=3, m=m, k=k, d=32, buckets=8, span=span, lengths=lengths, seed=m)
    case.table[0] = 100.0
    case.table[1, ::2] = 100.0
    got = step(case)
    want = reference(case.Q, case.K, case.V, case.scale, case.lengths, case.positions, case.seen, case.bucket_of, case.table, case.dO)
    Q, K, V, dO = (float(t.nan_to_num().abs().max()) for t in (case.Q, case.K, case.V, case.dO))
    slope = 2 * 32 * dO * V                              # the most that dP - D can be
    more = {"O": 2 * max(m, k) * V, "dV": 2 * max(m, k) * dO, "dQ": 2 * max(m, k) * case.scale * slope * K, "dK": 2 * max(m, k) * case.scale * slope * Q,
            "dtable": 2 * m * k * slope}
    for name, times in more.items():
        result, S = want[name]
        off = (got[name] - result).abs()
        tol, least = (TOL_F16, 2.0 ** -25) if dtype == "f16" else (TOL_F32, 0.0)
        assert (off <= tol * S + least + 2.0 ** -36 * times).all(), f"{name}: {off.max()}"
    assert ((got["lse"] - want["lse"][0]).abs() <= 1e-4).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("what", ["K", "V", "Q", "dO"])
@pytest.mark.parametrize("m,k,bias", [(40, 90, 0), (70, 2050, 0), (70, 2050, 8), (5, 90, 8)])
def test_rows_that_see_nothing_beside_non_finite_numbers(dtype, value, what, m, k, bias):
    """Every third row sees nothing: whatever its neighbours see, and whatever stands in its own Q and dO, it gives 0 and adds nothing."""
    case = Case(dtype, heads=2, m=m, k=k, d=48, mask=sparse_rows, buckets=bias, span=20, seed=m)
    empty = torch.arange(m) % 3 == 0
    at = k // 2
    case.seen[1::3, at] = True                           # neighbours of empty rows see what is put there
    case.mask = case.build_mask()
    clean = reference(case.Q, case.K, case.V, case.scale, None, None, case.seen, case.bucket_of, case.table, case.dO)
    if what in ("K", "V"):
        getattr(case, what)[0, 1, at] = value
    else:
        getattr(case, what)[0, 1, 3] = value             # a row that sees nothing
    got = step(case)
    assert (got["O"][0, :, empty] == 0).all() and torch.isneginf(got["lse"][0, :, empty]).all()
    assert (got["dQ"][0, :, empty] == 0).all()
    if what in ("Q", "dO"):
        tol = TOL_F16 if dtype == "f16" else TOL_F32
        for name in ("O", "dQ", "dK", "dV", "dtable")[: 5 if bias else 4]:
            want, S = clean[name]
            assert torch.isfinite(got[name]).all(), name
            assert ((got[name] - want).abs() <= tol * S + 2.0 ** -25).all(), name


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [3, 90])
def test_rows_whose_bias_is_minus_infinity_beside_non_finite_values(dtype, m):
    """Without a mask: all scores of a head are -inf, and V holds Inf."""
    case = Case(dtype, heads=2, m=m, k=150, d=32, buckets=8, span=16, seed=9)
    case.table[0] = -float("inf")
    case.V[0, 0, 70] = float("inf")
    got = step(case)
    assert (got["O"][0, 0] == 0).all() and torch.isneginf(got["lse"][0, 0]).all() and (got["dQ"][0, 0] == 0).all()
    assert all(torch.isfinite(got[name][0, 1]).all() for name in ("O", "lse", "dQ", "dK", "dV"))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("what", ["Q", "dO"])
@pytest.mark.parametrize("mask", [None, causal], ids=["all", "causal"])
@pytest.mark.parametrize("m,k,heads", [(50, 150, 2), (2050, 150, 1), (3, 150, 2)])
def test_gradients_behind_the_states_beside_non_finite_numbers(dtype, value, what, mask, m, k, heads):
    """What stands in Q and dO reaches no state that the sequence does not have: its gradients are 0."""
    lengths = [37, 150, 1, 0, 65]
    case = Case(dtype, batch=5, heads=heads, kv_heads=1, m=m, k=k, d=40, lengths=lengths, mask=mask, seed=m)
    getattr(case, what)[:, 0, m // 2] = value
    got = step(case)
    for b, n in enumerate(lengths):
        for name in ("dK", "dV"):
            assert (got[name][b, :, n:] == 0).all(), f"{name} of sequence {b}, behind {n} states"
    hit = got["dK"][1, 0, 100] if mask is None else got["dQ"][1, 0, m // 2]      # (and it does reach those that are seen)
    assert mask is not None or not torch.isfinite(hit).all()


def close(got, want, allowed, dtype, what):
    """Results of half precision that may be above its largest number, 65504, may be Inf."""
    beyond = (want.abs() + allowed > 65504) & (dtype == "f16")
    assert torch.isfinite(got[~beyond]).all() and not torch.isnan(got).any(), what
    off = torch.where(beyond, 0.0, (got - want).abs() - allowed)
    assert (off <= 0).all(), f"{what}: {off.max():.2e} more than allowed"


def pairs(dtype, m, k, d, score, bias=None, heads=2, seed=0):
    """States in pairs of equal K: each row's score is about `score` (and its bias) for both of one pair; the products of the others have random signs and
    add up to less than 0.6 of that.  P is 1/2 twice and 0 else by the definition.  Fp32 and fp16 numbers of any last bits."""
    case = Case(dtype, heads=heads, m=m, k=k, d=d, seed=seed, buckets=4 if bias is not None else 0, span=3)
    gen = torch.Generator().manual_seed(seed)
    half = (k + 1) // 2
    K = (torch.randint(0, 2, (1, heads, half, d), generator=gen) * 2 - 1) * (0.5 + 0.5 * torch.rand((1, heads, half, d), generator=gen))
    chosen = torch.arange(m) * 7 % half
    size = math.sqrt(score * math.sqrt(d) / (0.58 * d))  # the mean of squares of 0.5 .. 1 is 0.58
    Q = K[:, :, chosen] * size
    case.Q = Q.to(case.dt).cuda()
    case.K = (K * size).to(case.dt).repeat_interleave(2, 2)[:, :, :k].contiguous().cuda()
    if bias is not None:
        case.table[:] = bias
    return case


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("score", [1e3, 1e4, 1e5, 1e6, 1e7, 2e7, 1e8, 1e9, 1e10])
@pytest.mark.parametrize("m,k,bias", [(3, 200, None), (70, 200, None), (70, 60, None), (70, 2050, None), (200, 200, 3.0), (70, 200, -3.0), (12, 130, 3.0)])
def test_large_scores(dtype, score, m, k, bias):
    """Scores are sums of 128 products of one sign, off by at most 130 2^-24 of themselves, and P depends on their differences from the row's
    largest and from lse.  Equal states have equal products whatever is rounded, so that P is 1/2 to the last bits in the forward pass, and in the
    gradients as well once weights are taken over their sum: TOL_F32, or 2^-11 each for P, dS and the result and for D (TOL_F16)."""
    case = pairs(dtype, m, k, 128, score, bias, seed=m + k)
    got = step(case)
    want = reference(case.Q, case.K, case.V, case.scale, bucket_of=case.bucket_of, table=case.table, dO=case.dO)
    lse = want["lse"][0]
    assert (lse > 0.8 * score - 10).all()
    assert ((got["lse"] - lse).abs() <= 131 * 2.0 ** -24 * lse.abs() + 1e-5).all()
    tol = TOL_F16 if dtype == "f16" else TOL_F32
    for name in ("O", "dQ", "dK", "dV"):
        result, S = want[name]
        close(got[name], result, tol * S + 2.0 ** -25, dtype, name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("score", [1e3, 1e5, 1e8, 1e10])
@pytest.mark.parametrize("m,k,heads,bias,poisoned", [(9, 200, 2, None, False), (70, 200, 2, None, False), (70, 2050, 1, 3.0, False), (200, 140, 16, None, False),
                                                     (9, 200, 2, None, True), (70, 200, 2, None, True), (70, 2050, 1, 3.0, True)])
def test_large_scores_with_a_mask(dtype, score, m, k, heads, bias, poisoned):
    """As above, where rows see half of the states; poisoned: K and V of one that none sees are NaN, so that results are formed again one
    position at a time.  A score then is added up in another order than the row's sum was, and may be off by 2 * 131 * 2^-24 of itself,
    all of the weight above 1e5."""
    case = pairs(dtype, m, k, 128, score, bias, heads=heads, seed=m + k)
    gen = torch.Generator().manual_seed(m)
    case.seen = torch.rand((m, k), generator=gen) < 0.5
    chosen = torch.arange(m) * 7 % ((k + 1) // 2)
    for i in range(m):
        case.seen[i, 2 * chosen[i]:2 * chosen[i] + 2] = True
    if poisoned:
        at = int((torch.bincount(chosen, minlength=k // 2)[:k // 2] == 0).nonzero()[-1]) * 2      # of a pair that no row has chosen
        case.seen[:, at] = False
    case.mask = case.build_mask()
    want = reference(case.Q, case.K, case.V, case.scale, seen=case.seen, bucket_of=case.bucket_of, table=case.table, dO=case.dO)
    if poisoned:
        case.K[:, :, at] = case.V[:, :, at] = float("nan")
    got = step(case)
    tol = (TOL_F16 if dtype == "f16" else TOL_F32) + (math.expm1(min(1.0, 2 * 131 * 2.0 ** -24 * score)) if poisoned else 0.0)
    for name in ("O", "dQ", "dK", "dV"):
        result, S = want[name]
        if poisoned and name in ("dK", "dV"):
            assert (got[name][:, :, at] == 0).all(), name
        close(got[name], result, tol * S + 2.0 ** -25, dtype, name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,k,span", [(1, 150, 16), (40, 150, 16), (40, 150, 1000), (40, 2050, 16)])
@pytest.mark.parametrize("entry", [-65504.0, 1234.5])
def test_one_large_bias_for_all(dtype, m, k, span, entry):
    """Scores of one large number only: P is 1 / k to a rounding whatever lse's own costs (2^-9 at 65504).  dV then is dO's sum over k, off by
    2^-11 for P and 2^-11 for the result in half precision, and by TOL_F32 in single."""
    case = Case(dtype, heads=2, m=m, k=k, d=64, buckets=8, span=span, seed=3)
    case.Q.zero_()
    case.table[:] = entry
    got = step(case)
    tol = 2 * 2.0 ** -11 + 1e-5 if dtype == "f16" else TOL_F32
    dO = case.dO.cpu().double()
    err, S = (got["dV"] - dO.sum(2, keepdim=True) / k).abs(), dO.abs().sum(2, keepdim=True) / k
    assert (err <= tol * S + 2.0 ** -25).all(), f"{(err / S).max():.2e}"


@pytest.mark.parametrize("m,k", [(3, 300), (40, 300), (200, 333)])
def test_numbers_of_unequal_size_in_a_head(m, k):
    """Rows of K, V, dO (and of Q in the second head that shares K and V) between 1 and 2^-20 of the largest, in single precision.
    A factor counts to 2^-23 of itself or to 2^-39 of the largest of its kind (dS: to 2^-36): beside what TOL_F32 allows, each sum may be off
    by those times what they meet."""
    case = Case("f32", heads=2, kv_heads=1, m=m, k=k, d=64, seed=k)
    gen = torch.Generator().manual_seed(k)
    for t in (case.K, case.V, case.dO):
        t.mul_((2.0 ** -torch.randint(0, 21, t.shape[:3], generator=gen).double()).float()[..., None].cuda())
    case.Q[:, 1].mul_((2.0 ** -torch.randint(0, 21, case.Q.shape[2:3], generator=gen).double()).float()[:, None].cuda())
    got = step(case)
    want = reference(case.Q, case.K, case.V, case.scale, dO=case.dO)
    Q, K, V, dO = (t.cpu().double() for t in (case.Q, case.K, case.V, case.dO))
    most = lambda t: t.abs().max()
    # P: of scores off by 64 products of 2^-39 of the largest factor, and what it counts to itself
    p = 64 * case.scale * 2 * 2.0 ** -39 * most(Q) * most(K) + 2.0 ** -39
    dp = 2 * (64 * 2 * 2.0 ** -39 * most(dO) * most(V))                   # of dP - D
    # dS: P and dP as they are, and 2^-36 of the largest dS that a wave meets
    ds = p * 2 * 64 * most(dO) * most(V) + dp + 2.0 ** -36 * 2 * 64 * most(dO) * most(V)
    floor = {"O": p * V.abs().sum(2) + 2.0 ** -39 * most(V), "dV": (p * dO.abs().sum((1, 2)) + 2.0 ** -39 * 2 * m * most(dO))[None],
             "dQ": case.scale * (ds * K.abs().sum(2) + k * 2.0 ** -39 * most(K) * 128 * most(dO) * most(V)),
             "dK": case.scale * (ds * Q.abs().sum((1, 2)) + 2 * m * 2.0 ** -39 * most(Q) * 128 * most(dO) * most(V))[None]}
    for name, more in floor.items():
        result, S = want[name]
        off = (got[name] - result).abs() - more[:, :, None, :]
        assert (off <= TOL_F32 * S).all(), f"{name}: {off.max():.2e}"


@pytest.mark.parametrize("dtype,d", [("f32", 128), ("f16", 127)])
def test_more_rows_than_one_round_of_workgroups_copies(dtype, d):
    """A million states, whose terms (copies) take more blocks of rows than a grid has workgroups."""
    k, m = 65536 * 16 + 100, 17
    dt = torch.float16 if dtype == "f16" else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(5)
    Q, K, V = (torch.randn((1, 1, n, d), generator=gen, device="cuda").to(dt) for n in (m, k, k))
    Q *= 2
    K[0, 0, -1], V[0, 0, -1] = 3 * Q[0, 0, 3] / Q[0, 0, 3].norm() * 4, 100.0       # the last one is seen by some
    O = torch.full_like(Q, float("nan"))
    lse = torch.full((1, 1, m), float("nan"), device="cuda")
    scale = 1 / math.sqrt(d)
    p = spdl.attention_problem(Q, K, V, O, scale)
    workspace = torch.empty(spdl.spdl_attention_workspace(p, K.element_size()), dtype=torch.uint8, device="cuda")
    call = spdl.spdl_attention_f16 if dtype == "f16" else spdl.spdl_attention
    call(p, Q, K, V, None, None, None, None, None, O, lse, workspace)
    s = scale * (Q[0, 0].double() @ K[0, 0].double().T)
    want = torch.logsumexp(s, 1)
    P = torch.exp(s - want[:, None])
    assert ((lse[0, 0] - want).abs() <= 1e-4).all()
    S = P @ V[0, 0].double().abs()
    assert ((O[0, 0].double() - P @ V[0, 0].double()).abs() <= (TOL_F16 if dtype == "f16" else TOL_F32) * S + 2.0 ** -25).all()
    del Q, K, V, O, s, P, S, workspace
    torch.cuda.empty_cache()
