"""Attention where numbers, lengths and masks meet the ends of what they may be: large biases and scores, Inf and NaN beside rows that
see nothing and behind a sequence's states, numbers of unequal size in one head."""
import pytest
import torch

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
