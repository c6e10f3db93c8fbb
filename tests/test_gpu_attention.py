"""Attention in one call and its gradients against the definition in 64 bits, at the sizes, masks and layouts where a tile, a block of
keys or a split of the work can go wrong."""
import numpy as np
import pytest
import torch

import paper_2006_10901_amd as spdl
from tests.attention_util import Case, banded, blocks, causal, nothing, reference, sparse_rows

pytestmark = pytest.mark.gpu

TYPES = ["f32", "f16"]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,k,d", [(1, 1, 1), (1, 64, 64), (2, 3, 8), (5, 63, 20), (16, 65, 32), (17, 64, 40), (33, 130, 64), (64, 31, 96),
                                   (128, 128, 128), (129, 257, 80), (200, 77, 100), (300, 1000, 64), (31, 2050, 128), (700, 33, 32)])
def test_sizes(dtype, m, k, d):
    Case(dtype, batch=2, heads=3, m=m, k=k, d=d, seed=m + k).check(what=f"{dtype} {m}x{k} d {d}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [1, 3, 16, 17, 150])
@pytest.mark.parametrize("heads,kv_heads", [(8, 1), (6, 2), (40, 1)])
def test_shared_heads(dtype, m, heads, kv_heads):
    Case(dtype, batch=2, heads=heads, kv_heads=kv_heads, m=m, k=201, d=48, lengths=[201, 90], buckets=8, span=32, positions=[201 - m, 90 - m],
         seed=m).check(what=f"{dtype} {heads}/{kv_heads} m {m}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,k", [(1, 300), (7, 70), (90, 300), (300, 300)])
@pytest.mark.parametrize("bias", [0, 8])
def test_lengths(dtype, m, k, bias):
    Case(dtype, batch=6, heads=2, m=m, k=k, d=64, lengths=[k, 0, 1, 64, 65, k // 2], buckets=bias, seed=3).check(what=f"{dtype} lengths {m}x{k}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,heads,m", [(65, 2, 1), (65, 1, 40), (64, 8, 1), (9, 16, 130)])
def test_many_sequences_of_unequal_length(dtype, batch, heads, m):
    lengths = [(37 * b) % 150 for b in range(batch)]
    Case(dtype, batch=batch, heads=heads, m=m, k=149, d=32, lengths=lengths, buckets=8, span=20, seed=batch).check(what=f"{dtype} {batch} x {heads} x {m}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,m,k", [(2, 0, 70), (2, 9, 0), (2, 40, 0), (0, 9, 70)])
@pytest.mark.parametrize("mask", [None, causal], ids=["all", "causal"])
def test_nothing_to_attend(dtype, batch, m, k, mask):
    """No queries: the states' gradients are 0.  No states: results of 0, as for any row that sees nothing.  The table's gradient is 0."""
    case = Case(dtype, batch=batch, heads=2, m=m, k=k, d=32, mask=mask, buckets=8, span=20).prepare()
    case.forward()
    case.backward()
    for name, got in case.results().items():
        want = torch.full_like(got, float("-inf")) if name == "lse" else torch.zeros_like(got)
        assert torch.equal(got, want), name


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("mask", [banded, causal, blocks, nothing, sparse_rows], ids=lambda f: f.__name__)
@pytest.mark.parametrize("m,k", [(1, 200), (9, 129), (130, 260), (333, 333), (64, 5000)])
def test_masks(dtype, mask, m, k):
    Case(dtype, heads=2, m=m, k=k, d=64, mask=mask, buckets=16 if m % 2 else 0, span=40, seed=m).check(what=f"{dtype} {mask.__name__} {m}x{k}")


@pytest.mark.parametrize("dtype", TYPES)
def test_mask_with_lengths_and_shared_heads(dtype):
    Case(dtype, batch=3, heads=4, kv_heads=2, m=140, k=270, d=72, lengths=[270, 66, 0], mask=sparse_rows, buckets=32, span=128,
         seed=5).check(what=dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("buckets,span,both", [(3, 0, True), (3, 1, True), (20, 7, True), (2, 3, False), (32, 128, True), (32, 128, False), (128, 1024, True)])
@pytest.mark.parametrize("m,k,positions", [(1, 300, [299, 7]), (16, 100, [-50, 400]), (150, 150, None), (260, 900, [100, -3]),
                                           (40, 64, [2 ** 31 - 1, -2 ** 31])])
def test_bias(dtype, buckets, span, both, m, k, positions):
    Case(dtype, batch=2, heads=2, m=m, k=k, d=32, buckets=buckets, span=span, both=both, positions=positions,
         seed=span).check(what=f"{dtype} {buckets} {span} {m}x{k}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("heads,kv_heads,m,k", [(40, 1, 1, 400), (40, 1, 5, 90), (2, 2, 150, 2500)])
def test_the_largest_bias(dtype, d, heads, kv_heads, m, k):
    """What most LDS is taken for: 2049 relative positions and 128 buckets beside tiles of every width."""
    Case(dtype, heads=heads, kv_heads=kv_heads, m=m, k=k, d=d, buckets=128, span=1024, positions=[k // 2], seed=d).check(what=f"{dtype} {d} {m}x{k}")


@pytest.mark.parametrize("m,k,lengths,mask,buckets", [(300, 2, None, None, 0), (300, 5, None, None, 16), (300, 20, None, None, 0), (100, 700, [3, 40], None, 16),
                                                      (20, 700, [64, 2], None, 0), (64, 64, None, causal, 0), (128, 500, None, causal, 16)])
def test_gradients_of_rows_that_see_few_keys_in_half_precision(m, k, lengths, mask, buckets):
    """Two roundings of one size stand between a gradient and its exact value, that of P or dS and that of the result, independent of each
    other: sqrt(2) of what rounding the exact value costs, in the 2-norm.  Of the first there are 640 at least (16 heads of 20 queries and
    2 keys; a row of dK shares them).  The square of an even rounding error scatters by 0.9 of its mean, those of values whose fourth
    moment is 10 times their squared second by 0.9 sqrt(10), so that the first half of the sum of squares scatters by 0.9 sqrt(10 / 640)
    = 11 %, the sum by 5.6 %, its root by 2.8 %: sqrt(2) (1 + 4 * 0.028) = 1.57.  D = dO . O from the rounded O would make it 2.5 with
    two keys."""
    case = Case("f16", batch=2, heads=16, m=m, k=k, d=64, lengths=lengths, mask=mask, buckets=buckets, span=8, seed=m + k).prepare()
    case.forward()
    case.backward()
    ref = reference(case.Q, case.K, case.V, case.scale, case.lengths, case.positions, case.seen, case.bucket_of, case.table, case.dO)
    for name in ("dQ", "dK", "dV"):
        want = ref[name][0]
        off, least = (case.results()[name].cpu().double() - want).norm(), (want.half().double() - want).norm()
        assert off < 1.57 * least, f"{name}: {off / least:.3f}"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["rows", "odd"])
@pytest.mark.parametrize("m,k,d", [(1, 130, 33), (20, 50, 64), (140, 200, 41), (130, 130, 128)])
def test_layouts(dtype, layout, m, k, d):
    Case(dtype, batch=2, heads=4, kv_heads=2, m=m, k=k, d=d, layout=layout, seed=d).check(what=f"{dtype} {layout} {m}x{k} d {d}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0])
@pytest.mark.parametrize("m", [2, 70])
@pytest.mark.parametrize("bias", [0, 8])
def test_scales(dtype, scale, m, bias):
    Case(dtype, heads=2, m=m, k=100, d=16, scale=scale, mask=sparse_rows, buckets=bias, seed=2).check(what=f"{dtype} scale {scale}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("what", ["V", "K", "Q", "dO"])
@pytest.mark.parametrize("m,k,d,bias", [(3, 200, 64, 0), (12, 150, 96, 8), (200, 200, 64, 0), (150, 700, 128, 8)])
def test_non_finite_numbers_reach_what_sees_them(dtype, value, what, m, k, d, bias):
    """A row of Inf or NaN makes what depends on it Inf or NaN and nothing else: all other results are as without it."""
    case = Case(dtype, heads=2, m=m, k=k, d=d, mask=banded, buckets=bias, span=24, seed=11)
    at = (m if what in ("Q", "dO") else k) // 2
    case.seen[:, : k // 8] = True                       # a key that few rows see, and rows that see much
    if what in ("V", "K"):
        case.seen[:, at] = False
        case.seen[m // 3, at] = True
    case.mask = case.build_mask()
    case.prepare()
    clean = reference(case.Q, case.K, case.V, case.scale, None, None, case.seen, case.bucket_of, case.table, case.dO)
    getattr(case, what)[0, 1, at] = value               # of the second head only
    case.forward()
    case.backward()
    torch.cuda.synchronize()
    rows = case.seen[:, at] if what in ("V", "K") else torch.arange(m) == at           # rows that depend on it
    keys = case.seen[rows].any(0)                        # keys whose gradients such rows reach
    touched = {"O": rows if what != "dO" else torch.zeros(m, dtype=torch.bool), "lse": rows if what in ("K", "Q") else torch.zeros(m, dtype=torch.bool),
               "dQ": rows, "dK": keys, "dV": keys}
    if what in ("V",):
        touched["dV"] = torch.zeros(k, dtype=torch.bool)  # P does not depend on V
    for name, hit in touched.items():
        got = case.results()[name].cpu().double()
        want, S = clean[name]
        assert torch.isfinite(got[0, 0]).all(), f"{name}: the other head"
        part = got[0, 1]
        if value != value and hit.any():
            assert not torch.isfinite(part[hit]).any(), f"{name}: a number where a NaN is seen"
        ok = ~hit
        tol = (2e-3 if dtype == "f16" else 1e-4) if name != "lse" else 1e-4
        err = (part[ok] - want[0, 1][ok]).abs()
        assert torch.isfinite(part[ok]).all(), f"{name}: Inf or NaN where nothing sees it"
        assert (err <= tol * S[0, 1][ok] + 2.0 ** -25).all(), f"{name}: {err.max()}"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [1, 90])
def test_keys_and_values_that_all_share(dtype, m):
    """One source for all sequences and heads: strides of 0.  Their gradients are each sequence's own."""
    case = Case(dtype, batch=3, heads=4, m=m, k=130, d=64, seed=7)
    case.K, case.V = (t[:1, :1].expand(3, 4, 130, 64) for t in (case.K, case.V))
    case.output = lambda like: torch.full(like.shape, float("nan"), dtype=like.dtype, device="cuda")
    case.check(what=dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [1, 140])
def test_rows_of_everything(dtype, m):
    """Rows all of whose positions have the lowest finite bias see all of them alike; those with -inf see none."""
    case = Case(dtype, heads=3, m=m, k=150, d=32, buckets=8, span=16, seed=9)
    lowest = torch.finfo(case.dt).min
    case.table[0] = lowest
    case.table[1] = -float("inf")
    case.prepare()
    case.forward()
    case.backward()
    torch.cuda.synchronize()
    tol = 2e-3 if dtype == "f16" else 1e-4
    for t in (case.O, case.dQ, case.dK, case.dV, case.dtable):
        assert torch.isfinite(t).all()
    assert (case.O[0, 1] == 0).all() and torch.isneginf(case.lse[0, 1]).all()
    for t in (case.dQ, case.dK, case.dV):
        assert (t[0, 1] == 0).all()
    assert (case.dtable[1] == 0).all()
    if dtype == "f32":                                   # fp32's lowest: any score is lost beside it
        mean = case.V[0, 0].double().mean(0)
        assert ((case.O[0, 0].double() - mean).abs() <= tol * case.V[0, 0].double().abs().mean(0)).all()
        each = case.dO[0, 0].double().sum(0) / 150
        assert ((case.dV[0, 0].double() - each).abs() <= tol * case.dO[0, 0].double().abs().sum(0) / 150).all()
    # the third head, beside them
    ref = reference(case.Q[:, 2:], case.K[:, 2:], case.V[:, 2:], case.scale, bucket_of=case.bucket_of, table=case.table[2:], dO=case.dO[:, 2:])
    for name, got in (("O", case.O), ("dQ", case.dQ), ("dK", case.dK), ("dV", case.dV)):
        want, S = ref[name]
        assert ((got[:, 2:].cpu().double() - want).abs() <= tol * S + 2.0 ** -25).all(), name


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("low,high", [(-30, -20), (10, 14)])
def test_magnitudes(dtype, low, high):
    """Gradients and values far from 1, either way: fp16 terms and fp16 dS keep their bits (powers of two: exact scalings)."""
    case = Case(dtype, heads=2, m=100, k=180, d=64, buckets=8, span=16, seed=4)
    if dtype == "f16" and low < -20:
        low, high = -10, -8                              # within fp16's own range
    case.dO.mul_(2.0 ** low)
    case.V.mul_(2.0 ** (high if dtype == "f32" else min(high, 4)))
    case.check(what=f"{dtype} 2^{low} 2^{high}")


@pytest.mark.parametrize("dtype", TYPES)
def test_offsets_beyond_32_bits(dtype):
    """Heads of K and V that lie more than 2^31 elements into their array."""
    rows, d = 520, 64
    far = 2 ** 31 + 64
    case = Case(dtype, heads=2, m=3, k=rows, d=d, seed=6)
    room = torch.empty(far + rows * d, dtype=case.dt, device="cuda")
    K = torch.as_strided(room, (1, 2, rows, d), (0, far, d, 1))
    K.copy_(case.K)
    case.K = K
    case.output = lambda like: torch.full(like.shape, float("nan"), dtype=like.dtype, device="cuda")
    case.check(what=dtype)
    del room, K, case
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,k,mask", [(1, 3000, None), (100, 300, banded), (600, 200, None)])
def test_same_bits_every_time_and_inputs_left_alone(dtype, m, k, mask):
    case = Case(dtype, batch=1 if mask else 2, heads=4, kv_heads=2, m=m, k=k, d=80, mask=mask, buckets=16, span=64, seed=8).prepare()
    inputs = [t.clone() for t in (case.Q, case.K, case.V, case.dO, case.table)]
    first = None
    for i in range(3):
        if case.workspace is not None:
            case.workspace.fill_([255, 0, 127][i])       # what the workspace holds does not matter
        case.forward()
        case.backward()
        torch.cuda.synchronize()
        now = [t.clone() for t in case.results().values()]
        first = first or now
        assert all(torch.equal(x, y) for x, y in zip(first, now))
    assert all(torch.equal(x, y) for x, y in zip(inputs, (case.Q, case.K, case.V, case.dO, case.table)))


@pytest.mark.parametrize("dtype", TYPES)
def test_a_training_step_in_a_graph(dtype):
    """Captured on a stream of its own, replayed with new inputs and with eager work between the replays."""
    case = Case(dtype, batch=2, heads=4, m=70, k=333, d=64, lengths=[333, 150], buckets=8, span=32, seed=3).prepare()
    other = Case(dtype, heads=2, m=40, k=90, d=32, seed=12).prepare()
    stream = torch.cuda.Stream()
    case.forward(), case.backward()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        case.forward()
        case.backward()
    gen = torch.Generator().manual_seed(1)
    for i in range(3):
        for t in (case.Q, case.dO):
            t.copy_(torch.randn(t.shape, generator=gen).to(t.dtype))
        case.lengths.copy_(torch.tensor([333 - 40 * i, 100 + 50 * i], dtype=torch.int32))
        case.K.nan_to_num_(), case.V.nan_to_num_()
        other.forward()
        graph.replay()
        other.backward()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in case.results().values()]
        case.forward(), case.backward()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(replayed, case.results().values())), i


def test_two_streams_at_once():
    a, b = (Case("f16", batch=2, heads=8, m=200, k=700, d=64, seed=s).prepare() for s in (1, 2))
    a.forward(), a.backward(), b.forward(), b.backward()
    torch.cuda.synchronize()
    alone = [t.clone() for c in (a, b) for t in c.results().values()]
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        for c, s in zip((a, b), streams):
            for t in c.results().values():
                t.fill_(float("nan"))
        torch.cuda.synchronize()
        for c, s in zip((a, b), streams):
            c.forward(s)
        for c, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                c.backward()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(alone, (t for c in (a, b) for t in c.results().values())))


@pytest.mark.parametrize("m,k,nnz", [(1, 1, 1), (5, 70, 9), (64, 64, 4096), (65, 129, 1), (130, 5000, 20000), (300, 300, 0), (70, 40000, 9000), (67, 140000, 5000), (3, 600000, 5000)])
def test_mask_from_a_topology(m, k, nnz):
    """Every bit by rows and by columns, and which tiles hold any; indices in no order, and twice."""
    gen = torch.Generator().manual_seed(m * k)
    cells = torch.randperm(m * k, generator=gen)[:nnz]
    rows = torch.cat([cells // k, cells[: nnz // 3] // k])
    cols = torch.cat([cells % k, cells[: nnz // 3] % k])
    order = torch.argsort(rows, stable=True)
    ro = torch.zeros(m + 1, dtype=torch.int32)
    ro[1:] = torch.cumsum(torch.bincount(rows, minlength=m), 0)
    n = spdl.spdl_attention_mask_bytes(m, k)
    mask = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    spdl.spdl_build_attention_mask(m, k, rows.numel(), ro.cuda(), cols[order].to(torch.int32).cuda(), mask)
    words = mask.cpu().numpy().view(np.uint64)
    ti, tj = (m + 63) // 64, (k + 63) // 64
    seen = np.zeros((ti * 64, tj * 64), dtype=bool)
    seen[rows.numpy(), cols.numpy()] = True
    bits = lambda w: ((w[..., None] >> np.arange(64, dtype=np.uint64)) & np.uint64(1)).astype(bool)
    at = 0
    by_rows = bits(words[at:at + tj * ti * 64].reshape(tj, ti * 64))
    assert np.array_equal(by_rows.transpose(1, 0, 2).reshape(ti * 64, tj * 64), seen)
    at += tj * ti * 64
    by_cols = bits(words[at:at + ti * tj * 64].reshape(ti, tj * 64))
    assert np.array_equal(by_cols.transpose(0, 2, 1).reshape(ti * 64, tj * 64), seen)
    at += ti * tj * 64
    tiles = seen.reshape(ti, 64, tj, 64).any(axis=(1, 3))
    per_row, per_col = (tj + 63) // 64, (ti + 63) // 64
    assert np.array_equal(bits(words[at:at + ti * per_row].reshape(ti, per_row)).reshape(ti, -1)[:, :tj], tiles)
    at += ti * per_row
    assert np.array_equal(bits(words[at:at + tj * per_col].reshape(tj, per_col)).reshape(tj, -1)[:, :ti], tiles.T)
    assert at + tj * per_col == words.size


def test_calls_that_the_binding_refuses():
    case = Case("f32", batch=2, heads=2, m=20, k=40, d=16, buckets=4, span=8, lengths=[40, 30], seed=1).prepare()
    case.forward()
    torch.cuda.synchronize()
    good = dict(case.__dict__)

    def refused(error=ValueError, **change):
        case.__dict__.update(change)
        with pytest.raises(error):
            case.forward()
        with pytest.raises(error):
            case.backward()
        case.__dict__.update(good)

    refused(Q=case.Q[:, :, :19])                         # not the problem's sizes
    refused(K=case.K.transpose(1, 2).contiguous().transpose(1, 2))          # nor its strides
    refused(V=case.V.half())
    refused(O=case.O.cpu())
    refused(lengths=case.lengths[:1])
    refused(lengths=case.lengths.long())
    refused(table=case.table[:1])
    refused(bucket_of=case.bucket_of[:-1])
    refused(lse=case.lse[:1])
    refused(mask=torch.zeros(8, dtype=torch.uint8, device="cuda"))
    refused(problem=b"no problem")
    refused(spdl.SpdlError, table=None)
    if case.workspace is not None:
        with pytest.raises(spdl.SpdlError):
            case.workspace = case.workspace[:16]
            case.backward()
    with pytest.raises(ValueError):
        spdl.spdl_build_attention_mask(64, 64, 0, torch.zeros(65, dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"),
                                       torch.zeros(100, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_by_differences(dtype):
    """The gradients against differences of the loss sum(dO * O) in 64 bits, along random directions of every input."""
    case = Case(dtype, batch=1, heads=2, kv_heads=1, m=24, k=50, d=16, mask=sparse_rows, buckets=8, span=12, seed=10).prepare()
    case.forward()
    case.backward()
    torch.cuda.synchronize()
    inputs = {"Q": case.Q, "K": case.K, "V": case.V, "table": case.table}
    grads = {"Q": case.dQ, "K": case.dK, "V": case.dV, "table": case.dtable}
    x = {n: t.cpu().double() for n, t in inputs.items()}
    gen = torch.Generator().manual_seed(2)
    eps = 1e-5                                           # error of the difference: eps^2 and 1e-16 / eps, far below the tolerance

    def loss(x):
        out = reference(x["Q"], x["K"], x["V"], case.scale, None, None, case.seen, case.bucket_of, x["table"], None)
        return float((out["O"][0] * case.dO.cpu().double()).sum())

    clean = reference(case.Q, case.K, case.V, case.scale, None, None, case.seen, case.bucket_of, case.table, case.dO)
    for name in inputs:
        way = torch.randn(x[name].shape, generator=gen, dtype=torch.float64)
        there = (loss({**x, name: x[name] + eps * way}) - loss({**x, name: x[name] - eps * way})) / (2 * eps)
        here = float((grads[name].cpu().double() * way).sum())
        S = float((clean["d" + name][1] * way.abs()).sum())
        assert abs(here - there) <= (2e-3 if dtype == "f16" else 1e-4) * S, name


def test_a_layer_as_it_is_used():
    """An encoder-decoder step: sparse self-attention with a bias, then attention to an encoder's states of another length, forward and
    back through both, against the same in 64 bits."""
    self_attention = Case("f32", batch=1, heads=4, m=160, k=160, d=32, mask=causal, buckets=16, span=40, layout="rows", seed=20).prepare()
    cross = Case("f32", batch=1, heads=4, m=160, k=310, d=32, lengths=[280], layout="rows", seed=21)
    cross.Q = self_attention.O                           # the cross attention's queries are what the first one gives
    cross.prepare()
    self_attention.forward()
    cross.forward()
    cross.backward()
    self_attention.dO = cross.dQ
    self_attention.problem = spdl.attention_problem(self_attention.Q, self_attention.K, self_attention.V, self_attention.O, self_attention.scale,
                                                    bucket_of=self_attention.bucket_of, table=self_attention.table, dO=cross.dQ,
                                                    dQ=self_attention.dQ, dK=self_attention.dK, dV=self_attention.dV)
    self_attention.backward()
    torch.cuda.synchronize()
    c = self_attention
    first = reference(c.Q, c.K, c.V, c.scale, seen=c.seen, bucket_of=c.bucket_of, table=c.table)["O"][0]
    second = reference(first, cross.K.nan_to_num(), cross.V.nan_to_num(), cross.scale, lengths=cross.lengths, dO=cross.dO)
    back = reference(c.Q, c.K, c.V, c.scale, seen=c.seen, bucket_of=c.bucket_of, table=c.table, dO=second["dQ"][0])
    for got, want in ((cross.O, second["O"][0]), (cross.dK, second["dK"][0]), (cross.dV, second["dV"][0]), (c.dQ, back["dQ"][0]), (c.dK, back["dK"][0]),
                      (c.dV, back["dV"][0]), (c.dtable, back["dtable"][0])):
        # two layers, each within 1e-4 of sums of absolute values that are at most 30 times the results' 2-norm here
        assert (got.cpu().double() - want).norm() <= 2 * 30 * 1e-4 * want.norm()
