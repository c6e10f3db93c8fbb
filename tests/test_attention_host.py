"""Attention's host side: what is refused, before anything touches a GPU, and the buckets of relative positions."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2006_10901_amd as spdl

INVALID, UNSUPPORTED = -1, -4
ONE, NULL = ctypes.c_void_p(256), ctypes.c_void_p(0)     # never dereferenced: the checks fail first


def problem(batch=2, heads=4, kv_heads=2, m=100, k=300, d=64, span=8, buckets=4, scale=0.125, **strides):
    p = spdl.AttentionProblem(batch=batch, heads=heads, kv_heads=kv_heads, m=m, k=k, d=d, span=span, buckets=buckets, scale=scale)
    for name, n, rows in (("Q", heads, m), ("O", heads, m), ("dO", heads, m), ("dQ", heads, m), ("K", kv_heads, k), ("V", kv_heads, k),
                          ("dK", kv_heads, k), ("dV", kv_heads, k)):
        s = getattr(p, name)
        s.batch, s.head, s.row = strides.get(name, (n * rows * d, rows * d, d))
    return p


def forward(p, Q=ONE, K=ONE, V=ONE, bucket_of=NULL, table=NULL, O=ONE, workspace=NULL, size=0, f16=False):
    fn = spdl.lib().spdl_attention_f16 if f16 else spdl.lib().spdl_attention
    return fn(ctypes.byref(p), Q, K, V, NULL, NULL, NULL, bucket_of, table, O, NULL, workspace, ctypes.c_int64(size), NULL)


def backward(p, Q=ONE, K=ONE, V=ONE, bucket_of=NULL, table=NULL, O=ONE, lse=ONE, dO=ONE, dQ=ONE, dK=ONE, dV=ONE, dtable=NULL,
             workspace=NULL, size=0):
    return spdl.lib().spdl_attention_backward(ctypes.byref(p), Q, K, V, NULL, NULL, NULL, bucket_of, table, O, lse, dO, dQ, dK, dV, dtable,
                                              workspace, ctypes.c_int64(size), NULL)


@pytest.mark.parametrize("wrong", [dict(batch=-1), dict(heads=-4), dict(heads=5), dict(kv_heads=0), dict(m=-1), dict(k=-1), dict(d=0),
                                   dict(span=-1), dict(span=1025), dict(buckets=129), dict(buckets=-1), dict(scale=math.nan),
                                   dict(scale=math.inf), dict(m=2 ** 30), dict(batch=2 ** 20, heads=64, kv_heads=64),
                                   dict(batch=2 ** 19, heads=8, kv_heads=8), dict(batch=2 ** 10, heads=8, kv_heads=8, k=2 ** 20)])
def test_sizes_that_are_refused(wrong):
    p = problem(**wrong)
    assert forward(p) == INVALID and forward(p, f16=True) == INVALID and backward(p) == INVALID
    with pytest.raises(spdl.SpdlError):
        spdl.spdl_attention_workspace(p, 4)


def test_width_that_is_not_supported():
    p = problem(d=129)
    assert forward(p) == UNSUPPORTED and backward(p) == UNSUPPORTED


def test_pointers_that_are_refused():
    p = problem()
    assert spdl.spdl_attention_workspace(p, 4, True) > 0
    for name in ("Q", "K", "V", "O"):
        assert forward(p, **{name: NULL}) == INVALID, name
    for name in ("Q", "K", "V", "O", "lse", "dO", "dQ", "dK", "dV"):
        assert backward(p, workspace=ONE, size=1 << 40, **{name: NULL}) == INVALID, name
    assert forward(p, table=ONE) == INVALID and forward(p, bucket_of=ONE) == INVALID
    assert backward(p, dtable=ONE, workspace=ONE, size=1 << 40) == INVALID          # no table, no gradient of it
    assert forward(problem(buckets=0), table=ONE, bucket_of=ONE) == INVALID


def test_workspaces_that_are_refused():
    p = problem(batch=1, heads=1, kv_heads=1, m=1, k=100000)
    n = spdl.spdl_attention_workspace(p, 2)
    assert n > 0
    assert forward(p) == INVALID
    assert forward(p, workspace=ONE, size=n - 1) == INVALID
    assert forward(p, workspace=ctypes.c_void_p(264), size=n) == INVALID            # 16-byte alignment
    assert backward(p, workspace=ONE, size=15) == INVALID
    with pytest.raises(spdl.SpdlError):
        spdl.spdl_attention_workspace(p, 3)


@pytest.mark.parametrize("strides", [(0, 6400, 64), (25600, 0, 64), (25600, 6400, 0), (25600, 6400, 63), (25600, 6399, 64), (-25600, 6400, 64),
                                     (64, 64, 256), (2 ** 62, 6400, 64)])
def test_outputs_whose_elements_share_addresses_are_refused(strides):
    assert forward(problem(O=strides)) == INVALID
    assert backward(problem(dQ=strides), workspace=ONE, size=1 << 40) == INVALID


def test_input_strides():
    assert forward(problem(Q=(-1, 64, 64))) == INVALID
    # what a call does not take is not looked at, and inputs may be the same for all
    assert forward(problem(K=(0, 0, 0), V=(0, 0, 0), dQ=(0, 0, 0)), O=NULL) == INVALID          # for O alone
    assert forward(problem(m=0, K=(0, 0, 0), V=(0, 0, 0), dQ=(0, 0, 0))) == 0


def test_nothing_to_do():
    for p in (problem(batch=0), problem(m=0), problem(heads=0, kv_heads=0)):
        assert forward(p, Q=NULL, O=NULL) == 0
    assert backward(problem(batch=0), Q=NULL, K=NULL, V=NULL, dQ=NULL) == 0
    assert backward(problem(heads=0, kv_heads=0)) == 0


def test_mask_arguments():
    lib = spdl.lib()
    assert lib.spdl_build_attention_mask(-1, 4, 0, ONE, ONE, ONE, NULL) == INVALID
    assert lib.spdl_build_attention_mask(4, 4, -1, ONE, ONE, ONE, NULL) == INVALID
    assert lib.spdl_build_attention_mask(4, 4, 1, ONE, ONE, NULL, NULL) == INVALID
    assert lib.spdl_build_attention_mask(4, 4, 1, ONE, ONE, ctypes.c_void_p(260), NULL) == INVALID
    assert lib.spdl_build_attention_mask(4, 4, 1, NULL, ONE, ONE, NULL) == INVALID
    assert lib.spdl_build_attention_mask(0, 4, 0, NULL, NULL, NULL, NULL) == 0
    assert spdl.spdl_attention_mask_bytes(0, 100) == 0
    assert spdl.spdl_attention_mask_bytes(1, 1) == 8 * (64 + 64 + 1 + 1)
    assert spdl.spdl_attention_mask_bytes(130, 5000) == 8 * (2 * 64 * 3 * 79 + 3 * 2 + 79)
    with pytest.raises(spdl.SpdlError):
        spdl.spdl_attention_mask_bytes(-1, 4)


def whole_number_bucket(rel, buckets, distance, both):
    """The definition without logarithms: e is the most with (n / exact)^steps >= (distance / exact)^e."""
    side = buckets // 2 if both else buckets
    n = abs(rel) if both else max(-rel, 0)
    exact = side // 2
    steps = side - exact
    if n < exact:
        b = n
    else:
        e = 0
        while e + 1 < steps and n ** steps * exact ** (e + 1) >= distance ** (e + 1) * exact ** steps:
            e += 1
        b = exact + e
    return b + (side if both and rel > 0 else 0)


@pytest.mark.parametrize("both", [True, False])
@pytest.mark.parametrize("buckets,distance", [(32, 128), (16, 64), (64, 256), (128, 1024), (32, 20), (4, 3), (5, 100), (31, 1000), (33, 513)])
def test_relative_buckets(buckets, distance, both):
    got = spdl.spdl_build_relative_buckets_host(buckets, distance, both)
    assert got.dtype == np.int32
    assert got.tolist() == [whole_number_bucket(r, buckets, distance, both) for r in range(-distance, distance + 1)]
    assert got.min() == 0 and got.max() < buckets


@pytest.mark.parametrize("buckets,distance,both", [(0, 8, False), (1, 8, False), (3, 8, True), (129, 200, False), (32, 0, True), (32, 1025, True),
                                                   (32, 8, True), (32, 16, False)])
def test_relative_buckets_that_are_refused(buckets, distance, both):
    with pytest.raises(spdl.SpdlError):
        spdl.spdl_build_relative_buckets_host(buckets, distance, both)


def test_problem_from_tensors():
    Q = torch.zeros(2, 5, 4, 8).transpose(1, 2)
    K = torch.zeros(2, 2, 7, 8)
    p = spdl.attention_problem(Q, K, K, Q, 0.5, dK=K)
    assert (p.batch, p.heads, p.kv_heads, p.m, p.k, p.d) == (2, 4, 2, 5, 7, 8) and p.scale == 0.5
    assert (p.Q.batch, p.Q.head, p.Q.row) == (160, 8, 32) and (p.dK.batch, p.dK.head, p.dK.row) == (112, 56, 8)
    one = K[:1].expand(2, 2, 7, 8)                       # K and V of one source for all
    assert spdl.attention_problem(Q, one, one, Q, 0.5).K.batch == 0
    for bad in (lambda: spdl.attention_problem(Q, K, K[:, :, :6], Q, 0.5), lambda: spdl.attention_problem(Q[0], K, K, Q, 0.5),
                lambda: spdl.attention_problem(Q, K.transpose(2, 3), K, Q, 0.5), lambda: spdl.attention_problem(Q, K, K, Q, 0.5, dQ=K),
                lambda: spdl.attention_problem(Q, K, K, Q, 0.5, table=torch.zeros(4, 8)),
                lambda: spdl.attention_problem(Q, K, K, Q, 0.5, table=torch.zeros(3, 8), bucket_of=torch.zeros(9, dtype=torch.int32)),
                lambda: spdl.attention_problem(Q, K, K, Q, 0.5, table=torch.zeros(4, 8), bucket_of=torch.zeros(8, dtype=torch.int32))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(ValueError):                      # not on a GPU
        spdl.spdl_attention(p, Q, K, K, None, None, None, None, None, Q, None, None)
