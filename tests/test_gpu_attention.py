"""Attention in one call and its gradients against the definition in 64 bits, at the sizes, masks and layouts where a tile, a block of
keys or a split of the work can go wrong."""
import pytest
import torch

from tests.attention_util import Case, banded, blocks, causal, nothing, sparse_rows

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
