"""Attention's host side at the ends of what a problem may say."""
import pytest
import torch

import paper_2006_10901_amd as spdl
from tests.test_attention_host import INVALID, backward, forward, problem


def test_the_forward_pass_does_not_look_at_the_strides_of_gradients():
    """Its workspace is the same whatever a problem says of tensors that it does not take."""
    for f16 in (2, 4):
        for m in (1, 9, 300):
            plain = spdl.spdl_attention_workspace(problem(m=m, k=5000), f16)
            for name in ("dO", "dQ", "dK", "dV"):
                p = problem(m=m, k=5000, **{name: (2 ** 40, 2 ** 32, 2 ** 24)})
                assert spdl.spdl_attention_workspace(p, f16) == plain, (f16, m, name)
    # the backward pass takes copies of rows that far apart
    p = problem(m=300, k=5000)
    assert spdl.spdl_attention_workspace(problem(m=300, k=5000, dO=(2 ** 40, 2 ** 32, 2 ** 24)), 2, True) > spdl.spdl_attention_workspace(p, 2, True)


def test_heads_of_k_and_v_that_no_query_head_shares_are_refused():
    """Their gradients would have to be written, and there is nothing to write them."""
    for p in (problem(heads=0, kv_heads=2), problem(heads=0, kv_heads=1, m=0), problem(heads=0, kv_heads=4, batch=0)):
        assert forward(p) == INVALID and forward(p, f16=True) == INVALID and backward(p) == INVALID
        with pytest.raises(spdl.SpdlError):
            spdl.spdl_attention_workspace(p, 4, True)


def test_a_mask_from_arrays_that_are_too_short_is_refused():
    """Before anything reads them: the topology has m + 1 offsets and nnz columns."""
    n = spdl.spdl_attention_mask_bytes(64, 100)
    ints = lambda count: torch.zeros(count, dtype=torch.int32)
    good = (64, 100, 10, ints(65), ints(10), torch.zeros(n, dtype=torch.uint8))
    with pytest.raises(ValueError, match="GPU tensor"):
        spdl.spdl_build_attention_mask(*good)            # not on a GPU
    for at, short, name in ((3, ints(64), "row_offsets"), (4, ints(9), "column_indices"), (5, torch.zeros(n - 1, dtype=torch.uint8), "mask")):
        with pytest.raises(ValueError, match=name + " is too short"):
            spdl.spdl_build_attention_mask(*good[:at], short, *good[at + 1:])
    for at in (3, 4, 5):
        with pytest.raises(ValueError):
            spdl.spdl_build_attention_mask(*good[:at], None, *good[at + 1:])
