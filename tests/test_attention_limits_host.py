"""Attention's host side at the ends of what a problem may say."""
import pytest

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
