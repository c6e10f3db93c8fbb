"""Attention's host side at the ends of what a problem may say."""
import paper_2006_10901_amd as spdl
from tests.test_attention_host import problem


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
