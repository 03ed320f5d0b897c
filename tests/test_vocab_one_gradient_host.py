"""What a backward pass of one gradient is refused for; nothing is launched."""
import pytest

from paper_2401_09135_b200 import binding as B
from test_ops_host_decoder import PTR, matrix, vocab_desc


def call(name, dx, dw, work_bytes=0):
    top = 5 if name == "distill_bwd" else 0
    labels = (PTR, PTR) if top else (PTR,)
    m = matrix()
    return getattr(B.lib(), "alsgd_" + name)(vocab_desc(top=top), m, m, *labels, PTR, PTR, 1, dx, dw, PTR, work_bytes, None)


@pytest.mark.parametrize("name", ["xent_bwd", "distill_bwd"])
def test_one_gradient_is_checked_and_enough(name):
    to = matrix(2 * PTR)
    assert call(name, None, None) == B.E_ARG
    # a workspace that is too small is the last thing found
    assert call(name, to, None) == B.E_NOMEM and call(name, None, to) == B.E_NOMEM
    assert call(name, matrix(None), None) == B.E_ARG and call(name, None, matrix(None)) == B.E_ARG
    assert call(name, matrix(), None) == B.E_ARG and call(name, None, matrix()) == B.E_ARG
    assert call(name, matrix(2 * PTR, 56), None) == B.E_ARG and call(name, None, matrix(2 * PTR, 56)) == B.E_ARG
