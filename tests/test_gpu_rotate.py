"""rotate() in the forms that a caller needs besides queries and keys together."""
import pytest
import torch

from paper_2401_09135_b200 import binding as B
from paper_2401_09135_b200.rotary import rotate

pytestmark = pytest.mark.gpu


def operand(heads, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(2, 37, heads, 64, generator=g, device="cuda").bfloat16()


def test_without_key_heads():
    """The same bits as queries beside keys, results and gradients."""
    q, k, up = operand(3).requires_grad_(True), operand(2, 1), operand(3, 2)
    want, _ = rotate(B.Rotary(2, 37, 3, 2, 64, pos0=5), q, k)
    got, none = rotate(B.Rotary(2, 37, 3, 0, 64, pos0=5), q, None)
    assert none is None and torch.equal(got, want)
    assert torch.equal(torch.autograd.grad(got, q, up)[0], torch.autograd.grad(want, q, up)[0])
    with torch.no_grad():
        assert torch.equal(rotate(B.Rotary(2, 37, 3, 0, 64, pos0=5), q, None)[0], want)
    with pytest.raises(AssertionError):
        rotate(B.Rotary(2, 37, 3, 0, 64), q, k)
