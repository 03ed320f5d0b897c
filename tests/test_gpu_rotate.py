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
    with pytest.raises((AssertionError, B.AlsgdError)):
        rotate(B.Rotary(2, 37, 3, 0, 64), q, k)


@pytest.mark.parametrize("given", [False, True])
def test_one_operand_alone(given):
    """Queries or keys alone, of one plan: the same bits as side by side, in either direction."""
    q, k = operand(3), operand(2, 1)
    at = torch.randint(0, 5000, (2, 37), device="cuda") if given else None
    plan = B.Rotary(2, 37, 3, 2, 64, rot=32, interleaved=True, pos0=9)
    for inverse in (False, True):
        both, alone = ([torch.full_like(q, 7.0), torch.full_like(k, 7.0)] for _ in range(2))
        plan.alsgd_rope(q, k, *both, positions=at, inverse=inverse)
        plan.alsgd_rope(q, None, alone[0], None, positions=at, inverse=inverse)
        plan.alsgd_rope(None, k, None, alone[1], positions=at, inverse=inverse)
        assert all(torch.equal(a, b) for a, b in zip(both, alone))
    with pytest.raises(AssertionError):
        plan.alsgd_rope(q, None, alone[0], alone[1])


def test_only_what_needs_a_gradient_is_turned_back():
    q, k = operand(3).requires_grad_(True), operand(2, 1).requires_grad_(True)
    plan, up = B.Rotary(2, 37, 3, 2, 64), (operand(3, 2), operand(2, 3))
    want = torch.autograd.grad(rotate(plan, q, k), (q, k), up)
    assert torch.equal(torch.autograd.grad(rotate(plan, q, k.detach())[0], q, up[0])[0], want[0])
    assert torch.equal(torch.autograd.grad(rotate(plan, q.detach(), k)[1], k, up[1])[0], want[1])
