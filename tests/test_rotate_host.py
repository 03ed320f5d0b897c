"""rotate() on the host with a stand-in for the plan: what it asks the plan for."""
import torch

from paper_2401_09135_b200.rotary import rotate


class Plan:
    """Doubles what it is given, and keeps which operands came."""

    def __init__(self):
        self.calls = []

    def alsgd_rope(self, q, k, q_out, k_out, positions=None, inverse=False):
        assert (q is None) == (q_out is None) and (k is None) == (k_out is None)
        self.calls.append((inverse, q is not None, k is not None))
        for t, out in ((q, q_out), (k, k_out)):
            if t is not None:
                out.copy_(2 * t)


def test_without_key_heads():
    plan, q = Plan(), torch.randn(1, 3, 2, 8, requires_grad=True)
    got, none = rotate(plan, q, None)
    assert none is None and torch.equal(got, 2 * q)
    up = torch.randn_like(got)
    assert torch.equal(torch.autograd.grad(got, q, up)[0], 2 * up)
    assert plan.calls == [(False, True, False), (True, True, False)]


def test_only_what_needs_a_gradient_is_turned_back():
    for needs in ((True, False), (False, True), (True, True)):
        plan = Plan()
        q, k = (torch.randn(1, 3, h, 8, requires_grad=n) for h, n in zip((2, 1), needs))
        outs = [t for t, n in zip(rotate(plan, q, k), needs) if n]
        ups = [torch.randn_like(t) for t in outs]
        got = torch.autograd.grad(outs, [t for t, n in zip((q, k), needs) if n], ups)
        assert all(torch.equal(a, 2 * b) for a, b in zip(got, ups))
        assert plan.calls == [(False, True, True), (True,) + needs]
