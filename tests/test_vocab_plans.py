"""binding.VocabLoss and binding.Rotary on the host, with a stand-in for the library: whose memory a workspace is, calls of
several threads, and which descriptor a call goes out with."""
import threading
import types

import pytest
import torch

from paper_2401_09135_b200 import binding as B
from test_plan_threads import both
from test_workspaces import FakeTorch


class Library:
    def __init__(self):
        self.inside = self.most = 0
        self.lock, self.second = threading.Lock(), threading.Event()
        self.sizes, self.ropes = [], []

    def alsgd_vocab_bytes(self, desc, backward, out):
        out._obj.value = 4096 * (1 + backward)
        return B.OK

    def enter(self, *args):
        with self.lock:
            self.inside += 1
            self.most = max(self.most, self.inside)
            if self.inside > 1:
                self.second.set()
        self.second.wait(0.2)
        with self.lock:
            self.inside -= 1
        self.sizes.append(args[-2])
        return B.OK

    alsgd_xent_fwd = alsgd_xent_bwd = alsgd_distill_fwd = alsgd_distill_bwd = enter

    def alsgd_rope(self, desc, *args):
        self.ropes.append((desc.flags, desc.position_dtype))
        return B.OK


def plan_with(monkeypatch, fake=None, **kw):
    library = Library()
    monkeypatch.setattr(B, "lib", lambda: library)
    plan = B.VocabLoss(8, 100, 16, **kw)
    if fake is not None:
        plan.torch = types.SimpleNamespace(**{n: getattr(fake, n) for n in ("uint8", "empty", "_C", "cuda")})
    monkeypatch.setattr(plan, "_matrix", lambda slot, t, shape: None)
    monkeypatch.setattr(plan, "_plain", lambda t, shape, dtype: None)
    return library, plan


def test_workspaces_know_their_streams(monkeypatch):
    fake = FakeTorch()
    library, plan = plan_with(monkeypatch, fake)
    library.second.set()
    call = lambda raw: plan.alsgd_xent_fwd(*[None] * 5, stream=None if raw is None else types.SimpleNamespace(cuda_stream=raw))  # noqa: E731
    call(77)
    assert fake.log == [("made", 77)] and fake.current == 5
    for raw in (77, None, 9, 9):
        call(raw)
    assert fake.log == [("made", 77), ("used", 5), ("used", 9)]
    assert library.sizes == [4096] * 5


def test_calls_of_two_threads_go_out_one_by_one(monkeypatch):
    library, plan = plan_with(monkeypatch, top=3)
    monkeypatch.setattr(B, "_stream", lambda *a: 0)
    monkeypatch.setattr(B, "_Workspace", lambda torch, n, *a, **k: types.SimpleNamespace(ptr=1 << 20, nbytes=n, used_on=lambda raw: None))
    both(*[lambda: plan.alsgd_distill_fwd(*[None] * 6)] * 2)
    assert library.most == 1 and library.sizes == [4096] * 2


def test_rotary_directions_and_types_have_descriptors_of_their_own(monkeypatch):
    library = Library()
    monkeypatch.setattr(B, "lib", lambda: library)
    monkeypatch.setattr(B, "_stream", lambda *a: 0)
    plan = B.Rotary(2, 5, 2, 1, 16, interleaved=True)
    monkeypatch.setattr(plan, "_operand", lambda slot, t, shape: slot)
    for inverse in (False, True):
        for dtype in (None, torch.int32, torch.int64):
            at = None if dtype is None else types.SimpleNamespace(shape=(2, 5), is_contiguous=lambda: True, get_device=lambda: 0, dtype=dtype, data_ptr=lambda: 0)
            plan.alsgd_rope(*[None] * 4, positions=at, inverse=inverse)
    assert library.ropes == [(1, B.I32), (1, B.I32), (1, B.I64), (3, B.I32), (3, B.I32), (3, B.I64)]


def test_types_that_are_not_taken(monkeypatch):
    for kw in (dict(index_dtype=torch.int16), dict(teacher_dtype=torch.float16, top=2)):
        with pytest.raises(B.AlsgdError):
            B.VocabLoss(8, 100, 16, **kw)
    with pytest.raises(B.AlsgdError):
        B.Rotary(1, 1, 1, 1, 8, dtype=torch.float16)
