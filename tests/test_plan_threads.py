"""Two threads that call one plan at once: each call is enqueued as a whole, with its own tensors.  On the host, with a stand-in for
the library that lets a second call begin, as ctypes does by releasing the interpreter's lock."""
import threading
import types

import torch

from paper_2401_09135_b200 import binding as B


class Library:
    def __init__(self):
        self.inside, self.most, self.seen = 0, 0, []
        self.lock, self.second = threading.Lock(), threading.Event()

    def alsgd_clip_grads_bytes(self, n, out):
        out._obj.value = 4096
        return B.OK

    def alsgd_attn_bwd_bytes(self, desc, out):
        out._obj.value = 4096
        return B.OK

    def enter(self):
        with self.lock:
            self.inside += 1
            self.most = max(self.most, self.inside)
            if self.inside > 1:
                self.second.set()
        self.second.wait(0.3)                    # time for the other thread to come in
        with self.lock:
            self.inside -= 1

    def alsgd_clip_grads(self, desc, n, max_norm, *rest):
        self.enter()
        self.seen.append((max_norm, desc[0].data))
        return B.OK

    def alsgd_attn_bwd(self, *args):
        self.enter()
        return B.OK


def both(*calls):
    threads = [threading.Thread(target=c) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()


def setup(monkeypatch):
    library, made = Library(), []

    def workspace(*a, **k):
        made.append(1)
        return types.SimpleNamespace(ptr=1 << 20, nbytes=4096, used_on=lambda raw: None)
    monkeypatch.setattr(B, "lib", lambda: library)
    monkeypatch.setattr(B, "_stream", lambda *a: 0)
    monkeypatch.setattr(B, "_Workspace", workspace)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(synchronize=lambda: None))
    return library, made


def test_clip_hands_over_its_own_tensors(monkeypatch):
    library, _ = setup(monkeypatch)
    plan = B.GradClip([8], [0], [torch.float32], torch.float32)
    plan._index = -1                             # host tensors
    grads, stats = [torch.zeros(8) for _ in range(2)], torch.zeros(2)
    both(*[lambda g=g, m=m: plan.alsgd_clip_grads([g], m, None, stats) for g, m in zip(grads, (1.0, 2.0))])
    assert sorted(library.seen) == sorted((m, g.data_ptr()) for g, m in zip(grads, (1.0, 2.0)))
    assert library.most == 1


def test_backward_calls_do_not_mix(monkeypatch):
    """They share the workspace that delta and the partial sums of the table go through."""
    library, made = setup(monkeypatch)
    plan = B.Attention(1, 16, 16, 1, 1, 64)
    monkeypatch.setattr(plan, "_operand", lambda t, shape: None)
    monkeypatch.setattr(plan, "_plain", lambda t, shape, dtype: None)
    both(*[lambda: plan.alsgd_attn_bwd(*[None] * 9)] * 2)
    assert library.most == 1 and made == [1]
