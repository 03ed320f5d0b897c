"""Whose memory a plan's workspace is: made for the stream of its first call, known to every stream that uses it.  On the host
with a stand-in for torch's allocator and for the library; on the device by what the allocator hands out."""
import contextlib
import types

import pytest
import torch

from paper_2401_09135_b200 import binding as B


class FakeTorch:
    """The parts of torch that a workspace is made with; `log` holds (what, stream)."""
    uint8 = torch.uint8

    def __init__(self):
        self.log, self.current = [], 5
        self._C = types.SimpleNamespace(_cuda_getCurrentRawStream=lambda index: self.current)
        self.cuda = types.SimpleNamespace(ExternalStream=lambda raw, device=None: types.SimpleNamespace(cuda_stream=raw),
                                          stream=self.stream)

    @contextlib.contextmanager
    def stream(self, s):
        before, self.current = self.current, s.cuda_stream
        yield
        self.current = before

    def empty(self, n, dtype=None, device=None):
        self.log.append(("made", self.current))
        return types.SimpleNamespace(data_ptr=lambda: 1000, record_stream=lambda s: self.log.append(("used", s.cuda_stream)))


def test_the_backward_workspace_knows_its_streams(monkeypatch):
    fake = FakeTorch()

    def size(desc, out):
        out._obj.value = 4096
        return B.OK
    library = types.SimpleNamespace(alsgd_attn_bwd_bytes=size, alsgd_attn_bwd=lambda *a: B.OK)
    monkeypatch.setattr(B, "lib", lambda: library)
    plan = B.Attention(1, 16, 16, 1, 1, 64)
    plan.torch = types.SimpleNamespace(**{n: getattr(fake, n) for n in ("uint8", "empty", "_C", "cuda")}, int32=None, float32=None)
    monkeypatch.setattr(plan, "_operand", lambda t, shape: None)
    monkeypatch.setattr(plan, "_plain", lambda t, shape, dtype: None)
    call = lambda raw: plan.alsgd_attn_bwd(*[None] * 9, stream=None if raw is None else types.SimpleNamespace(cuda_stream=raw))  # noqa: E731
    call(77)
    assert fake.log == [("made", 77)] and fake.current == 5
    for raw in (77, None, 77, 9, None, 9):
        call(raw)
    assert fake.log == [("made", 77), ("used", 5), ("used", 9)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["attention", "clip"])
def test_memory_in_use_on_another_stream_is_not_handed_out(kind):
    """The plan goes while its call waits on a busy stream; memory of the same size is something else's."""
    s = torch.cuda.Stream()
    if kind == "attention":
        q = torch.randn(1, 256, 2, 64, device="cuda").bfloat16()
        plan, lse = B.Attention(1, 256, 256, 2, 2, 64), torch.zeros(1, 2, 256, device="cuda")
        outs = [torch.empty_like(q) for _ in range(4)]
        call = lambda stream: plan.alsgd_attn_bwd(q, q, q, outs[3], lse, q, *outs[:3], stream=stream)  # noqa: E731
    else:
        g = torch.randn(1 << 16, device="cuda")
        plan = B.GradClip([g.numel()], [0], [torch.float32], torch.float32)
        out, stats = torch.empty_like(g), torch.zeros(2, device="cuda")
        call = lambda stream: plan.alsgd_clip_grads([g], 1.0, out, stats, stream=stream)  # noqa: E731
    call(None)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(400_000_000)
    call(s)
    at, size = plan._work._bytes.data_ptr(), plan._work._bytes.numel()
    done = torch.cuda.Event()
    done.record(s)
    del plan, call
    others = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(4)]
    assert not done.query(), "the stream was not busy for long enough"
    assert all(t.data_ptr() != at for t in others)
    torch.cuda.synchronize()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["attention", "clip"])
@pytest.mark.parametrize("where", ["default", "current", "given"])
def test_a_next_plan_takes_the_memory_of_the_last(kind, where):
    """New plans allocate nothing on the device once one has come and gone, whatever stream they are used on."""
    side = torch.cuda.Stream()
    q = torch.randn(1, 256, 2, 64, device="cuda").bfloat16()
    lse, outs, stats = torch.zeros(1, 2, 256, device="cuda"), [torch.empty_like(q) for _ in range(4)], torch.zeros(2, device="cuda")
    torch.cuda.synchronize()

    def use(stream):
        if kind == "attention":
            B.Attention(1, 256, 256, 2, 2, 64).alsgd_attn_bwd(q, q, q, outs[3], lse, q, *outs[:3], stream=stream)
        else:
            B.GradClip([q.numel()], [0], [q.dtype], torch.bfloat16).alsgd_clip_grads([q], 1.0, outs[0].view(-1), stats, stream=stream)
        torch.cuda.synchronize()

    def once():
        if where == "current":
            with torch.cuda.stream(side):
                return use(None)
        use(side if where == "given" else None)
    segments = lambda: torch.cuda.memory_stats()["segment.all.allocated"]  # noqa: E731
    for _ in range(2):
        once()
    before = segments()
    for _ in range(20):
        once()
    assert segments() == before
