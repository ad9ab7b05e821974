"""What a token mixing call allocates belongs to the stream that it runs on.

On the CPU: a stand-in for torch's streams notes on which stream every tensor is made,
filled and handed over, and the launch itself is left out."""
import contextlib

import pytest
import torch

import paper_2308_15152_amd as pkg
from paper_2308_15152_amd import mixing

CURRENT, SIDE = 111, 222


class Fake(torch.Tensor):
    """A host tensor that says it is on device 0."""

    device = torch.device("cuda", 0)

    def get_device(self):
        return 0

    def record_stream(self, stream):
        self.recorded = stream


class Torch:
    """torch with streams that only have names, and makers that note the current one."""

    def __init__(self):
        self.now, self.made = CURRENT, []
        self._C, self.cuda = self, self

    def __getattr__(self, name):
        return getattr(torch, name)

    def ExternalStream(self, handle, device=None):
        return handle

    def current_device(self):
        return 0

    def current_stream(self, device=None):
        return self.now

    def _cuda_getCurrentRawStream(self, device):
        return self.now

    @contextlib.contextmanager
    def stream(self, stream):
        before, self.now = self.now, stream
        yield
        self.now = before

    def note(self, how, t):
        t = t.as_subclass(Fake)
        self.made.append((how, self.now, t))
        return t

    def empty(self, *args, device=None, **kw):
        return self.note("empty", torch.empty(*args, **kw))

    def empty_like(self, t):
        return self.note("empty", torch.empty(t.shape, dtype=t.dtype))

    def zeros(self, *args, device=None, **kw):
        return self.note("zeros", torch.zeros(*args, **kw))


@pytest.fixture
def world(monkeypatch):
    mixing._start()
    fake = Torch()
    monkeypatch.setattr(pkg, "_torch", fake)
    monkeypatch.setattr(pkg, "_load_torch", lambda: fake)
    monkeypatch.setattr(mixing, "_device", lambda *ts: 0)
    monkeypatch.setattr(mixing, "_launch", lambda *args: None)
    return fake


def inputs():
    q = torch.zeros(1, 40, 2, 16, dtype=torch.bfloat16).as_subclass(Fake)
    v = torch.zeros(1, 40, 4, 8, dtype=torch.bfloat16).as_subclass(Fake)
    g = torch.zeros(1, 40, 4).as_subclass(Fake)
    return q, q.clone(), v, g, g.clone()


def calls(stream):
    q, k, v, g, beta = inputs()
    cu = torch.tensor([0, 10, 40], dtype=torch.int32).as_subclass(Fake)
    cos = torch.zeros(64, 4).as_subclass(Fake)
    state = torch.zeros(1, 4, 16, 8).as_subclass(Fake)
    yield "forward", pkg.delta_emu_forward(q, k, v, g, beta, stream=stream), 3
    yield "packed", pkg.delta_emu_forward(q, k, v, g, beta, cu_seqlens=cu, stream=stream), 3
    yield "backward", pkg.delta_emu_backward(q, k, v, g, beta, v, stream=stream), 7
    yield "packed back", pkg.delta_emu_backward(q, k, v, g, beta, v, cu_seqlens=cu,
                                                stream=stream), 7
    yield "step", (pkg.delta_emu_step(q, k, v, g, beta, state, stream=stream),), 1
    yield "rotary", pkg.rotary_emu(q, k, cos, cos.clone(), stream=stream), 2


def test_on_the_stream_that_is_given(world):
    for name, out, made in calls(SIDE):
        assert len(world.made) == made, name
        assert all(on == SIDE for _, on, _ in world.made), name
        assert world.now == CURRENT
        # the caller has them on the current stream
        assert all(t.recorded == CURRENT for t in out), name
        world.made.clear()


@pytest.mark.parametrize("stream", [None, CURRENT])
def test_on_the_current_stream(world, stream):
    for name, out, made in calls(stream):
        assert len(world.made) == made, name
        assert all(on == CURRENT for _, on, _ in world.made), name
        assert not any(hasattr(t, "recorded") for t in out), name
        world.made.clear()


def test_tables(world, monkeypatch):
    monkeypatch.setattr(pkg, "_on_device", lambda *ts: contextlib.nullcontext())
    c, s = pkg.rotary_emu_table(0, 8, device="cuda", stream=SIDE)  # (no rows: no launch)
    assert [on for _, on, _ in world.made] == [SIDE, SIDE]
    assert c.recorded == CURRENT and s.recorded == CURRENT
