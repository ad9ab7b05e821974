"""What an attention call allocates belongs to the stream that it runs on (with the stand-in
for torch's streams of test_mixing_streams_cpu.py)."""
import pytest
import torch

import paper_2308_15152_amd as pkg
from paper_2308_15152_amd import attention
from test_mixing_streams_cpu import CURRENT, SIDE, Fake, Torch


@pytest.fixture
def world(monkeypatch):
    attention._start()
    fake = Torch()
    monkeypatch.setattr(pkg, "_torch", fake)
    monkeypatch.setattr(pkg, "_load_torch", lambda: fake)
    monkeypatch.setattr(attention, "_device", lambda *ts: 0)
    monkeypatch.setattr(attention, "_launch", lambda *args: None)
    return fake


def zeros(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(Fake)


def calls(stream):
    """(name, results, tensors made: results and workspace)."""
    q, k, lse = zeros(1, 40, 4, 16), zeros(1, 40, 2, 16), zeros(1, 40, 4, dtype=torch.float32)
    cu = torch.tensor([0, 10, 40], dtype=torch.int32).as_subclass(Fake)
    long = zeros(1, 9000, 2, 16)
    lengths = zeros(1, dtype=torch.int32)
    yield "forward", pkg.attention_emu_forward(q, k, k, stream=stream), 2
    yield "long", pkg.attention_emu_forward(q, long, long, stream=stream), 3
    yield "packed", pkg.attention_emu_forward(q, k, k, cu_seqlens=cu, stream=stream), 2
    yield "backward", pkg.attention_emu_backward(q, k, k, q, lse, q, stream=stream), 4
    yield "packed back", pkg.attention_emu_backward(q, k, k, q, lse, q, cu_seqlens=cu,
                                                    stream=stream), 4
    yield "step", (pkg.attention_emu_step(q[:, :1], k, k, lengths, stream=stream),), 1
    yield "prefix", (pkg.attention_emu_step(q[:, :1], k, k, lengths, long, long,
                                            stream=stream),), 2


def test_on_the_stream_that_is_given(world):
    for name, out, made in calls(SIDE):
        assert len(world.made) == made, name
        assert all(on == SIDE for _, on, _ in world.made), name
        assert world.now == CURRENT
        assert all(t.recorded == CURRENT for t in out), name
        world.made.clear()


@pytest.mark.parametrize("stream", [None, CURRENT])
def test_on_the_current_stream(world, stream):
    for name, out, made in calls(stream):
        assert len(world.made) == made, name
        assert all(on == CURRENT for _, on, _ in world.made), name
        assert not any(hasattr(t, "recorded") for t in out), name
        world.made.clear()
