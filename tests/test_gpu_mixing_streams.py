"""Token mixing calls on another stream than the current one, which is busy: what a call
allocates and fills for itself must neither come after its kernels nor be what the current
stream is still working on."""
import pytest
import torch

import paper_2308_15152_amd as emu
from test_gpu_delta_step import DEV, dev, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture
def busy():
    """Calls f on a stream of its own while the current one has some 20 ms of work."""
    a = torch.randn(8192, 8192, device=DEV).bfloat16()
    b = torch.empty_like(a)

    def run(f):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        for _ in range(20):
            torch.matmul(a, a, out=b)
        out = f(side.cuda_stream)
        side.synchronize()
        early = [x.cpu() for x in out]  # (after the current stream's work)
        return early
    return run


def check(busy, f):
    want = [x.clone() for x in f(None)]
    torch.cuda.synchronize()
    for _ in range(2):  # the second time from memory that the first gave back
        for got, w in zip(busy(f), want):
            assert torch.equal(got, w.cpu())


def test_packed_gradient(busy):
    x = dev(*inputs(1, 300, 2, 4, 64, 48, torch.bfloat16, decay=0.2))
    do = torch.randn(1, 300, 4, 48, device=DEV).bfloat16()
    cu = torch.tensor([5, 100, 100, 290], dtype=torch.int32, device=DEV)
    check(busy, lambda s: emu.delta_emu_backward(*x, do, cu_seqlens=cu, stream=s))


def test_forward(busy):
    x = dev(*inputs(2, 300, 2, 4, 64, 48, torch.bfloat16, decay=0.2))
    check(busy, lambda s: emu.delta_emu_forward(*x, stream=s))


def test_rotary_and_step(busy):
    x = dev(*inputs(3, 2, 2, 4, 64, 48, torch.float32))
    state = torch.randn(3, 4, 64, 48, device=DEV)
    states = iter([state.clone() for _ in range(3)])
    check(busy, lambda s: [emu.delta_emu_step(*x, next(states), stream=s)])
    tables = [t.clone() for t in emu.rotary_emu_table(16, 64, device=DEV)]
    check(busy, lambda s: emu.rotary_emu(x[0], x[1], *tables, stream=s))
    check(busy, lambda s: emu.rotary_emu_table(16, 64, device=DEV, stream=s))


def test_the_default_streams_handle_from_another_stream():
    x = dev(*inputs(1, 100, 1, 2, 64, 48, torch.bfloat16, decay=0.2))
    want = emu.delta_emu_forward(*x)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        got = emu.delta_emu_forward(*x, stream=0)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
