"""Batches that fill the device.  Walks of more than 128 blocks of 32 columns take kernels of
their own (32 columns a block and more helping waves), as do sequences cut into parts in a batch of
several.  A few sequences are repeated over the batch in mixed order, so that the recurrence in
64 bits is computed for those only, and copies have to be equal.  Tolerances: those of
test_gpu_delta_forward.py, test_gpu_delta_backward.py and test_gpu_delta_long.py."""
import pytest
import torch

import paper_2308_15152_amd as emu
from delta_plain import delta, delta_gradients
from test_gpu_delta_backward import check, gradients
from test_gpu_delta_forward import near, run
from test_gpu_delta_long import near_long
from test_gpu_delta_step import DEV, inputs

pytestmark = pytest.mark.gpu

# tokens, key heads, value heads, key size, value size, copies
SHAPES = [(200, 2, 4, 64, 80, 14), (200, 1, 2, 128, 80, 24), (140, 2, 2, 96, 36, 40),
          (260, 1, 3, 33, 64, 30), (257, 2, 2, 128, 128, 20)]


@pytest.fixture(autouse=True)
def seeded():
    torch.manual_seed(11)


def order(copies, distinct):
    """Which sequence each of the batch is: the distinct ones first, then any."""
    g = torch.Generator().manual_seed(copies)
    return torch.cat([torch.arange(distinct),
                      torch.randint(0, distinct, (copies - distinct,), generator=g)])


def spread(ys, which, shift=0):
    """The batch on the device; with shift, its rows not at multiples of 16 bytes."""
    out = []
    for y in ys:
        z = y[which]
        flat = torch.empty(z.numel() + shift, dtype=z.dtype, device=DEV)
        flat[shift:] = z.flatten().to(DEV)
        out.append(flat[shift:].view(z.shape))
    return out


def gathered(ys, which, distinct):
    """The distinct sequences' results; all copies must be equal."""
    for y in ys:
        assert torch.equal(y, y[:distinct][which.to(DEV)])
    return [y[:distinct] for y in ys]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("shift", [0, 1])
def test_forward(dtype, shape, shift):
    t, hk, hv, ks, vs, copies = shape
    assert copies * hv * -(-vs // 32) > 128 and t > 128
    x = inputs(2, t, hk, hv, ks, vs, dtype, seed=t, decay=0.2)
    first = torch.randn(2, hv, ks, vs)
    which = order(copies, 2)
    got = emu.delta_emu_forward(*spread(x, which, shift), first[which].to(DEV))
    o, state = gathered(got, which, 2)
    want, last = delta(*x, first)
    near(o, want, t, dtype)
    near(state, last, t)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("shift", [0, 1])
def test_gradient(dtype, shape, shift):
    t, hk, hv, ks, vs, copies = shape
    x = inputs(2, t, hk, hv, ks, vs, dtype, seed=t, decay=0.2)
    do = torch.randn(2, t, hv, vs).to(dtype)
    first, dfinal = torch.randn(2, hv, ks, vs), torch.randn(2, hv, ks, vs)
    which = order(copies, 2)
    got = emu.delta_emu_backward(*spread((*x, do), which, shift), first[which].to(DEV),
                                 dfinal[which].to(DEV))
    got = gathered(got, which, 2)
    check(got, delta_gradients(*x, do, first, dfinal), x, do, t, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_packed(dtype):
    """Sequences of 0 to 200 tokens, in mixed order; every sequence's copies are equal."""
    lengths = [200, 1, 64, 130, 0, 65]
    which = order(40, 6)
    bounds, parts = [0], []
    for n in lengths:
        bounds.append(bounds[-1] + n)
    x = inputs(1, bounds[-1], 2, 2, 64, 80, dtype, seed=3, decay=0.3)
    do = torch.randn(1, bounds[-1], 2, 80).to(dtype)
    first, dfinal = torch.randn(6, 2, 64, 80), torch.randn(6, 2, 64, 80)
    rows = torch.cat([torch.arange(bounds[i], bounds[i + 1]) for i in which.tolist()])
    ends = torch.cat([torch.zeros(1, dtype=torch.long),
                      torch.tensor([lengths[i] for i in which]).cumsum(0)])
    cu = ends.int().to(DEV)
    y = [z[:, rows].to(DEV) for z in (*x, do)]
    o, state = emu.delta_emu_forward(*y[:5], first[which].to(DEV), cu_seqlens=cu)
    want, last = delta(*x, first, bounds=bounds)
    assert torch.equal(o, o[:, :bounds[-1]][:, rows.to(DEV)])
    near(o[:, :bounds[-1]], want, 200, dtype)
    state, = gathered([state], which, 6)
    near(state, last, 200)
    got = emu.delta_emu_backward(*y, first[which].to(DEV), dfinal[which].to(DEV), cu_seqlens=cu)
    for z in got[:5]:
        assert torch.equal(z, z[:, :bounds[-1]][:, rows.to(DEV)])
    dinitial, = gathered(got[5:], which, 6)
    check([*(z[:, :bounds[-1]] for z in got[:5]), dinitial],
          delta_gradients(*x, do, first, dfinal, bounds=bounds), x, do, 200, dtype)


def test_parts_of_several_sequences():
    b, t, ks, vs = 3, 4500, 64, 48
    x = inputs(b, t, 1, 1, ks, vs, torch.bfloat16, seed=2, decay=0.05)
    first, dfinal = torch.randn(b, 1, ks, vs), torch.randn(b, 1, ks, vs)
    do = torch.randn(b, t, 1, vs).bfloat16()
    # cut: more workspace than chunks' records alone (many heads are not)
    need = emu.delta_emu_forward_workspace(*x)
    wide = [y.expand(b, t, 64, *y.shape[3:]) for y in x]
    assert need > emu.delta_emu_forward_workspace(*wide) / 64
    want, last = delta(*x, first)
    o, state = run(x, first)
    near_long(o, want, t, torch.bfloat16)
    near_long(state, last, t)
    check(gradients(x, do, first, dfinal), delta_gradients(*x, do, first, dfinal), x, do, 4 * t,
          torch.bfloat16)
