"""The gated delta rule over sequences against the recurrence in 64 bits.

Tolerances (2-norm, relative to the result's).  Products of a chunk are
emulated FP32: operands to 2^-22, sums in FP32.  A result of t tokens went
through ceil(t / 64) chunk steps whose errors add like the roundings of
independent FP32 operations: 2^-22 (4 + sqrt(chunks)) covers a handful of
operations of 2^-23 to 2^-22 per chunk.  bfloat16 and float16 outputs are rounded once more:
2^-8 and 2^-11 at most, and float16's smallest step where values are small."""
import math

import pytest
import torch

import paper_2308_15152_amd as emu
from delta_plain import delta
from test_gpu_delta_step import dev, inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


@pytest.fixture(autouse=True)
def seeded():
    torch.manual_seed(11)


def near(got, want, tokens, dtype=torch.float32):
    got, want = got.cpu().double(), want.detach()
    assert got.shape == want.shape
    assert torch.isfinite(got).all()
    tol = 2.0 ** -22 * (4 + math.sqrt(tokens / 64)) + UNIT[dtype]
    norm = float(want.norm())
    off = float((got - want).norm())
    assert off <= tol * norm + 1e-30, (off / max(norm, 1e-300), tol)


def run(x, first, **kw):
    return emu.delta_emu_forward(*dev(*x, first), **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("b,t,hk,hv,ks,vs", [
    (1, 1, 1, 1, 64, 64), (2, 63, 1, 2, 64, 32), (1, 64, 2, 2, 128, 128), (2, 65, 1, 1, 128, 16),
    (1, 200, 1, 3, 96, 80), (3, 130, 2, 4, 33, 7), (1, 257, 1, 1, 1, 1), (1, 333, 1, 2, 128, 256),
    (2, 70, 1, 2, 100, 36)])
def test_sequences(dtype, b, t, hk, hv, ks, vs):
    x = inputs(b, t, hk, hv, ks, vs, dtype, seed=t, decay=0.2)
    for first in (None, torch.randn(b, hv, ks, vs)):
        want, last = delta(*x, first)
        o, state = run(x, first)
        near(o, want, t, dtype)
        near(state, last, t)


def test_no_tokens():
    x = inputs(2, 0, 1, 2, 16, 24, torch.float32)
    first = torch.randn(2, 2, 16, 24)
    o, state = run(x, first)
    assert o.shape == (2, 0, 2, 24) and torch.equal(state.cpu(), first)
    o, state = run(x, None)
    assert not state.any()


@pytest.mark.parametrize("lengths", [[5], [64, 0, 1, 130, 0, 63], [0, 0], [1] * 70, [200, 3]])
def test_packed(lengths):
    bounds = [0]
    for n in lengths:
        bounds.append(bounds[-1] + n)
    x = inputs(1, bounds[-1], 2, 4, 64, 48, torch.float32, seed=3, decay=0.3)
    first = torch.randn(len(lengths), 4, 64, 48)
    want, last = delta(*x, first, bounds=bounds)
    cu = torch.tensor(bounds, dtype=torch.int32, device=DEV)
    o, state = run(x, first, cu_seqlens=cu)
    near(o, want, max(lengths))
    near(state, last, max(lengths))


def test_rows_of_no_sequence():
    """Rows outside the bounds hold NaN and are neither read nor written."""
    x = list(inputs(1, 150, 1, 2, 32, 32, torch.float32, decay=0.3))
    bounds = [10, 80, 140]
    want, last = delta(*x, None, bounds=bounds)
    for y in x:
        y[:, :10] = torch.nan
        y[:, 140:] = torch.nan
    out = torch.full((1, 150, 2, 32), 7.0, device=DEV)
    cu = torch.tensor(bounds, dtype=torch.int32, device=DEV)
    o, state = run(x, None, cu_seqlens=cu, out=out)
    near(o[:, 10:140], want, 70)
    near(state, last, 70)
    assert (o[:, :10] == 7).all() and (o[:, 140:] == 7).all()


def test_one_sequence_does_not_reach_another():
    x = list(inputs(1, 100, 1, 1, 32, 16, torch.float32))
    x[2][:, 40:] = torch.nan
    bounds = [0, 40, 100]
    want, last = delta(*x, None, bounds=bounds)
    cu = torch.tensor(bounds, dtype=torch.int32, device=DEV)
    o, state = run(x, None, cu_seqlens=cu)
    near(o[:, :40], want[:, :40], 40)
    near(state[:1], last[:1], 40)
    assert o[:, 40:].isnan().all()


def test_bounds_outside_the_rows_are_clamped():
    x = inputs(1, 90, 1, 1, 32, 16, torch.float32)
    cu = torch.tensor([-5, 50, 1000], dtype=torch.int32, device=DEV)
    want, last = delta(*x, None, bounds=[0, 50, 90])
    o, state = run(x, None, cu_seqlens=cu)
    near(o, want, 50)
    near(state, last, 50)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_extreme_decays(dtype):
    """Decays of nothing, of nearly nothing and of the lowest value, at the
    ends of chunks and inside; what follows a reset does not see what was
    before."""
    x = list(inputs(1, 200, 1, 4, 64, 32, dtype, decay=0.05))
    for t in (0, 1, 63, 64, 100, 127, 128, 199):
        x[3][0, t, 0] = -torch.inf
        x[3][0, t, 1] = torch.finfo(torch.float32).min
        x[3][0, t, 2] = -100.0
    x[3][0, :, 3] = -12.0
    first = 1e3 * torch.randn(1, 4, 64, 32)
    want, last = delta(*x, first)
    o, state = run(x, first)
    for h in range(4):
        near(o[:, :, h], want[:, :, h], 200, dtype)
        near(state[:, h], last[:, h], 200)


def test_tokens_that_do_nothing():
    """beta = 0 and g = 0 leave the state; keys or values of zero too."""
    x = list(inputs(1, 140, 1, 2, 64, 32, torch.float32, decay=0.0))
    x[4][:] = 0
    first = torch.randn(1, 2, 64, 32)
    o, state = run(x, first)
    near(state, first.double(), 140)
    x = list(inputs(1, 140, 1, 2, 64, 32, torch.float32, decay=0.0))
    x[1][:] = 0
    o, state = run(x, first)
    near(state, first.double(), 140)


def test_equal_keys():
    """The triangular systems of equal keys and beta = 1 have the largest
    off-diagonal entries."""
    x = list(inputs(1, 150, 1, 1, 64, 32, torch.float32, decay=0.0))
    x[1][:] = x[1][:, :1].clone()
    x[4][:] = 1
    want, last = delta(*x, None)
    o, state = run(x, None)
    near(o, want, 150)
    near(state, last, 150)


@pytest.mark.parametrize("scale", [1e-6, 1e-3, 1e4, 1e9])
def test_values_of_any_magnitude(scale):
    x = list(inputs(1, 150, 1, 2, 64, 48, torch.float32, decay=0.1))
    x[2] *= scale
    x[2][..., 0] *= 1e-8  # columns keep their own magnitude
    first = scale * torch.randn(1, 2, 64, 48)
    want, last = delta(*x, first)
    o, state = run(x, first)
    for c in (0, slice(1, None)):
        near(o[..., c], want[..., c], 150)
    near(state, last, 150)


@pytest.mark.parametrize("size", [1e-5, 30.0])
def test_keys_of_other_lengths(size):
    x = list(inputs(1, 150, 1, 2, 64, 48, torch.float32, decay=0.1))
    x[1] *= size
    x[4] *= min(1.0, size ** -2)
    first = torch.randn(1, 2, 64, 48)
    want, last = delta(*x, first)
    o, state = run(x, first)
    near(o, want, 150)
    near(state, last, 150)


def test_strides_scale_and_in_place_state():
    x = inputs(2, 100, 2, 4, 32, 64, torch.bfloat16, decay=0.3)
    rows = torch.cat([y.flatten(2) for y in x[:3]], 2).transpose(0, 1).contiguous().to(DEV)
    q, k, v = rows.transpose(0, 1).split([64, 64, 256], 2)
    gates = torch.stack([x[3], x[4]], 0).transpose(1, 3).contiguous().to(DEV).transpose(1, 3)
    first = torch.randn(2, 4, 32, 64)
    want, last = delta(*x, first, scale=0.3)
    state = first.to(DEV)
    out = torch.empty(2, 4, 100, 64, dtype=torch.bfloat16, device=DEV).transpose(1, 2)
    o, s = emu.delta_emu_forward(q.unflatten(2, (2, 32)), k.unflatten(2, (2, 32)),
                                 v.unflatten(2, (4, 64)), gates[0], gates[1], state, scale=0.3,
                                 out=out, final_state=state)
    assert o is out and s is state
    near(o, want, 100, torch.bfloat16)
    near(state, last, 100)


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_rows_of_any_alignment(shift):
    x = inputs(1, 70, 1, 2, 64, 48, torch.bfloat16, decay=0.3)
    want, last = delta(*x, None)

    def moved(y):
        flat = torch.empty(y.numel() + shift, dtype=y.dtype, device=DEV)
        flat[shift:] = y.flatten().to(DEV)
        return flat[shift:].view(y.shape)

    out = moved(torch.zeros_like(x[2]))
    o, state = emu.delta_emu_forward(*(moved(y) for y in x), out=out)
    near(o, want, 70, torch.bfloat16)
    near(state, last, 70)


def test_same_result_again_and_on_another_stream():
    x = dev(*inputs(2, 300, 1, 4, 64, 64, torch.bfloat16, decay=0.1))
    a, sa = emu.delta_emu_forward(*x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b, sb = emu.delta_emu_forward(*x, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(a, b) and torch.equal(sa, sb)


def test_graph_replays():
    x = dev(*inputs(2, 150, 1, 2, 64, 64, torch.bfloat16, decay=0.1))
    eager, last = emu.delta_emu_forward(*x)
    out, state = torch.empty_like(eager), torch.empty_like(last)
    need = emu.delta_emu_forward_workspace(*x)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        emu.delta_emu_forward(*x, out=out, final_state=state, workspace=ws)
    for _ in range(3):
        out.zero_()
        state.zero_()
        ws.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(state, last)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("which", ["q", "k", "v", "g", "beta"])
@pytest.mark.parametrize("t,at", [(10, 4), (150, 0), (150, 21), (150, 63), (150, 64), (150, 149)])
def test_what_is_not_finite_reaches_no_earlier_token(dtype, which, t, at):
    """Nor another column, sequence or head than the recurrence takes it to."""
    x = list(inputs(2, t, 1, 2, 64, 48, dtype, seed=at, decay=0.2))
    i = ("q", "k", "v", "g", "beta").index(which)
    first = torch.randn(2, 2, 64, 48)
    for value in (torch.nan, torch.inf):
        if which == "g" and value == torch.inf:
            continue
        y = list(x)
        y[i] = x[i].clone()
        y[i][(1, at, -1, 7)[:y[i].dim()]] = value
        want, last = delta(*y, first)
        o, state = run(y, first)
        for a, b, kind in ((o, want, dtype), (state, last, torch.float32)):
            a, keep = a.cpu(), b.isfinite()
            assert torch.equal(a.isfinite(), keep), value
            near(a[keep], b[keep], t, kind)
