"""The gated delta rule's gradient against the recurrence's in 64 bits.

Tolerances (2-norm, relative to the result's).  A gradient goes through the
walk forward, the walk back and a dozen products of a chunk, each with a few
FP32-like roundings (2^-23 to 2^-22), which add like independent ones: 2^-22 (8
+ 2 sqrt(chunks)); 16-bit results are rounded once more.  dg sums over a chunk's later
tokens terms q.dq and k.dk that largely cancel, so its error goes with those:
the same factor of its own norm plus 8 (= sqrt 64) times theirs.  dinitial is a
sum over tokens of scale q do^T and -k dv^T (as it leaves a chunk), whose
rounding goes with the norm of the terms where they cancel to a few values:
that norm is added to its own; likewise for dbeta, a difference of sums of
dY v and K (S dY) over the value's elements, the norm of the terms dY v (dY = dv /
beta)."""
import math

import pytest
import torch

import paper_2308_15152_amd as emu
from delta_plain import delta, delta_gradients
from test_gpu_delta_step import dev, inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
NAMES = ("dq", "dk", "dv", "dg", "dbeta", "dinitial")


@pytest.fixture(autouse=True)
def seeded():
    torch.manual_seed(11)


def check(got, want, x, do, tokens, dtype):
    q, k = x[0].double(), x[1].double()
    c = 2.0 ** -22 * (8 + 2 * math.sqrt(tokens / 64))
    terms = ((q * want[0]).sum(-1).abs() + (k * want[1]).sum(-1).abs()).norm()
    for name, a, b in zip(NAMES, got, want):
        if b is None:
            assert a is None, name
            continue
        a = a.cpu().double()
        assert a.shape == b.shape and torch.isfinite(a).all(), name
        rounded = name in ("dq", "dk", "dv")
        tol = (c + (UNIT[dtype] if rounded else 2.0 ** -24)) * float(b.norm())
        if name == "dg":
            tol += c * 8 * float(terms)
        if name == "dinitial" and tokens > 0:
            size = x[0].shape[-1] ** -0.5
            tol += c * math.hypot(size * float(do.double().norm() * q.norm(dim=-1).max()),
                                  float(want[2].norm() * k.norm(dim=-1).max()))
        if name == "dbeta" and tokens > 0:
            dy = want[2] / x[4].double().clamp_min(1e-3)[..., None]
            tol += c * float((dy * x[2].double()).norm())
        if rounded and dtype == torch.float16:
            tol += 2.0 ** -25 * math.sqrt(b.numel())
        off = float((a - b).norm())
        norm = max(float(b.norm()), 1e-300)
        assert off <= tol + 1e-30, (name, off / norm, tol / norm)


def gradients(x, do, first, dfinal, **kw):
    return emu.delta_emu_backward(*dev(*x, do, first, dfinal), **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("b,t,hk,hv,ks,vs", [
    (1, 1, 1, 1, 64, 64), (2, 63, 1, 2, 64, 32), (1, 64, 2, 2, 128, 128), (2, 65, 1, 1, 128, 16),
    (1, 200, 1, 3, 96, 80), (3, 130, 2, 4, 33, 7), (1, 140, 1, 1, 1, 1), (1, 200, 1, 2, 128, 256),
    (2, 70, 1, 2, 100, 36)])
def test_sequences(dtype, b, t, hk, hv, ks, vs):
    x = inputs(b, t, hk, hv, ks, vs, dtype, seed=t, decay=0.2)
    do = torch.randn(b, t, hv, vs).to(dtype)
    for first, dfinal in ((None, None), (torch.randn(b, hv, ks, vs), torch.randn(b, hv, ks, vs))):
        want = delta_gradients(*x, do, first, dfinal)
        check(gradients(x, do, first, dfinal), want, x, do, t, dtype)


def test_against_differences():
    """Directional differences of the forward recurrence in 64 bits."""
    x = inputs(1, 90, 1, 2, 32, 24, torch.float32, seed=5, decay=0.2)
    first, do = torch.randn(1, 2, 32, 24), torch.randn(1, 90, 2, 24)
    dfinal = torch.randn(1, 2, 32, 24)
    got = gradients(x, do, first, dfinal)
    names = [*x, first]
    for i in range(6):
        way, h = torch.randn_like(names[i], dtype=torch.float64), 1e-5
        ends = []
        for s in (h, -h):
            y = [z.double() + (s * way if j == i else 0) for j, z in enumerate(names)]
            o, last = delta(*y)
            ends.append(float((o * do).sum() + (last * dfinal).sum()))
        slope = (ends[0] - ends[1]) / (2 * h)
        d = got[i].cpu().double()
        # 2^-20 of the terms' norm, and the differences' own 1e-10-ish
        assert abs(float((d * way).sum()) - slope) < 2.0 ** -20 * float((d * way).norm()) * 8 + 1e-5, i


@pytest.mark.parametrize("lengths", [[5], [64, 0, 1, 130, 0, 63], [0, 0], [1] * 70, [200, 3]])
def test_packed(lengths):
    bounds = [0]
    for n in lengths:
        bounds.append(bounds[-1] + n)
    x = inputs(1, bounds[-1], 2, 4, 64, 48, torch.float32, seed=3, decay=0.3)
    n = len(lengths)
    first, dfinal = torch.randn(n, 4, 64, 48), torch.randn(n, 4, 64, 48)
    do = torch.randn(1, bounds[-1], 4, 48)
    want = delta_gradients(*x, do, first, dfinal, bounds=bounds)
    cu = torch.tensor(bounds, dtype=torch.int32, device=DEV)
    check(gradients(x, do, first, dfinal, cu_seqlens=cu), want, x, do, max(lengths),
          torch.float32)


def test_rows_of_no_sequence():
    x = list(inputs(1, 150, 1, 2, 32, 32, torch.float32, decay=0.3))
    do = torch.randn(1, 150, 2, 32)
    bounds = [10, 80, 140]
    want = delta_gradients(*(y[:, 10:140] for y in x), do[:, 10:140], None, None,
                           bounds=[0, 70, 130])
    for y in (*x, do):
        y[:, :10] = torch.nan
        y[:, 140:] = torch.nan
    cu = torch.tensor(bounds, dtype=torch.int32, device=DEV)
    got = gradients(x, do, None, None, cu_seqlens=cu)
    for d in got[:5]:
        assert not d[:, :10].any() and not d[:, 140:].any()
    inside = [d[:, 10:140] for d in got[:5]] + [got[5]]
    check(inside, want, [y[:, 10:140] for y in x], do[:, 10:140], 70, torch.float32)


def test_no_tokens():
    x = inputs(2, 0, 1, 2, 16, 24, torch.float32)
    dfinal = torch.randn(2, 2, 16, 24)
    got = gradients(x, torch.zeros(2, 0, 2, 24), None, dfinal)
    assert torch.equal(got[5].cpu(), dfinal)


@pytest.mark.parametrize("lengths", [None, [1, 1, 1, 1, 1]])
def test_first_tokens_without_a_state_have_no_decay_gradient(lengths):
    """Nothing decays there: exactly zero."""
    cu = None
    x = inputs(5, 1, 1, 2, 64, 32, torch.bfloat16)
    do = torch.randn(5, 1, 2, 32).bfloat16()
    if lengths:
        x, do = [y.transpose(0, 1) for y in x], do.transpose(0, 1)
        cu = torch.tensor([0, 1, 2, 3, 4, 5], dtype=torch.int32, device=DEV)
    got = gradients(x, do, None, None, cu_seqlens=cu)
    assert not got[3].any() and got[4].abs().min() > 0


def test_without_decay_or_strength():
    x = inputs(1, 100, 1, 2, 32, 32, torch.float32)[:3]
    x = (x[0], 0.3 * x[1], x[2], None, None)
    do = torch.randn(1, 100, 2, 32)
    want = delta_gradients(*x, do, None, None, scale=0.7)
    check(gradients(x, do, None, None, scale=0.7), want, x, do, 100, torch.float32)


def test_strength_of_zero_has_a_gradient():
    x = list(inputs(1, 100, 1, 2, 32, 32, torch.float32, decay=0.2))
    x[4][:, ::3] = 0
    do = torch.randn(1, 100, 2, 32)
    want = delta_gradients(*x, do, None, None)
    assert want[4][:, ::3].abs().min() > 0
    check(gradients(x, do, None, None), want, x, do, 100, torch.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_extreme_decays(dtype):
    x = list(inputs(1, 200, 1, 4, 64, 32, dtype, decay=0.05))
    for t in (0, 1, 63, 64, 100, 127, 128, 199):
        x[3][0, t, 0] = -torch.inf
        x[3][0, t, 1] = torch.finfo(torch.float32).min
        x[3][0, t, 2] = -100.0
    x[3][0, :, 3] = -12.0
    first, do = torch.randn(1, 4, 64, 32), torch.randn(1, 200, 4, 32).to(dtype)
    y = list(x)
    y[3] = x[3].clamp_min(-200.0)  # the plain gradient at -infinity is 0 times infinity
    want = delta_gradients(*y, do, first, None)
    check(gradients(x, do, first, None), want, x, do, 200, dtype)


@pytest.mark.parametrize("scale", [1e-12, 1e-6, 1e5])
def test_gradients_of_any_magnitude(scale):
    x = inputs(1, 150, 1, 2, 64, 48, torch.float32, decay=0.1)
    do = scale * torch.randn(1, 150, 2, 48)
    want = delta_gradients(*x, do, None, None)
    check(gradients(x, do, None, None), want, x, do, 150, torch.float32)


def test_strides_and_given_outputs():
    x = inputs(2, 100, 2, 4, 32, 64, torch.bfloat16, decay=0.3)
    do = torch.randn(2, 100, 4, 64).bfloat16()
    first, dfinal = torch.randn(2, 4, 32, 64), torch.randn(2, 4, 32, 64)
    want = delta_gradients(*x, do, first, dfinal)
    rows = torch.cat([y.flatten(2) for y in x[:3]], 2).transpose(0, 1).contiguous().to(DEV)

    def parts(r):
        q, k, v = r.transpose(0, 1).split([64, 64, 256], 2)
        return q.unflatten(2, (2, 32)), k.unflatten(2, (2, 32)), v.unflatten(2, (4, 64))

    grads = parts(torch.zeros_like(rows))
    gates = torch.zeros(2, 4, 2, 100, device=DEV).permute(2, 0, 3, 1)
    state = dfinal.to(DEV)
    out = (*grads, gates[0], gates[1], state)
    do_ = do.transpose(1, 2).contiguous().to(DEV).transpose(1, 2)
    got = emu.delta_emu_backward(*parts(rows), *dev(*x[3:]), do_, first.to(DEV), state, out=out)
    assert all(a is b for a, b in zip(got, out))
    check(got, want, x, do, 100, torch.bfloat16)


@pytest.mark.parametrize("shift", [1, 3])
def test_rows_of_any_alignment(shift):
    x = inputs(1, 70, 1, 2, 64, 48, torch.bfloat16, decay=0.3)
    do = torch.randn(1, 70, 2, 48).bfloat16()
    want = delta_gradients(*x, do, None, None)

    def moved(y):
        flat = torch.empty(y.numel() + shift, dtype=y.dtype, device=DEV)
        flat[shift:] = y.flatten().to(DEV)
        return flat[shift:].view(y.shape)

    got = emu.delta_emu_backward(*(moved(y) for y in (*x, do)))
    check(got, want, x, do, 70, torch.bfloat16)


def test_same_result_again_on_another_stream_and_in_a_graph():
    x = dev(*inputs(2, 300, 1, 4, 64, 64, torch.bfloat16, decay=0.1))
    do = torch.randn(2, 300, 4, 64, device=DEV).bfloat16()
    a = emu.delta_emu_backward(*x, do)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b = emu.delta_emu_backward(*x, do, stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(c, d) for c, d in zip(a, b))
    out = [torch.empty_like(c) for c in a]
    ws = torch.empty(emu.delta_emu_backward_workspace(*x), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        emu.delta_emu_backward(*x, do, out=out, workspace=ws)
    for _ in range(3):
        for c in out:
            c.zero_()
        ws.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(c, d) for c, d in zip(a, out))
