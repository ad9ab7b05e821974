"""Long sequences of few heads, which are cut into parts that run side by side,
sequences about the length up to which tokens go one by one, and views whose
offsets pass 32 bits, against the recurrence in 64 bits.

Tolerances: those of whole sequences (test_gpu_delta_forward.py), with twice the
chunk steps and four more operations: a part's state comes from its
predecessor's through the part's own transition, a walk of as many chunks.
For gradients the same of test_gpu_delta_backward.py's bounds, whose count of tokens is
taken four times (the bounds grow with its root)."""
import math

import pytest
import torch

import paper_2308_15152_amd as emu
from delta_plain import delta, delta_gradients
from test_gpu_delta_backward import check, gradients
from test_gpu_delta_forward import UNIT, near
from test_gpu_delta_step import DEV, dev, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def seeded():
    torch.manual_seed(11)


def near_long(got, want, tokens, dtype=torch.float32):
    got, want = got.cpu().double(), want.detach()
    assert got.shape == want.shape and torch.isfinite(got).all()
    tol = 2.0 ** -22 * (8 + 2 * math.sqrt(tokens / 64)) + UNIT[dtype]
    assert float((got - want).norm()) <= tol * float(want.norm())


def test_long_sequences_take_more_workspace_than_their_chunks():
    """The sequences below are cut: their workspace holds more than the chunks'
    records, which grow in proportion to the tokens."""
    def need(t, heads):
        q, v = torch.empty(1, t, heads, 64), torch.empty(1, t, heads, 64)
        g = torch.empty(1, t, heads)
        return emu.delta_emu_forward_workspace(q, q, v, g, g)
    assert need(4500, 1) > need(4544, 64) / 64


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("t,hk,hv,ks,vs,decay", [
    (4500, 1, 1, 64, 64, 0.02), (4097, 1, 2, 128, 48, 0.2), (6000, 1, 1, 33, 20, 0.0)])
def test_parts(dtype, t, hk, hv, ks, vs, decay):
    x = inputs(1, t, hk, hv, ks, vs, dtype, seed=t, decay=decay)
    for first in (None, torch.randn(1, hv, ks, vs)):
        want, last = delta(*x, first)
        o, state = emu.delta_emu_forward(*dev(*x, first))
        near_long(o, want, t, dtype)
        near_long(state, last, t)


@pytest.mark.parametrize("lengths", [[4500, 4000], [9000, 3], [0, 8192], [64, 6000, 1]])
def test_packed_parts(lengths):
    bounds = [0]
    for n in lengths:
        bounds.append(bounds[-1] + n)
    x = inputs(1, bounds[-1], 1, 1, 64, 32, torch.float32, seed=3, decay=0.05)
    first = torch.randn(len(lengths), 1, 64, 32)
    cu = torch.tensor(bounds, dtype=torch.int32, device=DEV)
    want, last = delta(*x, first, bounds=bounds)
    o, state = emu.delta_emu_forward(*dev(*x, first), cu_seqlens=cu)
    near_long(o, want, max(lengths))
    near_long(state, last, max(lengths))


def test_a_reset_inside_a_part():
    x = list(inputs(1, 5000, 1, 1, 64, 32, torch.float32, decay=0.01))
    x[3][0, 2500] = -torch.inf
    first = 1e4 * torch.randn(1, 1, 64, 32)
    want, last = delta(*x, first)
    o, state = emu.delta_emu_forward(*dev(*x, first))
    near_long(o[:, :2500], want[:, :2500], 5000)
    near_long(o[:, 2500:], want[:, 2500:], 5000)
    near_long(state, last, 5000)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("t,hk,hv,ks,vs,decay", [
    (4500, 1, 1, 64, 64, 0.05), (4097, 1, 2, 128, 48, 0.2)])
def test_gradient_of_parts(dtype, t, hk, hv, ks, vs, decay):
    x = inputs(1, t, hk, hv, ks, vs, dtype, seed=t, decay=decay)
    do = torch.randn(1, t, hv, vs).to(dtype)
    for first, dfinal in ((None, None), (torch.randn(1, hv, ks, vs), torch.randn(1, hv, ks, vs))):
        want = delta_gradients(*x, do, first, dfinal)
        check(gradients(x, do, first, dfinal), want, x, do, 4 * t, dtype)


def test_gradient_of_packed_parts():
    bounds = [0, 4200, 4200, 8500]
    x = inputs(1, bounds[-1], 1, 1, 64, 32, torch.float32, seed=3, decay=0.05)
    do = torch.randn(1, bounds[-1], 1, 32)
    first, dfinal = torch.randn(3, 1, 64, 32), torch.randn(3, 1, 64, 32)
    cu = torch.tensor(bounds, dtype=torch.int32, device=DEV)
    want = delta_gradients(*x, do, first, dfinal, bounds=bounds)
    check(gradients(x, do, first, dfinal, cu_seqlens=cu), want, x, do, 4 * 4300, torch.float32)


@pytest.mark.parametrize("t", [15, 16, 17, 18])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_lengths_about_those_taken_token_by_token(t, dtype):
    x = inputs(3, t, 2, 4, 96, 36, dtype, seed=t, decay=0.2)
    first = torch.randn(3, 4, 96, 36)
    want, last = delta(*x, first)
    o, state = emu.delta_emu_forward(*dev(*x, first))
    near(o, want, t, dtype)
    near(state, last, t)
    # in place on the states
    y = dev(*x, first)
    o, state = emu.delta_emu_forward(*y, final_state=y[5])
    assert state is y[5]
    near(o, want, t, dtype)
    near(state, last, t)


@pytest.mark.parametrize("t", [3, 40])
def test_a_gate_that_is_not_a_number_is_seen(t):
    x = list(inputs(1, t, 1, 2, 32, 16, torch.float32))
    x[3][0, 1, 0] = torch.nan
    want, last = delta(*x, None)
    o, state = emu.delta_emu_forward(*dev(*x))
    assert o[0, 1:, 0].isnan().all() and state[0, 0].isnan().all()
    near(o[:, :, 1], want[:, :, 1], t)
    near(state[:, 1], last[:, 1], t)


def far(x, token):
    """x's values in a view whose tokens are `token` elements apart."""
    size = x.shape[2] * (x.shape[3] if x.dim() == 4 else 1)
    base = torch.empty((x.shape[1] - 1) * token + size, dtype=x.dtype, device=DEV)
    y = base.as_strided(x.shape, (x.shape[1] * token, token, *x.stride()[2:]))
    return y.copy_(x)


def test_offsets_of_more_than_32_bits():
    t, token = 600, 1 << 22  # 2.5e9 elements
    x = inputs(1, t, 1, 1, 64, 32, torch.bfloat16, decay=0.05)
    want, last = delta(*x, None)
    for i in range(5):
        y = dev(*x)
        y[i] = far(x[i], token)
        o, state = emu.delta_emu_forward(*y)
        near(o, want, t, torch.bfloat16)
        near(state, last, t)
        del y
    out = far(torch.zeros(1, t, 1, 32, dtype=torch.bfloat16), token)
    o, _ = emu.delta_emu_forward(*dev(*x), out=out)
    near(o, want, t, torch.bfloat16)


def test_gradient_offsets_of_more_than_32_bits():
    t, token = 600, 1 << 22
    x = inputs(1, t, 1, 1, 64, 32, torch.bfloat16, decay=0.05)
    do = torch.randn(1, t, 1, 32).bfloat16()
    want = delta_gradients(*x, do, None, None)
    for i in (1, 2, 3):
        y = dev(*x)
        y[i] = far(x[i], token)
        check(emu.delta_emu_backward(*y, do.to(DEV)), want, x, do, t, torch.bfloat16)
        del y
    check(emu.delta_emu_backward(*dev(*x), far(do, token)), want, x, do, t, torch.bfloat16)


def test_a_pool_of_more_than_32_bits():
    n, hv, ks, vs = 34000, 1, 64, 1024  # 2.2e9 elements, 8.9 GB
    pool = torch.empty(n, hv, ks, vs, device=DEV)
    slots = torch.tensor([n - 1, 0, 33000], dtype=torch.int32)
    x = inputs(3, 1, 1, hv, ks, vs, torch.float32)
    first = torch.randn(3, hv, ks, vs)
    for b, s in enumerate(slots.tolist()):
        pool[s] = first[b].to(DEV)
    want, last = delta(*x, first)
    o = emu.delta_emu_step(*dev(*x), pool, slots=slots.to(DEV))
    near(o, want, 1)
    near(pool[slots.to(DEV).long()], last, 1)


def test_rotary_offsets_of_more_than_32_bits():
    t, token = 300, 1 << 23
    x = torch.randn(1, t, 2, 64).bfloat16()
    cos, sin = emu.rotary_emu_table(t, 64, device=DEV)
    want, _ = emu.rotary_emu(x.to(DEV), None, cos, sin)
    y = far(x, token)
    got, _ = emu.rotary_emu(y, None, cos, sin)
    assert torch.equal(got, want)
    emu.rotary_emu(y, None, cos, sin, out=(y, None))  # in place
    assert torch.equal(y, want)
