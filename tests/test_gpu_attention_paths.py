"""Attention where the kernels take other ways than for small inputs: many blocks, few rows
behind many keys (which are cut into parts and joined), wide groups of query heads, operands far
apart, magnitudes far from one.  Against the formulas in 64 bits (attention_plain.py)."""
import math

import pytest
import torch

import paper_2308_15152_amd as emu
from attention_plain import attention, near, unit
from test_gpu_attention_backward import check as check_gradient
from test_gpu_attention_backward import gradient_of, gradients
from test_gpu_attention_forward import DEV, TYPES, check, dev, inputs

pytestmark = pytest.mark.gpu


def both(x, causal=True, scale=None, seed=1, **kw):
    do = gradient_of(x, seed)
    check(x, emu.attention_emu_forward(*dev(*x), causal=causal, scale=scale), causal, scale)
    check_gradient(x, do, gradients(x, do, causal, scale), causal, scale)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("b,t,n,hq,hk,size", [
    (40, 300, 300, 8, 4, 64), (24, 280, 280, 16, 2, 128), (6, 800, 800, 8, 8, 96),
    (70, 129, 129, 8, 8, 40)])
def test_many_blocks(dtype, b, t, n, hq, hk, size):
    """Some of the sequences are looked at."""
    x = inputs(b, t, n, hq, hk, size, dtype, seed=t)
    do = gradient_of(x)
    o, lse = emu.attention_emu_forward(*dev(*x))
    got = gradients(x, do)
    some = [0, b // 2, b - 1]
    few = [y[some] for y in x]
    check(few, (o[some], lse[some]))
    check_gradient(few, do[some], [y[some] for y in got])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("b,t,n,hq,hk,size,causal", [
    (1, 3, 5001, 8, 2, 128, True), (2, 40, 3001, 4, 2, 64, False), (1, 130, 4500, 2, 1, 80, True),
    (3, 1, 2500, 3, 3, 24, True), (1, 5000, 40, 2, 1, 64, False), (1, 3000, 3, 4, 1, 128, False)])
def test_few_rows_or_keys(dtype, b, t, n, hq, hk, size, causal):
    both(inputs(b, t, n, hq, hk, size, dtype, seed=n), causal)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,n,causal", [(3, 700, True), (2, 90, False), (40, 40, True), (1, 1, True)])
def test_wide_groups(dtype, t, n, causal):
    """More query heads for a key head than a tile has rows."""
    both(inputs(1, t, n, 300, 1, 64, dtype, seed=t), causal)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths", [[1] * 40 + [2000], [700] * 9 + [0, 3], [300] * 30])
def test_packed(dtype, lengths):
    bounds = [0]
    for m in lengths:
        bounds.append(bounds[-1] + m)
    x = inputs(1, bounds[-1], bounds[-1], 4, 2, 64, dtype, seed=len(lengths))
    do = gradient_of(x)
    cu = torch.tensor(bounds, dtype=torch.int32, device=DEV)
    check(x, emu.attention_emu_forward(*dev(*x), cu_seqlens=cu), True, None, bounds)
    check_gradient(x, do, gradients(x, do, cu_seqlens=cu), True, None, bounds)


@pytest.mark.parametrize("size", [128, 64, 96])
@pytest.mark.parametrize("dtype", TYPES)
def test_strides_that_are_not_whole_chunks(dtype, size):
    """Rows that start at any element."""
    x = inputs(2, 400, 400, 4, 2, size, dtype, seed=size)
    do = gradient_of(x)
    on = []
    for y in (*x, do):
        wide = torch.full((2, 400, y.shape[2], size + 3), math.nan, dtype=dtype, device=DEV)
        wide[..., 1:1 + size] = y.to(DEV)
        on.append(wide[..., 1:1 + size])
    o, lse = emu.attention_emu_forward(*on[:3])
    check(x, (o, lse))
    out = [torch.full((2, 400, y.shape[2], size + 3), 7.0, dtype=dtype, device=DEV) for y in x]
    got = emu.attention_emu_backward(*on[:3], o, lse, on[3],
                                     out=[y[..., 2:2 + size] for y in out])
    check_gradient(x, do, got)
    for y in out:
        assert (y[..., :2] == 7).all() and (y[..., 2 + size:] == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,n,h", [(600, 600, 2), (300, 300, 40), (3, 4000, 2)])
def test_neighbours_are_not_read(dtype, t, n, h):
    x = inputs(1, t, n, h, 1, 64, dtype, seed=8)
    do = gradient_of(x)
    on = []
    for y in (*x, do):
        wide = torch.full((1, y.shape[1] + 40, y.shape[2], 64), math.nan, dtype=dtype, device=DEV)
        wide[:, 20:-20] = y.to(DEV)
        on.append(wide[:, 20:-20])
    o, lse = emu.attention_emu_forward(*on[:3])
    check(x, (o, lse))
    check_gradient(x, do, emu.attention_emu_backward(*on[:3], o, lse, on[3]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("b,t,h,at", [(1, 600, 4, 70), (1, 600, 4, 599), (40, 300, 8, 100),
                                      (40, 300, 8, 299)])
def test_values_that_are_not_finite(dtype, b, t, h, at):
    q, k, v = dev(*inputs(b, t, t, h, h // 2, 64, dtype, seed=7))
    want, lses = emu.attention_emu_forward(q, k, v)
    for value in (math.inf, math.nan):
        v[0, at, 1, 5] = value
        o, lse = emu.attention_emu_forward(q, k, v)
        hit = torch.zeros_like(o, dtype=torch.bool)
        hit[0, at:, 2:4, 5] = True
        assert torch.equal(lse, lses) and torch.equal(o[~hit], want[~hit])
        assert not torch.isfinite(o[hit]).any()


@pytest.mark.parametrize("dtype", TYPES)
def test_values_that_are_not_finite_behind_many_keys(dtype):
    q, k, v = dev(*inputs(1, 40, 4000, 4, 2, 64, dtype, seed=7))
    want, lses = emu.attention_emu_forward(q, k, v)
    for at in (3999, 3970, 100):
        v2 = v.clone()
        v2[0, at, 1, 5] = math.nan
        o, lse = emu.attention_emu_forward(q, k, v2)
        hit = torch.zeros_like(o, dtype=torch.bool)
        hit[0, max(at - 3960, 0):, 2:, 5] = True
        assert torch.equal(lse, lses) and torch.equal(o[~hit], want[~hit])
        assert torch.isnan(o[hit]).all()


@pytest.mark.parametrize("t", [200, 500])
@pytest.mark.parametrize("q_by,k_by,v_by,do_by", [
    (2.0 ** 50, 2.0 ** -50, 2.0 ** 20, 2.0 ** 30), (2.0 ** -40, 2.0 ** 40, 2.0 ** -20, 2.0 ** -20),
    (1.0, 1.0, 2.0 ** -20, 2.0 ** 40)])
def test_magnitudes_in_fp32(t, q_by, k_by, v_by, do_by):
    q, k, v = inputs(1, t, t, 4, 2, 64, torch.float32, seed=t)
    x = q * q_by, k * k_by, v * v_by
    do = gradient_of(x) * do_by
    o, lse = emu.attention_emu_forward(*dev(*x))
    check(x, (o, lse))
    check_gradient(x, do, gradients(x, do))


@pytest.mark.parametrize("t", [200, 500])
def test_rows_of_other_magnitudes_in_fp32(t):
    """Every row of v and do, and of q against a common k, has a magnitude of its own, and some
    are zero."""
    q, k, v = inputs(1, t, t, 4, 2, 64, torch.float32, seed=t)
    g = torch.Generator().manual_seed(t)

    def by(low, high):
        return 2.0 ** torch.randint(low, high, (1, t, 1, 1), generator=g)

    x = q * by(-20, 1), k, v * by(-20, 20)
    do = gradient_of(x) * by(-20, 20)
    for y in (*x, do):
        y[:, 17::50] = 0.0
    check(x, emu.attention_emu_forward(*dev(*x)))
    check_gradient(x, do, gradients(x, do))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_offsets_past_32_bits(dtype):
    """Rows and heads of every operand, and of every gradient, more than 2^32 bytes behind
    each other."""
    t, stride, head = 600, 1 << 22, 1 << 32
    ins, outs = (torch.empty(3 * head, dtype=dtype, device=DEV) for _ in range(2))
    x = inputs(1, t, t, 3, 1, 64, dtype, seed=9)
    do = gradient_of(x)

    def spread(buffer, shape, at):
        return buffer.as_strided(shape, (0, stride, head, 1), 64 * at)

    on = [spread(ins, y.shape, i).copy_(y.to(DEV)) for i, y in enumerate((*x, do))]
    o, lse = emu.attention_emu_forward(*on[:3], out=spread(outs, x[0].shape, 0))
    check(x, (o, lse))
    check_gradient(x, do, emu.attention_emu_backward(*on[:3], o, lse, on[3]))
    apart = o.contiguous()
    got = emu.attention_emu_backward(*on[:3], apart, lse, on[3], out=[
        spread(outs, y.shape, i) for i, y in enumerate(x)])
    check_gradient(x, do, got)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("t,n,joined", [(40, 40, False), (400, 400, False), (16, 5000, True)])
def test_scores_of_any_magnitude(dtype, sign, t, n, joined):
    """All scores of a row are the same, of magnitude 2^107, so that its weights are equal: o is
    the mean of what it sees (weights and o are rounded to the type, sums of n terms to n 2^-24).
    Where parts of the keys are joined by their log-sums, those hold 24 bits, 2^83 and up, and
    the number of a part's keys is not in them: o is some mean of the values then."""
    q, k, v = inputs(1, t, n, 2, 1, 64, dtype, seed=n)
    q[:], k[:] = 0.0, 0.0
    q[..., 3], k[..., 3] = 2.0 ** 55, sign * 2.0 ** 55
    o, lse = emu.attention_emu_forward(*dev(q, k, v))
    assert (lse == sign * 2.0 ** 107).all()  # log n is far below its last bit
    e = unit(dtype) + n * 2.0 ** -24
    values = v[0, :, 0].double()
    if not joined:
        seen = (torch.arange(n) <= torch.arange(t)[:, None] + n - t).double()
        seen /= seen.sum(1, keepdim=True)
        want, size = seen @ values, seen @ values.abs()
        for h in range(2):
            assert ((o[0, :, h].double().cpu() - want).abs() <= e * size + e * want.abs()).all()
    step = emu.attention_emu_step(*dev(q[:, -1:], k, v, torch.tensor([n], dtype=torch.int32)),
                                  *dev(k, v))
    for y in (o[0, -1], step[0, 0]):
        y = y.double().cpu()
        margin = 2 * e * values.abs().amax(0)
        assert (y <= values.amax(0) + margin).all() and (y >= values.amin(0) - margin).all()
        assert (y != 0).any()


def test_a_row_of_much_larger_scores():
    """One query's scores are thousands, its neighbours' of order one."""
    x = inputs(1, 400, 400, 2, 1, 64, torch.bfloat16, seed=2)
    x[0][:, 123] *= 500
    x[1][:, 77] *= 20
    both(x)


@pytest.mark.parametrize("dtype", TYPES)
def test_parts_joined_by_their_lse(dtype):
    x = inputs(1, 100, 700, 4, 2, 64, dtype, seed=3)
    q, k, v = dev(*x)
    o, lse = emu.attention_emu_forward(q, k, v, causal=False)
    parts = [emu.attention_emu_forward(q, k[:, y], v[:, y], causal=False)
             for y in (slice(0, 300), slice(300, None))]
    both_ = torch.logsumexp(torch.stack([y[1].double() for y in parts]), 0)
    want = attention(x[0][0], x[1][0], x[2][0], False)
    near(both_[0], (want["lse"][0], 2 * want["lse"][1] + 2.0 ** -22), "lse")
    joined = sum((y[0].double() * (y[1].double() - both_).exp()[..., None]) for y in parts)
    near(joined[0], (want["o"][0], 2 * want["o"][1] + 2 * torch.finfo(dtype).eps * sum(
        y[0].double().cpu()[0].abs() for y in parts)), "o")
