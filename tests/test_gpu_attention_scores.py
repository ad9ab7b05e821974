"""Attention where scores are so large that their last bits are no longer small beside one: which
key has the largest may be a matter of rounding, but weights are weights."""
import math

import pytest
import torch

import paper_2308_15152_amd as emu
from attention_plain import attention, near
from test_gpu_attention_backward import gradient_of
from test_gpu_attention_forward import DEV, TYPES, dev, inputs

pytestmark = pytest.mark.gpu


def of_size(t, n, hq, hk, size, dtype, power, seed):
    """Random inputs and a scale, with a largest scaled score of about 2^power; q and k up to 2^13,
    which FP16 holds."""
    q, k, v = inputs(1, t, n, hq, hk, size, dtype, seed=seed, spread=1.0)
    by = 2.0 ** min(math.floor((power - 3) / 2), 10)
    scale = size ** -0.5 * 2.0 ** (power - 3) / by / by
    return (q * by, k * by, v), scale


def in_the_values_range(o, v, n, t, group, causal, dtype):
    """o is between the least and the largest value that its row sees (weights and results are
    rounded to the type, sums to n 2^-24), and not zero."""
    e = torch.finfo(dtype).eps + n * 2.0 ** -23
    v = v.cpu().double().repeat_interleave(group, 1)
    margin = e * v.abs().amax(0)
    if causal:
        last = (torch.arange(t) + n - t)
        low, high = (torch.cummin(v, 0)[0][last], torch.cummax(v, 0)[0][last])
    else:
        low, high = v.amin(0), v.amax(0)
    o = o.cpu().double()
    assert torch.isfinite(o).all()
    assert (o >= low - margin).all() and (o <= high + margin).all()
    assert (o.abs().amax(-1) > 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("power", [20, 23, 26, 28, 30, 34])
@pytest.mark.parametrize("t,n,hq,hk,size", [
    (90, 90, 4, 2, 64), (400, 400, 4, 2, 64), (300, 900, 2, 1, 128), (16, 5000, 2, 1, 96)])
@pytest.mark.parametrize("causal", [True, False])
def test_forward(dtype, power, t, n, hq, hk, size, causal):
    x, scale = of_size(t, n, hq, hk, size, dtype, power, seed=power)
    o, lse = emu.attention_emu_forward(*dev(*x), causal=causal, scale=scale)
    in_the_values_range(o[0], x[2][0], n, t, hq // hk, causal, dtype)
    near(lse[0], attention(*(y[0] for y in x), causal, scale)["lse"], "lse")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("power", [28, 34])
def test_packed_forward(dtype, power):
    bounds = [0, 300, 301, 420, 600]
    x, scale = of_size(600, 600, 4, 2, 64, dtype, power, seed=power)
    cu = torch.tensor(bounds, dtype=torch.int32, device=DEV)
    o, lse = emu.attention_emu_forward(*dev(*x), cu_seqlens=cu, scale=scale)
    for a, b in zip(bounds, bounds[1:]):
        in_the_values_range(o[0, a:b], x[2][0, a:b], b - a, b - a, 2, True, dtype)
        near(lse[0, a:b], attention(*(y[0, a:b] for y in x), True, scale)["lse"], "lse")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("power", [24, 28, 30, 34])
@pytest.mark.parametrize("prefix", [0, 700])
@pytest.mark.parametrize("t", [1, 5])
def test_step(dtype, power, prefix, t):
    b, n = 3, 300
    x = [of_size(t, prefix + n, 4, 2, 64, dtype, power, seed=power + i)[0] for i in range(b)]
    scale = of_size(t, n, 4, 2, 64, dtype, power, 0)[1]
    q = torch.cat([y[0] for y in x])
    k, v = (torch.cat([y[i][:, prefix:] for y in x]) for i in (1, 2))
    pk, pv = x[0][1][:, :prefix], x[0][2][:, :prefix]
    lengths = torch.tensor([300, 250, t], dtype=torch.int32)
    o = emu.attention_emu_step(*dev(q, k, v, lengths), *(dev(pk, pv) if prefix else ()),
                               scale=scale)
    for i, m in enumerate(lengths.tolist()):
        in_the_values_range(o[i], torch.cat([pv[0], v[i, :m]]), prefix + m, t, 2, True, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("power", [20, 24, 28, 30, 34])
@pytest.mark.parametrize("t,n,hq,hk,size", [
    (90, 90, 4, 2, 64), (400, 400, 4, 2, 64), (300, 900, 2, 1, 128)])
@pytest.mark.parametrize("causal", [True, False])
def test_gradient(dtype, power, t, n, hq, hk, size, causal):
    """Weights of at most one: |dv| <= sum |do|, |ds| <= |do| |v| + |do| |o|, all over what may
    see each other, and 1% for roundings."""
    (q, k, v), scale = of_size(t, n, hq, hk, size, dtype, power, seed=power)
    x = q, k, v * 2.0 ** -8
    do = gradient_of(x, size=2.0 ** -8)
    if dtype == torch.float16:  # (which has to hold the gradients, up to scale |do| |v| |k|)
        do = do * 2.0 ** -max(power - 22, 0)
    on = dev(*x)
    o, lse = emu.attention_emu_forward(*on, causal=causal, scale=scale)
    got = [y[0].cpu().double() for y in
           emu.attention_emu_backward(*on, o, lse, do.to(DEV), causal=causal, scale=scale)]
    q, k, v, o, do = (y[0].cpu().double().abs().movedim(1, 0) for y in (*x, o, do))
    kk, vv = k.repeat_interleave(hq // hk, 0), v.repeat_interleave(hq // hk, 0)
    seen = torch.ones(t, n, dtype=torch.float64)
    if causal:
        seen = seen.tril(n - t)
    ds = seen * (do @ vv.mT + (do * o).sum(-1, keepdim=True))

    def fold(y):
        return y.unflatten(0, (hk, -1)).sum(1)

    most = scale * ds @ kk, fold(scale * ds.mT @ q), fold(seen.mT @ do)
    for name, y, z in zip(("dq", "dk", "dv"), got, most):
        assert z.max() < torch.finfo(dtype).max, name
        assert torch.isfinite(y).all(), name
        assert (y.movedim(1, 0).abs() <= 1.01 * z + torch.finfo(dtype).tiny).all(), name
