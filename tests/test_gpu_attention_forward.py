"""Attention over whole sequences against the formulas in 64 bits (tolerances:
attention_plain.py)."""
import math

import pytest
import torch

import paper_2308_15152_amd as emu
from attention_plain import attention, near

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def inputs(b, t, n, hq, hk, size, dtype, seed=0, spread=1.5):
    g = torch.Generator().manual_seed(seed)

    def r(*shape):
        return torch.randn(shape, generator=g)

    return ((spread * r(b, t, hq, size)).to(dtype), r(b, n, hk, size).to(dtype),
            r(b, n, hk, size).to(dtype))


def check(x, got, causal=True, scale=None, bounds=None, key_bounds=None):
    """Every sequence's results; bounds: of packed ones."""
    q, k, v = x
    o, lse = got
    key_bounds = bounds if key_bounds is None else key_bounds
    for n in range(q.shape[0] if bounds is None else len(bounds) - 1):
        if bounds is None:
            part = q[n], k[n], v[n], o[n], lse[n]
        else:
            a, b, c, d = bounds[n], bounds[n + 1], key_bounds[n], key_bounds[n + 1]
            part = q[0, a:b], k[0, c:d], v[0, c:d], o[0, a:b], lse[0, a:b]
        want = attention(*part[:3], causal, scale)
        near(part[3], want["o"], ("o", n))
        near(part[4], want["lse"], ("lse", n))


def dev(*ts):
    return [t.to(DEV) for t in ts]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("b,t,n,hq,hk,size", [
    (1, 1, 1, 1, 1, 1), (2, 1, 1, 4, 2, 64), (1, 2, 2, 2, 2, 128), (3, 5, 5, 3, 1, 17),
    (1, 31, 31, 2, 2, 80), (2, 64, 64, 2, 1, 64), (1, 65, 65, 4, 4, 128), (1, 77, 77, 4, 2, 33),
    (2, 129, 129, 6, 2, 96), (1, 257, 257, 2, 1, 72), (1, 300, 300, 5, 5, 64),
    # other keys than tokens: a later part of a prompt, and tokens that see nothing
    (1, 1, 200, 8, 1, 128), (2, 3, 65, 4, 2, 40), (1, 100, 333, 2, 2, 64), (1, 40, 1000, 3, 1, 128),
    (2, 70, 5, 2, 1, 64), (1, 200, 64, 4, 2, 128), (1, 3, 0, 2, 1, 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_sizes(dtype, b, t, n, hq, hk, size, causal):
    x = inputs(b, t, n, hq, hk, size, dtype, seed=t + n)
    got = emu.attention_emu_forward(*dev(*x), causal=causal)
    check(x, got, causal)


@pytest.mark.parametrize("dtype", TYPES)
def test_many_tiles(dtype):
    x = inputs(1, 700, 1500, 4, 2, 128, dtype, seed=2)
    check(x, emu.attention_emu_forward(*dev(*x)))
    check(x, emu.attention_emu_forward(*dev(*x), causal=False), False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [1.0, 0.01, -0.3])
def test_scales_and_large_scores(dtype, scale):
    x = inputs(1, 90, 150, 2, 1, 64, dtype, spread=4.0)
    check(x, emu.attention_emu_forward(*dev(*x), scale=scale), scale=scale)


@pytest.mark.parametrize("dtype", TYPES)
def test_rising_scores(dtype):
    """Every tile's scores above those of the one before, and then below."""
    t = 320
    q = torch.ones(1, 4, 1, 16, dtype=dtype)
    ramp = torch.arange(t, dtype=torch.float32)
    for s in (ramp, -ramp):
        k = (0.25 * s)[None, :, None, None].expand(1, t, 1, 16).to(dtype).contiguous()
        v = torch.randn(1, t, 1, 16, generator=torch.Generator().manual_seed(3)).to(dtype)
        x = (q, k, v)
        check(x, emu.attention_emu_forward(*dev(*x)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [64, 80, 5])
@pytest.mark.parametrize("causal", [True, False])
def test_packed(dtype, size, causal):
    lengths = [1, 0, 130, 7, 64, 0, 33, 200, 1]
    bounds = [0]
    for n in lengths:
        bounds.append(bounds[-1] + n)
    x = inputs(1, bounds[-1], bounds[-1], 4, 2, size, dtype, seed=1)
    cu = torch.tensor(bounds, dtype=torch.int32, device=DEV)
    check(x, emu.attention_emu_forward(*dev(*x), cu_seqlens=cu, causal=causal), causal, None, bounds)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_many_packed_sequences(dtype):
    """More than the 64 that a wave looks over at a time, rows of no sequence at both ends."""
    g = torch.Generator().manual_seed(4)
    lengths = torch.randint(0, 9, (150,), generator=g).tolist()
    lengths[70] = 170
    bounds = [3]
    for n in lengths:
        bounds.append(bounds[-1] + n)
    total = bounds[-1] + 5
    x = inputs(1, total, total, 2, 1, 32, dtype, seed=1)
    cu = torch.tensor(bounds, dtype=torch.int32, device=DEV)
    o = torch.full((1, total, 2, 32), 7.0, dtype=dtype, device=DEV)
    lse = torch.full((1, total, 2), 7.0, device=DEV)
    got = emu.attention_emu_forward(*dev(*x), cu_seqlens=cu, out=o, lse=lse)
    assert got[0] is o and got[1] is lse
    check(x, got, True, None, bounds)
    for y in (o, lse):
        assert (y[:, :3] == 7).all() and (y[:, bounds[-1]:] == 7).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("causal", [True, False])
def test_packed_with_other_keys(dtype, causal):
    bounds, key_bounds = [0, 5, 5, 40, 41, 90], [0, 70, 80, 115, 115, 150]
    x = inputs(1, 90, 150, 4, 2, 64, dtype, seed=5)
    cu, cu_k = (torch.tensor(y, dtype=torch.int32, device=DEV) for y in (bounds, key_bounds))
    got = emu.attention_emu_forward(*dev(*x), cu_seqlens=cu, cu_seqlens_k=cu_k, causal=causal)
    check(x, got, causal, None, bounds, key_bounds)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [64, 24])
def test_strides(dtype, size):
    """Slices of one projection, broadcast keys, heads first, rows at odd addresses, outputs in
    a wider buffer."""
    b, t, hq, hk = 2, 100, 4, 2
    x = inputs(b, t, t, hq, hk, size, dtype, seed=6)
    rows = torch.cat([y.flatten(2) for y in x], 2).to(DEV)
    q, k, v = (y.unflatten(2, (-1, size)) for y in rows.split([hq * size, hk * size, hk * size], 2))
    wide = torch.full((b, t, hq + 1, size + 8), 3.0, dtype=dtype, device=DEV)
    lse = torch.zeros(b, hq, t, device=DEV).transpose(1, 2)
    check(x, emu.attention_emu_forward(q, k, v, out=wide[:, :, :hq, :size], lse=lse))
    assert (wide[:, :, hq] == 3).all() and (wide[..., size:] == 3).all()
    first = [y.transpose(1, 2).contiguous().transpose(1, 2) for y in dev(*x)]
    check(x, emu.attention_emu_forward(*first))
    odd = []
    for y in dev(*x):
        flat = torch.empty(y.numel() + 1, dtype=dtype, device=DEV)
        flat[1:] = y.flatten()
        odd.append(flat[1:].view(y.shape))
    check(x, emu.attention_emu_forward(*odd))
    same = (x[0], x[1][:1].expand(b, t, hk, size), x[2][:, :, :1].expand(b, t, hk, size))
    on = (dev(x[0])[0], dev(x[1][:1])[0].expand(b, t, hk, size),
          dev(x[2][:, :, :1])[0].expand(b, t, hk, size))
    check(same, emu.attention_emu_forward(*on))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("t,at", [(40, 0), (70, 69), (200, 50), (200, 130), (300, 299)])
def test_not_finite_reaches_those_that_see_it(dtype, value, t, at):
    x = inputs(2, t, t, 4, 2, 64, dtype, seed=7)
    want = emu.attention_emu_forward(*dev(*x))
    q, k, v = dev(*x)
    v[1, at, 1, 5] = value
    o, lse = emu.attention_emu_forward(q, k, v)
    assert torch.equal(lse, want[1])
    hit = torch.zeros_like(o, dtype=torch.bool)
    hit[1, at:, 2:, 5] = True
    assert torch.equal(o[~hit], want[0][~hit])
    if math.isnan(value):
        assert torch.isnan(o[hit]).all()
    else:
        assert (o[1, at, 2:, 5] == value).all()  # where it is the newest key
        assert not torch.isfinite(o[hit]).any()
    k[0, at, 0] = math.nan
    o, lse = emu.attention_emu_forward(q, k, v)
    assert torch.isnan(o[0, at:, :2]).all() and torch.isnan(lse[0, at:, :2]).all()
    assert torch.equal(o[0, :at], want[0][0, :at]) and torch.equal(o[0, :, 2:], want[0][0, :, 2:])


@pytest.mark.parametrize("dtype", TYPES)
def test_neighbours_are_not_read(dtype):
    """What lies behind a sequence's rows, NaN here, does not matter, packed or not."""
    x = inputs(1, 100, 100, 2, 1, 40, dtype, seed=8)
    wide = [torch.full((1, 140, y.shape[2], 48), math.nan, dtype=dtype, device=DEV) for y in x]
    for y, z in zip(x, wide):
        z[:, 20:120, :, :40] = y.to(DEV)
    views = [z[:, 20:120, :, :40] for z in wide]
    check(x, emu.attention_emu_forward(*views))
    check(x, emu.attention_emu_forward(*views, causal=False), False)
    cu = torch.tensor([20, 120], dtype=torch.int32, device=DEV)
    whole = [z[..., :40] for z in wide]
    o, lse = emu.attention_emu_forward(*whole, cu_seqlens=cu)
    check(x, (o[:, 20:120], lse[:, 20:120]))


def test_offsets_past_32_bits():
    """Keys and values more than 2^32 bytes, and 2^31 elements, behind each other."""
    stride = 1 << 22
    k = torch.empty((600 * stride,), dtype=torch.bfloat16, device=DEV)
    x = inputs(1, 3, 600, 1, 1, 64, torch.bfloat16, seed=9)
    keys = k.as_strided((1, 600, 1, 64), (k.numel(), stride, 64, 1))
    values = k.as_strided((1, 600, 1, 64), (k.numel(), stride, 64, 1), 64)
    keys.copy_(x[1].to(DEV)), values.copy_(x[2].to(DEV))
    check(x, emu.attention_emu_forward(x[0].to(DEV), keys, values))


def test_the_same_call_gives_the_same_bits():
    x = dev(*inputs(2, 500, 500, 8, 2, 128, torch.bfloat16, seed=10))
    first = emu.attention_emu_forward(*x)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, emu.attention_emu_forward(*x)))


def test_many_sequences_and_heads():
    """More blocks than one launch of small grids: tokens of many sequences."""
    b, t, h = 3000, 3, 12
    x = inputs(4, t, t, h, h, 16, torch.float16, seed=11)
    which = torch.arange(b) % 4
    o, lse = emu.attention_emu_forward(*[y[which].to(DEV) for y in x])
    assert torch.equal(o, o[:4][which.to(DEV)]) and torch.equal(lse, lse[:4][which.to(DEV)])
    check(x, (o[:4], lse[:4]))
