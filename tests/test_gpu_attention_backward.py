"""The gradient of attention against the formulas in 64 bits (tolerances:
attention_plain.py) and against differences of the forward pass."""
import pytest
import torch

import paper_2308_15152_amd as emu
from attention_plain import attention, near, unit
from test_gpu_attention_forward import DEV, TYPES, dev, inputs

pytestmark = pytest.mark.gpu


def gradients(x, do, causal=True, scale=None, **kw):
    """dq, dk, dv, with o and lse of the forward pass."""
    on = dev(*x)
    o, lse = emu.attention_emu_forward(*on, causal=causal, scale=scale, **{
        m: kw[m] for m in ("cu_seqlens", "cu_seqlens_k") if m in kw})
    return emu.attention_emu_backward(*on, o, lse, do.to(DEV), causal=causal, scale=scale, **kw)


def gradient_of(x, seed=1, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return (size * torch.randn(x[0].shape, generator=g)).to(x[0].dtype)


def check(x, do, got, causal=True, scale=None, bounds=None, key_bounds=None):
    q, k, v = x
    key_bounds = bounds if key_bounds is None else key_bounds
    for n in range(q.shape[0] if bounds is None else len(bounds) - 1):
        if bounds is None:
            rows, keys = (n, slice(None)), (n, slice(None))
        else:
            rows = (0, slice(bounds[n], bounds[n + 1]))
            keys = (0, slice(key_bounds[n], key_bounds[n + 1]))
        want = attention(q[rows], k[keys], v[keys], causal, scale, do[rows])
        for name, y, at in (("dq", got[0], rows), ("dk", got[1], keys), ("dv", got[2], keys)):
            near(y[at], want[name], (name, n))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("b,t,n,hq,hk,size", [
    (1, 1, 1, 1, 1, 1), (2, 1, 1, 4, 2, 64), (1, 2, 2, 2, 2, 128), (3, 5, 5, 3, 1, 17),
    (1, 31, 31, 2, 2, 80), (2, 64, 64, 2, 1, 64), (1, 65, 65, 4, 4, 128), (1, 77, 77, 4, 2, 33),
    (2, 129, 129, 6, 2, 96), (1, 257, 257, 2, 1, 72), (1, 300, 300, 5, 5, 64),
    (1, 1, 200, 8, 1, 128), (2, 3, 65, 4, 2, 40), (1, 100, 333, 2, 2, 64),
    (2, 70, 5, 2, 1, 64), (1, 200, 64, 4, 2, 128), (1, 3, 0, 2, 1, 64), (1, 0, 70, 2, 1, 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_sizes(dtype, b, t, n, hq, hk, size, causal):
    x = inputs(b, t, n, hq, hk, size, dtype, seed=t + n)
    do = gradient_of(x)
    check(x, do, gradients(x, do, causal), causal)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [64, 128])
def test_many_tiles(dtype, size):
    x = inputs(1, 700, 900, 4, 2, size, dtype, seed=2)
    do = gradient_of(x)
    check(x, do, gradients(x, do))
    check(x, do, gradients(x, do, False), False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [1.0, 0.01, -0.3])
def test_scales(dtype, scale):
    x = inputs(1, 90, 150, 2, 1, 64, dtype)
    do = gradient_of(x)
    check(x, do, gradients(x, do, scale=scale), scale=scale)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [1e-3, 1e3])
def test_small_and_large_gradients(dtype, size):
    """Gradients of a mean over many tokens are small, and FP16's range does not hold
    what is between them."""
    x = inputs(1, 260, 260, 2, 1, 64, dtype, seed=3)
    do = gradient_of(x, size=size)
    do[:, ::7] *= 2.0 ** -6
    x[2][:, 100:] *= 4
    check(x, do, gradients(x, do))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [64, 80, 5])
@pytest.mark.parametrize("causal", [True, False])
def test_packed(dtype, size, causal):
    lengths = [1, 0, 130, 7, 64, 0, 33, 200, 1]
    bounds = [2]
    for n in lengths:
        bounds.append(bounds[-1] + n)
    total = bounds[-1] + 3
    x = inputs(1, total, total, 4, 2, size, dtype, seed=1)
    do = gradient_of(x)
    cu = torch.tensor(bounds, dtype=torch.int32, device=DEV)
    got = gradients(x, do, causal, cu_seqlens=cu)
    check(x, do, got, causal, None, bounds)
    for y in got:  # rows of no sequence
        assert (y[:, :2] == 0).all() and (y[:, bounds[-1]:] == 0).all()
    out = [torch.full_like(y, 7.0) for y in got]
    again = gradients(x, do, causal, cu_seqlens=cu, out=out)
    for y, z in zip(got, again):
        assert torch.equal(y[:, 2:bounds[-1]], z[:, 2:bounds[-1]])
        assert (z[:, :2] == 7).all() and (z[:, bounds[-1]:] == 7).all()


@pytest.mark.parametrize("causal", [True, False])
def test_packed_with_other_keys(causal):
    bounds, key_bounds = [0, 5, 5, 40, 41, 90], [0, 70, 80, 115, 115, 150]
    x = inputs(1, 90, 150, 4, 2, 64, torch.bfloat16, seed=5)
    do = gradient_of(x)
    cu, cu_k = (torch.tensor(y, dtype=torch.int32, device=DEV) for y in (bounds, key_bounds))
    got = gradients(x, do, causal, cu_seqlens=cu, cu_seqlens_k=cu_k)
    check(x, do, got, causal, None, bounds, key_bounds)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [64, 24])
def test_strides(dtype, size):
    """Slices of one projection, and their gradients as slices of one buffer; gradients of
    broadcast outputs."""
    b, t, hq, hk = 2, 100, 4, 2
    x = inputs(b, t, t, hq, hk, size, dtype, seed=6)
    do = gradient_of(x)
    parts = [hq * size, hk * size, hk * size]

    def split(rows):
        return [y.unflatten(2, (-1, size)) for y in rows.split(parts, 2)]

    q, k, v = split(torch.cat([y.flatten(2) for y in x], 2).to(DEV))
    o, lse = emu.attention_emu_forward(q, k, v, lse=torch.empty(b, hq, t, device=DEV).transpose(1, 2))
    out = split(torch.empty(b, t, sum(parts), dtype=dtype, device=DEV))
    got = emu.attention_emu_backward(q, k, v, o, lse, do.to(DEV), out=out)
    assert all(y is z for y, z in zip(got, out))
    check(x, do, got)
    one = do[:, :1, :1].expand(b, t, hq, size)
    check(x, one, emu.attention_emu_backward(q, k, v, o, lse, do[:, :1, :1].to(DEV).expand(
        b, t, hq, size)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cut", [30, 170, 250])
def test_parts_of_the_keys(dtype, cut):
    """o and lse of all keys, the gradient over some of them at a time: dq in two parts."""
    x = inputs(1, 100, 300, 4, 2, 64, dtype, seed=14)
    do = gradient_of(x)
    q, k, v = dev(*x)
    o, lse = emu.attention_emu_forward(q, k, v, causal=False)
    parts = [emu.attention_emu_backward(q, k[:, y], v[:, y], o, lse, do.to(DEV), causal=False)
             for y in (slice(0, cut), slice(cut, None))]
    want = attention(x[0][0], x[1][0], x[2][0], False, None, do[0])
    halves = [y[0].double().cpu() for y, _, _ in parts]
    value, bound = want["dq"]  # and each part is rounded
    near(sum(halves), (value, bound + unit(dtype) * sum(y.abs() for y in halves)), "dq")
    for i, name in ((1, "dk"), (2, "dv")):
        near(torch.cat([y[i][0] for y in parts]), want[name], name)


def test_against_differences():
    """FP32: (f(x + h y) - f(x - h y)) / 2h for f = sum(do o).  Third derivatives along
    directions of length one are of order one here, and f is formed in 64 bits from outputs with
    errors of 2^-24 |do| |o| sqrt(size): h^2 + 1e-5 / h covers both."""
    x = inputs(1, 50, 60, 2, 1, 32, torch.float32, seed=12, spread=1.0)
    do = gradient_of(x)
    got = gradients(x, do)
    h = 2.0 ** -6
    for i in range(3):
        y = torch.randn(x[i].shape, generator=torch.Generator().manual_seed(i))
        y /= torch.linalg.vector_norm(y)
        f = []
        for s in (h, -h):
            z = [a.clone() for a in x]
            z[i] += s * y
            o, _ = emu.attention_emu_forward(*dev(*z))
            f.append(float((o.cpu().double() * do.double()).sum()))
        slope = float((got[i].cpu().double() * y.double()).sum())
        assert abs((f[0] - f[1]) / (2 * h) - slope) < h * h + 1e-5 / h


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_not_finite_stays_in_its_head(dtype):
    x = inputs(2, 100, 100, 4, 2, 64, dtype, seed=7)
    do = gradient_of(x)
    want = gradients(x, do)
    do[1, 40, 3, 2] = float("nan")
    got = gradients(x, do)
    for y, z, heads in zip(got, want, (slice(2, 4), slice(1, 2), slice(1, 2))):
        assert not torch.isfinite(y[1, :, heads]).all()
        assert torch.equal(y[0], z[0])
        assert torch.equal(y[1, :, :heads.start], z[1, :, :heads.start])


def test_the_same_call_gives_the_same_bits():
    x = inputs(2, 500, 500, 8, 2, 128, torch.bfloat16, seed=10)
    do = gradient_of(x)
    first = gradients(x, do)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, gradients(x, do)))


@pytest.mark.parametrize("dtype", TYPES)
def test_broadcast_inputs(dtype):
    """Keys and values that all sequences, or all key heads, share: a gradient for each."""
    x = inputs(3, 90, 90, 4, 2, 64, dtype, seed=15)
    q, k, v = dev(*x)
    k, v = k[:1].expand(3, -1, -1, -1), v[:, :, :1].expand(-1, -1, 2, -1)
    do = gradient_of(x)
    o, lse = emu.attention_emu_forward(q, k, v)
    got = emu.attention_emu_backward(q, k, v, o, lse, do.to(DEV))
    check((x[0], x[1][:1].expand(3, -1, -1, -1), x[2][:, :, :1].expand(-1, -1, 2, -1)), do, got)


@pytest.mark.parametrize("dtype", TYPES)
def test_large_scores_keep_gradients_finite(dtype):
    """Scores of 2^30, whose last bits are whole numbers: weights are not exact, but dv, a
    sum of weights up to one times do, is finite and no larger than the sum of |do|."""
    x = inputs(1, 100, 100, 2, 1, 64, dtype, seed=16)
    x = x[0] * 2048, x[1] * 8192, x[2]
    do = gradient_of(x)
    got = gradients(x, do)
    assert all(torch.isfinite(y).all() for y in got)
    if dtype == torch.float16:
        most = do.double().abs().sum((1, 2))
        assert (got[2][0, :, 0].double().cpu().abs() <= 1.01 * most).all()
