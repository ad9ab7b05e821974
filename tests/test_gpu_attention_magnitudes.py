"""Attention on values of very different magnitudes, in FP32 but for the last tests, against the
formulas in 64 bits (attention_plain.py): what a row does not see, or weighs next to nothing, takes
no bits from what it does."""
import math

import pytest
import torch

import paper_2308_15152_amd as emu
from attention_plain import attention, least, near
from test_gpu_attention_backward import check as check_gradient
from test_gpu_attention_backward import gradient_of, gradients
from test_gpu_attention_forward import DEV, check, dev, inputs

pytestmark = pytest.mark.gpu
F32 = torch.float32


@pytest.mark.parametrize("size", [64, 128])
@pytest.mark.parametrize("by", [2.0 ** 20, 2.0 ** 40, 2.0 ** 100])
@pytest.mark.parametrize("b,t,n,h,at", [
    (1, 500, 500, 2, 40), (1, 500, 500, 2, 0), (1, 700, 700, 2, 333), (40, 300, 300, 8, 65),
    (1, 40, 4000, 2, 3990), (1, 200, 3000, 1, 2900)])
def test_a_large_value(b, t, n, h, at, by, size):
    """Rows before it give what they give without it, bit for bit."""
    x = inputs(b, t, n, h, h // 2 or 1, size, F32, seed=t)
    want, lses = emu.attention_emu_forward(*dev(*x))
    x[2][0, at] *= by
    o, lse = emu.attention_emu_forward(*dev(*x))
    seen = max(at - (n - t), 0)  # the first row that sees it
    assert torch.equal(o[0, :seen], want[0, :seen]) and torch.equal(o[1:], want[1:])
    assert torch.equal(lse, lses)
    check([y[:1] for y in x], (o[:1], lse[:1]))


def test_a_large_value_in_packed_sequences():
    bounds = [0, 300, 301, 420, 600]
    x = inputs(1, 600, 600, 4, 2, 64, F32, seed=1)
    for at in (100, 310, 599):
        x[2][0, at] *= 2.0 ** 30
    cu = torch.tensor(bounds, dtype=torch.int32, device=DEV)
    do = gradient_of(x)
    check(x, emu.attention_emu_forward(*dev(*x), cu_seqlens=cu), True, None, bounds)
    check_gradient(x, do, gradients(x, do, cu_seqlens=cu), True, None, bounds)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("score,by", [(-20.0, 2.0 ** 20), (-30.0, 2.0 ** 40), (-200.0, 2.0 ** 60)])
@pytest.mark.parametrize("at", [0, 70, 450])
def test_a_large_value_of_little_weight(at, score, by, causal):
    """All rows see it with a weight of about e^score: before the keys that count, among them
    and behind them."""
    t = 500
    x = inputs(1, t, t, 2, 1, 64, F32, seed=at)
    x[0][..., 0] = 8.0  # the scale is 1 / 8
    x[1][..., 0] = 0.0
    x[1][:, at, :, 1:] = 0.0
    x[1][:, at, :, 0] = score
    x[2][:, at] *= by
    do = gradient_of(x)
    check(x, emu.attention_emu_forward(*dev(*x), causal=causal), causal)
    check_gradient(x, do, gradients(x, do, causal), causal)


@pytest.mark.parametrize("causal", [True, False])
def test_large_values_before_rising_scores(causal):
    """Every tile's weights make those before it small, whose values are larger by as much or
    by less."""
    t = 600
    x = inputs(1, t, t, 2, 1, 64, F32, seed=2)
    ramp = torch.arange(t, dtype=F32) // 32
    x[0][..., 0] = 8.0
    for per_tile, fall in ((20.0, 20.0), (40.0, 3.0), (12.0, 24.0)):
        x[1][..., 0] = per_tile * 0.693147 * ramp[:, None]
        y = x[0], x[1], x[2] * (2.0 ** (100 - fall * ramp).clamp(min=-100))[:, None, None]
        check(y, emu.attention_emu_forward(*dev(*y), causal=causal), causal)


@pytest.mark.parametrize("first", [-20, 20])
@pytest.mark.parametrize("seed", range(4))
def test_rows_of_every_magnitude(first, seed):
    """Every row of v and do, and of q against a common k, has a magnitude of its own; the first
    16 of v are the smallest, or the largest."""
    t = 500
    q, k, v = inputs(1, t, t, 4, 2, 64, F32, seed=seed)
    g = torch.Generator().manual_seed(seed)

    def by(low, high):
        return 2.0 ** torch.randint(low, high, (1, t, 1, 1), generator=g)

    of_v = by(-20, 20)
    of_v[:, :16] = 2.0 ** first
    x = q * by(-20, 1), k, v * of_v
    do = gradient_of(x, seed) * by(-20, 20)
    check(x, emu.attention_emu_forward(*dev(*x)))
    check_gradient(x, do, gradients(x, do))


@pytest.mark.parametrize("size", [64, 128])
@pytest.mark.parametrize("t", [200, 500])
@pytest.mark.parametrize("q_by,k_by,v_by,do_by", [
    (2.0 ** -110, 2.0 ** 110, 1.0, 1.0), (2.0 ** 110, 2.0 ** -110, 1.0, 1.0),
    (1.0, 1.0, 2.0 ** 110, 2.0 ** -100), (1.0, 1.0, 2.0 ** -100, 2.0 ** 110),
    (1.0, 1.0, 2.0 ** -100, 2.0 ** -10), (1.0, 1.0, 2.0 ** -10, 2.0 ** -100)])
def test_magnitudes_near_the_ends(t, q_by, k_by, v_by, do_by, size):
    """No product on the way to a result that has a value in FP32 passes its range."""
    q, k, v = inputs(1, t, t, 4, 2, size, F32, seed=t)
    x = q * q_by, k * k_by, v * v_by
    do = gradient_of(x) * do_by
    for value, _ in attention(*(y[0] for y in x), do=do[0]).values():
        assert value.abs().max() < 2.0 ** 127
    check(x, emu.attention_emu_forward(*dev(*x)))
    check_gradient(x, do, gradients(x, do))


@pytest.mark.parametrize("t", [200, 500])
@pytest.mark.parametrize("by", [2.0 ** 30, 2.0 ** -30])
def test_scales_beside_magnitudes(t, by):
    """Small and large factors of the scores, with rows of zeros among those of q and k."""
    q, k, v = inputs(1, t, t, 4, 2, 64, F32, seed=t)
    x = q * by, k, v
    for y in x[:2]:
        y[:, 17::50] = 0.0
    do = gradient_of(x)
    scale = 0.125 / by
    check(x, emu.attention_emu_forward(*dev(*x), scale=scale), scale=scale)
    check_gradient(x, do, gradients(x, do, scale=scale), scale=scale)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, F32])
@pytest.mark.parametrize("n,cut", [(100, 80), (600, 500), (1500, 1400)])
@pytest.mark.parametrize("score,by", [(-6.5, 2.0 ** 8), (-9.0, 2.0 ** 12), (-9.5, 2.0 ** 6),
                                      (-9.5, 2.0 ** 13)])
def test_keys_elsewhere_that_matter_little_but_for_their_values(dtype, n, cut, score, by):
    """o and lse of all keys, the gradient over some: the others have a weight in all of about
    e^score, and values so large that delta is theirs as well.  delta is off by the rounding
    of o, half a step, and by what the kernel may take for that of o and of the weights that
    made it: a step of sum |do o| + sum |ds| + |delta|, over the keys that are given."""
    t, size = 150, 64
    q, k, v = inputs(1, t, n, 2, 1, size, F32, seed=n, spread=1.0)
    q[..., 0], k[..., 0] = 8.0, 0.0  # the scale is 1 / 8
    k[:, cut:, :, 1:] = 0.0
    k[:, cut:, :, 0] = score + math.log(cut / (n - cut))
    v[:, cut:] *= by
    q, k, v = (y.to(dtype) for y in (q, k, v))
    do = gradient_of((q, k, v)).to(dtype)
    scale = size ** -0.5
    Q, K, V, D = (y[0].double().movedim(1, 0) for y in (q, k, v, do))
    s = scale * Q @ K.mT
    lse = torch.logsumexp(s, -1)
    p = (s - lse[..., None]).exp()
    o = p @ V
    on = dev(q, k[:, :cut], v[:, :cut], o.movedim(0, 1)[None].to(dtype),
             lse.mT[None].float().contiguous(), do)
    got = emu.attention_emu_backward(*on, causal=False)
    g, mean = D @ V.mT, (D * o).sum(-1, keepdim=True)
    e, r = 2.0 ** -24, torch.finfo(dtype).eps / 2
    u = r if dtype != F32 else 0.0
    of_mean = (D * o).abs().sum(-1, keepdim=True)
    b = scale * Q.abs() @ K.abs().mT
    w = ((size + 8) * e * b.amax(-1) + (n + 64) * e + e * lse.abs())[..., None]
    ds = p * (g - mean)
    of_delta = (r + (size + 4) * e) * of_mean
    of_delta = of_delta + 2 * r * (of_mean + ds[..., :cut].abs().sum(-1, keepdim=True) + mean.abs())
    off = p * (2 * w * (D.abs() @ V.abs().mT + of_mean) + of_delta)
    off = off + u * ds.abs() + n * e * ds.abs() + e * ds.abs().amax(-1, keepdim=True)
    off_k = off + e * ds.abs().amax(-2, keepdim=True)
    ds, off, off_k, K = ds[..., :cut], off[..., :cut], off_k[..., :cut], K[:, :cut]
    near(got[0][0].movedim(1, 0), bounded(scale * ds @ K, scale * off @ K.abs(), dtype), "dq")
    near(got[1][0, :, 0], bounded((scale * ds.mT @ Q).sum(0), (scale * off_k.mT @ Q.abs()).sum(0),
                                  dtype), "dk")


def bounded(value, bound, dtype):
    """With the result's own rounding."""
    return value, bound + torch.finfo(dtype).eps / 2 * value.abs() + least(dtype)


@pytest.mark.parametrize("size", [1, 2, 3])
@pytest.mark.parametrize("seed", [26, 28, 43, 68])
def test_heads_of_few_elements(seed, size):
    """Where o is next to zero, delta's error is that of the weights that made it."""
    lengths = [300, 38, 290, 444, 1]
    bounds = [sum(lengths[:i]) for i in range(6)]
    x = inputs(1, bounds[-1], bounds[-1], 2, 2, size, torch.bfloat16, seed=seed)
    do = gradient_of(x, seed % 97)
    cu = torch.tensor(bounds, dtype=torch.int32, device=DEV)
    check_gradient(x, do, gradients(x, do, cu_seqlens=cu), True, None, bounds)
