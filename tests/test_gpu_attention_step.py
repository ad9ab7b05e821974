"""Single tokens behind a shared prefix and caches of their own against the formulas
in 64 bits (tolerances: attention_plain.py), and prompts followed by single tokens."""
import math

import pytest
import torch

import paper_2308_15152_amd as emu
from attention_plain import attention, near
from test_gpu_attention_forward import DEV, TYPES, dev

pytestmark = pytest.mark.gpu


def inputs(b, t, prefix, capacity, hq, hk, size, dtype, seed=0, pool=2):
    g = torch.Generator().manual_seed(seed)

    def r(*shape):
        return torch.randn(shape, generator=g).to(dtype)

    x = {"q": r(b, t, hq, size) * 1.5, "k": r(b + pool, capacity, hk, size),
         "v": r(b + pool, capacity, hk, size)}
    if prefix is not None:
        x["prefix_k"], x["prefix_v"] = r(1, prefix, hk, size), r(1, prefix, hk, size)
    lengths = torch.randint(0, capacity + 1, (b,), generator=g).int()
    lengths[0] = capacity
    slots = torch.randperm(b + pool, generator=g)[:b].int()
    return x, lengths, slots


def run(x, lengths, slots, **kw):
    y = {m: z.to(DEV) for m, z in x.items()}
    return emu.attention_emu_step(y["q"], y["k"], y["v"], lengths.to(DEV), y.get("prefix_k"),
                                  y.get("prefix_v"), slots=None if slots is None
                                  else slots.to(DEV), **kw)


def check(x, lengths, slots, o, scale=None):
    for n in range(x["q"].shape[0]):
        slot = n if slots is None else int(slots[n])
        if not 0 <= slot < x["k"].shape[0]:
            assert (o[n] == 0).all()
            continue
        m = min(max(int(lengths[n]), 0), x["k"].shape[1])
        k, v = x["k"][slot, :m], x["v"][slot, :m]
        t = x["q"].shape[1]
        # (a cache shorter than the new tokens: the first of them see the prefix only)
        seen = [max(m - t + 1 + i, 0) for i in range(t)]
        for i in range(t):
            keys, values = k[:seen[i]], v[:seen[i]]
            if "prefix_k" in x:
                keys = torch.cat([x["prefix_k"][0], keys])
                values = torch.cat([x["prefix_v"][0], values])
            want = attention(x["q"][n, i:i + 1], keys, values, False, scale)
            near(o[n, i:i + 1], joined(want["o"], x["q"].dtype, keys), (n, i))


def joined(want, dtype, keys):
    """Parts are normalized in FP32 and joined: a few roundings more."""
    return want[0], want[1] + 8 * 2.0 ** -24 * want[0].abs() + 2.0 ** -22


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("b,t,prefix,capacity,hq,hk,size", [
    (1, 1, 1, 1, 1, 1, 1), (2, 1, None, 64, 4, 2, 64), (3, 1, 70, 33, 8, 1, 128),
    (2, 5, 100, 40, 12, 4, 96), (5, 1, 600, 700, 6, 2, 80), (1, 3, 1000, 10, 2, 2, 17),
    (40, 1, 300, 65, 8, 2, 64), (2, 40, 90, 100, 2, 1, 64), (4, 2, None, 900, 4, 4, 33),
    (3, 1, 0, 50, 2, 1, 64), (2, 1, 50, 0, 2, 1, 64), (1, 1, 4000, 2000, 4, 1, 128)])
def test_sizes(dtype, b, t, prefix, capacity, hq, hk, size):
    x, lengths, slots = inputs(b, t, prefix, capacity, hq, hk, size, dtype, seed=b + capacity)
    check(x, lengths, slots, run(x, lengths, slots))
    check(x, lengths, None, run(x, lengths, None))


@pytest.mark.parametrize("dtype", TYPES)
def test_scales(dtype):
    x, lengths, slots = inputs(3, 2, 90, 100, 4, 2, 64, dtype)
    for scale in (0.5, -0.2):
        check(x, lengths, slots, run(x, lengths, slots, scale=scale), scale)


def test_slots_and_lengths_outside():
    x, lengths, slots = inputs(6, 2, 90, 100, 4, 2, 64, torch.bfloat16)
    lengths = torch.tensor([0, 1, -5, 101, 2 ** 31 - 1, 50], dtype=torch.int32)
    slots = torch.tensor([0, 1, 2, -1, 8, 3], dtype=torch.int32)
    check(x, lengths, slots, run(x, lengths, slots))
    x.pop("prefix_k"), x.pop("prefix_v")
    o = run(x, lengths, slots)
    check(x, lengths, slots, o)
    assert (o[0] == 0).all()  # nothing to see
    # two sequences may read one cache
    check(x, lengths, slots * 0, run(x, lengths, slots * 0))


@pytest.mark.parametrize("dtype", TYPES)
def test_what_lies_behind_is_not_used(dtype):
    x, lengths, slots = inputs(5, 3, 100, 300, 4, 2, 64, dtype, seed=3)
    want = run(x, lengths, slots)
    for n in range(5):
        for m in ("k", "v"):
            x[m][slots[n], lengths[n]:] = math.nan
    for slot in set(range(7)) - set(slots.tolist()):
        x["v"][slot] = math.inf
    assert torch.equal(run(x, lengths, slots), want)


@pytest.mark.parametrize("dtype", TYPES)
def test_not_finite_reaches_the_tokens_that_see_it(dtype):
    """Drafted tokens: the last one's value is not the first one's to see."""
    x, lengths, _ = inputs(2, 3, 40, 80, 4, 2, 64, dtype, seed=4)
    lengths[:] = torch.tensor([80, 45])
    want = run(x, lengths, None)
    x["v"][1, 44, 0, 7] = math.inf
    x["v"][0, 78, 1, 3] = math.nan
    o = run(x, lengths, None)
    hit = torch.zeros_like(o, dtype=torch.bool)
    hit[1, 2, :2, 7] = True
    hit[0, 1:, 2:, 3] = True
    assert torch.equal(o[~hit], want[~hit])
    assert (o[1, 2, :2, 7] == math.inf).all() and torch.isnan(o[0, 1:, 2:, 3]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_strides(dtype):
    """Caches with heads first, rows at odd addresses, outputs in a wider buffer."""
    x, lengths, slots = inputs(4, 1, 70, 90, 4, 2, 40, dtype, seed=5)
    y = dict(x)
    for m in ("k", "v", "prefix_k", "prefix_v"):
        y[m] = x[m].transpose(1, 2).contiguous().transpose(1, 2)
    y = {m: z.to(DEV) if m == "q" else z.transpose(1, 2).to(DEV).transpose(1, 2)
         for m, z in y.items()}
    wide = torch.full((4, 1, 5, 41), 3.0, dtype=dtype, device=DEV)
    o = emu.attention_emu_step(y["q"], y["k"], y["v"], lengths.to(DEV), y["prefix_k"],
                               y["prefix_v"], slots=slots.to(DEV), out=wide[:, :, :4, :40])
    check(x, lengths, slots, o)
    assert (wide[:, :, 4] == 3).all() and (wide[..., 40:] == 3).all()


def test_offsets_past_32_bits():
    """A pool of caches of more than 2^31 elements."""
    b, capacity, hk, size = 3, 4096, 8, 128
    pool = 2 ** 31 // (capacity * hk * size) + 5
    k = torch.empty(pool, capacity, hk, size, dtype=torch.bfloat16, device=DEV)
    v = torch.empty(pool, capacity, hk, size, dtype=torch.bfloat16, device=DEV)
    x, lengths, _ = inputs(b, 1, 20, capacity, hk, hk, size, torch.bfloat16, seed=6, pool=0)
    lengths = torch.tensor([4096, 70, 1000], dtype=torch.int32)
    slots = torch.tensor([pool - 1, 0, pool - 3], dtype=torch.int32, device=DEV)
    k[slots.long()], v[slots.long()] = x["k"].to(DEV), x["v"].to(DEV)
    o = emu.attention_emu_step(x["q"].to(DEV), k, v, lengths.to(DEV), x["prefix_k"].to(DEV),
                               x["prefix_v"].to(DEV), slots=slots)
    check(x, lengths, None, o)


@pytest.mark.parametrize("dtype", TYPES)
def test_a_prompt_and_single_tokens(dtype):
    """A prefix and prompts read at once, then token by token, with rotary positions: what
    whole sequences give.  Both sides are within attention_plain.py's bounds of the same
    values, so their difference is within their sum."""
    b, shared, prompt, more, hq, hk, size = 3, 70, 40, 5, 4, 2, 64
    g = torch.Generator().manual_seed(9)
    tokens = shared + prompt + more

    def sequences(h):
        x = torch.randn(b, tokens, h, size, generator=g).to(dtype)
        x[:, :shared] = x[:1, :shared]
        return x.to(DEV)

    cos, sin = emu.rotary_emu_table(256, size, device=DEV)
    q, k = emu.rotary_emu(sequences(hq), sequences(hk), cos, sin)
    v = sequences(hk)
    o, _ = emu.attention_emu_forward(q, k, v)
    prefix = [y[:1, :shared].contiguous() for y in (k, v)]
    caches = [torch.full((b, prompt + more, hk, size), math.nan, dtype=dtype, device=DEV)
              for _ in range(2)]
    for cache, y in zip(caches, (k, v)):
        cache[:, :prompt] = y[:, shared:shared + prompt]
    part, _ = emu.attention_emu_forward(q[:, shared:shared + prompt], k[:, :shared + prompt],
                                        v[:, :shared + prompt])
    got = [part]
    for t in range(more):
        at = shared + prompt + t
        for cache, y in zip(caches, (k, v)):
            cache[:, prompt + t] = y[:, at]
        lengths = torch.full((b,), prompt + t + 1, dtype=torch.int32, device=DEV)
        got.append(emu.attention_emu_step(q[:, at:at + 1], *caches, lengths, *prefix))
    got = torch.cat(got, 1)
    for n in range(b):
        want = attention(q[n], k[n], v[n])["o"]
        near(o[n], want)
        near(got[n], joined((want[0][shared:], want[1][shared:]), dtype, None))
    # several drafted tokens at once
    lengths = torch.full((b,), prompt + more, dtype=torch.int32, device=DEV)
    drafted = emu.attention_emu_step(q[:, -more:], *caches, lengths, *prefix)
    for n in range(b):
        want = attention(q[n], k[n], v[n])["o"]
        near(drafted[n], joined((want[0][-more:], want[1][-more:]), dtype, None))
