"""The softmax attention operators of a language model, as such a model calls
them: over whole prompts, their gradient, and single tokens of a batch of
sequences that share a prefix.

Shapes: q and o are (batch, tokens, query heads, size), k and v (batch, keys, key
heads, size); query head h reads key head h // (query heads / key heads).  Token
i of a sequence of t tokens and n keys sees, if causal, keys 0 to i + n - t:
    s_j = scale q k_j,  lse = log sum_j e^s_j,  o = sum_j e^(s_j - lse) v_j,
and zeros (lse = -infinity) where it sees none.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # a short prompt on small heads in FP32: bound by latency
        forward("prompt_short", 1, 77, 77, 4, 4, 64, "f32"),
        # a training batch, or prompts of one length
        forward("prompt_4096", 4, 4096, 4096, 32, 8, 128, "bf16"),
        # one very long prompt on few heads
        forward("prompt_long", 1, 32768, 32768, 8, 2, 128, "bf16"),
        # packed prompts of 1 to 2000 tokens
        forward("prompt_packed", 24, 2000, 2000, 16, 4, 128, "f16", packed=True),
        # the next part of a prompt, on what the cache holds of it
        forward("prompt_part", 1, 512, 8192, 16, 4, 128, "bf16"),
        # every token sees every key, odd sizes, slices of one projection
        forward("whole_odd", 3, 1001, 1001, 6, 2, 80, "bf16", causal=False, strided=True),
        # a training step's gradient, ordinary sizes
        backward("gradient_4096", 2, 4096, 4096, 16, 4, 128, "bf16"),
        # gradient over packed sequences of 1 to 2500 tokens, small heads
        backward("gradient_packed", 16, 2500, 2500, 8, 8, 64, "f16", packed=True),
        # gradient with other keys than tokens, odd lengths and sizes, in FP32
        backward("gradient_odd", 3, 1001, 1234, 6, 2, 80, "f32", causal=False),
        # the next token of one sequence behind a short prefix: bound by latency
        step("step_one", 1, 1, 512, 64, 16, 4, 128, "bf16"),
        # the next token of many sequences behind a long instruction
        step("step_128", 128, 1, 16384, 1024, 32, 8, 128, "bf16"),
        # a few drafted tokens per sequence, odd sizes
        step("step_draft", 33, 5, 1000, 300, 12, 4, 96, "f16"),
    ]


def whole(kind, name, batch, tokens, keys, q_heads, k_heads, size, dtype, causal=True,
          strided=False, packed=False):
    c = {"kind": kind, "batch": batch, "tokens": tokens, "keys": keys, "q_heads": q_heads,
         "k_heads": k_heads, "size": size, "dtype": dtype, "causal": causal, "strided": strided,
         "packed": packed}
    return dict(c, name=name) if name else c


def forward(*args, **more):
    return whole("forward", *args, **more)


def backward(*args, **more):
    return whole("backward", *args, **more)


def step(name, batch, tokens, prefix, capacity, q_heads, k_heads, size, dtype):
    c = {"kind": "step", "batch": batch, "tokens": tokens, "prefix": prefix,
         "capacity": capacity, "q_heads": q_heads, "k_heads": k_heads, "size": size,
         "dtype": dtype}
    return dict(c, name=name) if name else c


# Most of a drawn case: tokens x keys x query heads, as in the largest listed
# cases of the kind (FP32 takes an eighth of that), and the values of a step's caches.
MOST = {"forward": 2 ** 32, "backward": 2 ** 28, "step": 2 ** 27}
VALUES = 2 ** 28


def log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["forward", "forward", "backward", "backward", "step"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    k_heads = log_int(rng, 1, 16)
    q_heads = k_heads * rng.choice([1, 2, 3, 4, 8])
    size = rng.choice([64, 64, 80, 96, 128, 128, 128, log_int(rng, 16, 128)])
    most = MOST[kind] / (8 if dtype == "f32" else 1)
    if kind == "step":
        tokens = rng.choice([1, 1, 1, 2, 5])
        prefix = log_int(rng, 1, 32768)
        capacity = log_int(rng, max(tokens, 16), 4096)
        batch = log_int(rng, 1, max(1.0, min(256.0, VALUES / (2 * capacity * k_heads * size),
                                             most / (tokens * q_heads * (prefix + capacity)))))
        return step(None, batch, tokens, prefix, capacity, q_heads, k_heads, size, dtype)
    # (behind one key alone a gradient is zero, but for dv)
    least = 2 if kind == "backward" else 1
    tokens = log_int(rng, least, min(16384.0, math.sqrt(most / q_heads)))
    packed = rng.random() < 0.3
    keys = tokens
    if not packed and rng.random() < 0.3:
        keys = log_int(rng, tokens, max(tokens, min(32768.0, most / (q_heads * tokens))))
    batch = log_int(rng, 1, max(1.0, min(64.0, most / (q_heads * tokens * keys))))
    return whole(kind, None, batch, tokens, keys, q_heads, k_heads, size, dtype,
                 causal=rng.random() < 0.8, strided=keys == tokens and rng.random() < 0.3,
                 packed=packed and batch > 1)


# --------------------------------------------------------------------------
# Inputs


def normal(g, *shape):
    return torch.randn(shape, generator=g, dtype=torch.float32, device=DEVICE)


def lengths(case):
    """Tokens of each packed sequence: 1 to the most, which the first has, even over the
    logarithm; of each cache: the new tokens to its capacity, even.  Every seed has the
    same ones, so that outputs have one shape and passes the same work."""
    n, most = case["batch"], case.get("capacity", case["tokens"])
    g = torch.Generator().manual_seed(n * 65536 + most)
    r = torch.rand(n, generator=g, dtype=torch.float64)
    r[0] = 1.0
    if case["kind"] == "step":
        return (case["tokens"] + r * (most + 1 - case["tokens"])).long().clamp(max=most)
    return torch.exp(r * math.log(most)).round().long().clamp(1, most)


def inputs(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    b, t, hq, hk, size = (case[n] for n in ("batch", "tokens", "q_heads", "k_heads", "size"))
    if case["kind"] == "step":  # (behind a sequence's keys a cache holds what others left)
        pool, prefix, n = b + 3, case["prefix"], case["capacity"]
        return {"q": (1.5 * normal(g, b, t, hq, size)).to(dtype),
                "prefix_k": normal(g, 1, prefix, hk, size).to(dtype),
                "prefix_v": normal(g, 1, prefix, hk, size).to(dtype),
                "k": normal(g, pool, n, hk, size).to(dtype),
                "v": normal(g, pool, n, hk, size).to(dtype),
                "lengths": lengths(case).int().to(DEVICE),
                "slots": torch.randperm(pool, generator=g, device=DEVICE)[:b].int()}
    n, x = case["keys"], {}
    if case["packed"]:
        ends = torch.cat([torch.zeros(1, dtype=torch.long), lengths(case).cumsum(0)])
        x["cu_seqlens"] = ends.int().to(DEVICE)
        x["ends"] = ends.tolist()
        b, t, n = 1, x["ends"][-1], x["ends"][-1]
    # scores with a spread of a few units, as trained layers have
    q = (1.5 * normal(g, b, t, hq, size)).to(dtype)
    k = normal(g, b, n, hk, size).to(dtype)
    v = normal(g, b, n, hk, size).to(dtype)
    if case["strided"]:
        rows = torch.cat([q.flatten(2), k.flatten(2), v.flatten(2)], dim=2)
        q, k, v = rows.split([hq * size, hk * size, hk * size], dim=2)
        q, k, v = q.unflatten(2, (hq, size)), k.unflatten(2, (hk, size)), v.unflatten(2, (hk, size))
    x.update(q=q, k=k, v=v)
    if case["kind"] == "backward":
        # gradients of a mean over many tokens are small
        x["do"] = (1e-3 * normal(g, b, t, hq, size)).to(dtype)
    return x


def prepare(case, seed):
    s = dict(inputs(case, seed), case=case)
    if case["kind"] == "backward":  # what a training step keeps of its forward pass
        s["o"], s["lse"] = plain_forward(s)
    return s


# --------------------------------------------------------------------------
# One pass


def run(state):
    kind = state["case"]["kind"]
    return {"forward": run_forward, "backward": run_backward, "step": run_step}[kind](state)


def run_forward(s):
    if own:
        import paper_2308_15152_amd as emu

        o, lse = emu.attention_emu_forward(s["q"], s["k"], s["v"], causal=s["case"]["causal"],
                                           cu_seqlens=s.get("cu_seqlens"))
    else:
        o, lse = plain_forward(s)
    return {"o": o, "lse": lse}


def run_backward(s):
    if own:
        import paper_2308_15152_amd as emu

        dq, dk, dv = emu.attention_emu_backward(s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"],
                                                causal=s["case"]["causal"],
                                                cu_seqlens=s.get("cu_seqlens"))
    else:
        dq, dk, dv = plain_backward(s)
    return {"dq": dq, "dk": dk, "dv": dv}


def run_step(s):
    if own:
        import paper_2308_15152_amd as emu

        o = emu.attention_emu_step(s["q"], s["k"], s["v"], s["lengths"], s["prefix_k"],
                                   s["prefix_v"], slots=s["slots"])
    else:
        o = plain_step(s)
    return {"o": o}


def padded(x, s):
    """(sequences, heads, tokens, size) in FP32; packed sequences as rows of a batch."""
    if "ends" in s:
        at, inside = places(s)
        x = torch.where(inside[:, :, None, None], x[0][at], 0)
    return x.transpose(1, 2).float()


def unpadded(y, s):
    y = y.transpose(1, 2)
    return y[places(s)[1]][None] if "ends" in s else y.contiguous()


def places(s):
    cu = s["cu_seqlens"].long()
    n = cu[1:] - cu[:-1]
    j = torch.arange(s["case"]["tokens"], device=DEVICE)
    inside = j[None] < n[:, None]
    return torch.where(inside, cu[:-1, None] + j, 0), inside


def grouped(x, hk):
    """(sequences, key heads, query heads of each x tokens, size)."""
    return x.unflatten(1, (hk, -1)).flatten(2, 3)


def apart(x, group):
    """The inverse: (sequences, query heads, tokens, size)."""
    return x.unflatten(2, (group, -1)).flatten(1, 2)


def scores(q, k, first, s):
    """Scores of a block of tokens, from number `first` on: -infinity where a key is not
    seen."""
    case = s["case"]
    group, n = q.shape[1] // k.shape[1], k.shape[2]
    y = grouped(q, k.shape[1]) @ k.mT.contiguous() / math.sqrt(case["size"])
    j = torch.arange(n, device=DEVICE)
    seen = torch.ones(1, 1, 1, n, dtype=torch.bool, device=DEVICE)
    if "ends" in s:
        cu = s["cu_seqlens"].long()
        seen = (j < (cu[1:] - cu[:-1])[:, None])[:, None, None]
    if case["causal"]:
        i = first + torch.arange(q.shape[2], device=DEVICE)
        seen = seen & (j <= (i + n - case["tokens"])[:, None]).repeat(group, 1)
    return torch.where(seen, y, -torch.inf)


def weights(y):
    """(e^(y - lse), lse) along the last dimension; zeros where nothing is seen."""
    top = y.amax(-1, keepdim=True)
    p = (y - torch.where(top == -torch.inf, 0.0, top)).exp()
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total == 0, 1.0, total), (top + total.log())


def blocks(q, k):
    """Tokens of a block: at most 2^29 scores at a time."""
    return max(1, 2 ** 29 // (q.shape[0] * q.shape[1] * k.shape[2]))


def plain_forward(s):
    q, k, v = (padded(s[n], s) for n in "qkv")
    group, rows = q.shape[1] // k.shape[1], blocks(q, k)
    o, lse = [], []
    for first in range(0, q.shape[2], rows):  # (memory)
        p, z = weights(scores(q[:, :, first:first + rows], k, first, s))
        o.append(apart(p @ v, group))
        lse.append(apart(z, group))
    o, lse = torch.cat(o, 2), torch.cat(lse, 2)
    return unpadded(o, s).to(s["q"].dtype), unpadded(lse, s)[..., 0]


def plain_backward(s):
    q, k, v, do = (padded(s[n], s) for n in ("q", "k", "v", "do"))
    hk, scale = k.shape[1], 1.0 / math.sqrt(q.shape[3])
    group, rows = q.shape[1] // hk, blocks(q, k)
    dq, dk, dv = [], torch.zeros_like(k), torch.zeros_like(v)
    for first in range(0, q.shape[2], rows):  # (memory)
        part = slice(first, first + rows)
        p, _ = weights(scores(q[:, :, part], k, first, s))
        d = grouped(do[:, :, part], hk)
        dp = d @ v.mT.contiguous()
        dy = p * (dp - (p * dp).sum(-1, keepdim=True)) * scale
        dq.append(apart(dy @ k, group))
        dk += dy.mT @ grouped(q[:, :, part], hk)
        dv += p.mT @ d
    return tuple(unpadded(y, s).to(s["q"].dtype) for y in (torch.cat(dq, 2), dk, dv))


def plain_step(s):
    b, t, hq, size = s["q"].shape
    hk, n = s["k"].shape[2], s["k"].shape[1]
    at = s["slots"].long()
    q = grouped(s["q"].transpose(1, 2).float(), hk) / math.sqrt(size)
    pk, pv = (s[m][0].transpose(0, 1).float() for m in ("prefix_k", "prefix_v"))
    k, v = (s[m][at].transpose(1, 2).float() for m in ("k", "v"))
    rows = q.transpose(0, 1).flatten(1, 2)  # of all sequences, by key head
    near = q @ k.mT.contiguous()
    seen = s["lengths"].long()[:, None] - t + torch.arange(t, device=DEVICE) + 1
    seen = torch.arange(n, device=DEVICE) < seen.repeat(1, hq // hk)[:, None, :, None]
    far = (rows @ pk.mT.contiguous()).unflatten(1, (b, -1)).transpose(0, 1)
    p, _ = weights(torch.cat([far, torch.where(seen, near, -torch.inf)], -1))
    far, near = p.split([pk.shape[1], n], -1)
    o = (far.transpose(0, 1).flatten(1, 2) @ pv).unflatten(1, (b, -1)).transpose(0, 1)
    o = apart(o + near @ v, hq // hk)
    return o.transpose(1, 2).to(s["q"].dtype)


# --------------------------------------------------------------------------
# What a pass cannot do without


def seen_pairs(case):
    """(token, key) pairs of all sequences, for one head."""
    t, n = case["tokens"], case.get("keys", 0)
    if case["kind"] == "step":  # keys of the caches only
        return sum(t * m - t * (t - 1) // 2 for m in lengths(case).tolist())
    if case["packed"]:
        return sum(m * (m + 1) // 2 if case["causal"] else m * m for m in lengths(case).tolist())
    return case["batch"] * (t * n - t * (t - 1) // 2 if case["causal"] else t * n)


def work(case):
    e = BYTES[case["dtype"]]
    hq, hk, size = case["q_heads"], case["k_heads"], case["size"]
    pairs, rows = seen_pairs(case), case["batch"] * case["tokens"]
    if case["kind"] == "step":
        keys = case["prefix"] + int(lengths(case).sum())
        pairs += rows * case["prefix"]
        return {"bytes": 2 * rows * hq * size * e + 2 * keys * hk * size * e + 8 * case["batch"],
                "flops": 4 * pairs * hq * size}
    keys = case["batch"] * case["keys"]
    if case["packed"]:
        rows = keys = int(lengths(case).sum())
    qo, kv, lse = rows * hq * size * e, keys * hk * size * e, rows * hq * 4
    if case["kind"] == "forward":
        return {"bytes": 2 * qo + 2 * kv + lse, "flops": 4 * pairs * hq * size}
    return {"bytes": 4 * qo + 4 * kv + lse, "flops": 10 * pairs * hq * size}


# --------------------------------------------------------------------------
# The definition in 64 bits, head by head


def exact(case, seed):
    x = inputs(case, seed)
    if case["kind"] == "step":
        return exact_step(case, x)
    ends = x.get("ends")
    names = [n for n in ("q", "k", "v", "do") if n in x]
    parts = []
    for n in range(case["batch"]):
        y = {m: x[m][0, ends[n]:ends[n + 1]] if ends else x[m][n] for m in names}
        parts.append(exact_sequence(case, y))
    join = (lambda ys: torch.cat(ys)[None]) if ends else torch.stack
    return {m: join([p[m] for p in parts]) for m in parts[0]}


def exact_sequence(case, y):
    t, hq = y["q"].shape[:2]
    n, hk = y["k"].shape[:2]
    group, scale = hq // hk, case["size"] ** -0.5
    i, j = torch.arange(t, device=DEVICE), torch.arange(n, device=DEVICE)
    span = max(1, 2 ** 27 // max(1, n))
    like = {m: torch.zeros(y[m].shape, dtype=torch.float64, device=DEVICE) for m in y}
    lse = torch.zeros(t, hq, dtype=torch.float64, device=DEVICE)
    o = like["q"].clone()
    for h in range(hq):
        k, v = y["k"][:, h // group].double(), y["v"][:, h // group].double()
        for a in range(0, t, span):
            q = y["q"][a:a + span, h].double()
            z = torch.mm(q, k.T) * scale
            if case["causal"]:
                z.masked_fill_(j[None] - i[a:a + span, None] > n - t, -math.inf)
            total = torch.logsumexp(z, -1)
            p = z.sub_(torch.where(total == -math.inf, 0.0, total)[:, None]).exp_()
            if case["kind"] == "forward":
                lse[a:a + span, h] = total
                o[a:a + span, h] = torch.mm(p, v)
                continue
            d = y["do"][a:a + span, h].double()
            like["v"][:, h // group] += torch.mm(p.T, d)
            g = torch.mm(d, v.T)
            mean = torch.linalg.vecdot(p, g)
            g = g.sub_(mean[:, None]).mul_(p)
            like["q"][a:a + span, h] = scale * torch.mm(g, k)
            like["k"][:, h // group] += scale * torch.mm(g.T, q)
    if case["kind"] == "forward":
        return {"o": o, "lse": lse}
    return {"dq": like["q"], "dk": like["k"], "dv": like["v"]}


def exact_step(case, x):
    b, t, hq, size = x["q"].shape
    group = hq // x["k"].shape[2]
    o = torch.zeros(b, t, hq, size, dtype=torch.float64, device=DEVICE)
    slots, filled = x["slots"].tolist(), x["lengths"].tolist()
    prefix = [(x["prefix_k"][0, :, h].double(), x["prefix_v"][0, :, h].double())
              for h in range(hq // group)]
    for n in range(b):
        k = x["k"][slots[n], :filled[n]].double()
        v = x["v"][slots[n], :filled[n]].double()
        hidden = torch.ones(t, t, dtype=torch.bool, device=DEVICE).triu(1)
        for h in range(hq // group):
            heads = slice(h * group, (h + 1) * group)
            keys = torch.cat([prefix[h][0], k[:, h]])
            z = torch.tensordot(x["q"][n, :, heads].double(), keys, ([2], [1])) * size ** -0.5
            z[:, :, keys.shape[0] - t:].masked_fill_(hidden[:, None], -math.inf)
            p = torch.softmax(z, -1)
            o[n, :, heads] = torch.tensordot(p, torch.cat([prefix[h][1], v[:, h]]), ([2], [0]))
    return {"o": o}
