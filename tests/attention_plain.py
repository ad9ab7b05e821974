"""Softmax attention and its gradient in 64 bits, on the CPU, with the most that the
kernels' roundings can move each result.

With u half a step of the type (the operands' weights and the results are rounded to it) and
e = 2^-24 for FP32, for each element:
  scores: |ds_ij| <= (size + 4) e b_ij, b_ij = |scale| sum |q_id k_jd|, so that a weight
    is off by 2 w relative, w = (size + 8) e max_j b_ij + (keys + 64) e (scores, the row's sum,
    exponentials of arguments rounded relative to the largest score);
  o: (u + 2 w) sum_j p_ij |v_jd| + u |o_id|;
  lse: w + 4 e |lse|;
  delta_i from an o that is rounded itself: d_i = (u + (size + 4) e) sum |do_id o_id|;
  ds_ij: p_ij (2 w g_ij + d_i) + u |ds_ij|, g_ij = sum |do_id v_jd| + sum |do_id o_id|;
  gradients: the sums of those with |k|, |q| and |do|, sums of n terms n e more, and u
    of the result.
A result that is subnormal is off by half of the type's smallest step, and where weights of FP16
are small against a column's largest by 2^-24 of that at most."""
import math

import torch

E = 2.0 ** -24


def unit(dtype):
    return torch.finfo(dtype).eps / 2


def least(dtype):
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


def attention(q, k, v, causal=True, scale=None, do=None, lengths=None):
    """One sequence: q (tokens, query heads, size), k, v (keys, key heads, size).  Returns
    {name: (value, bound)} for o, lse and, with do, dq, dk and dv."""
    dtype = q.dtype
    u = unit(dtype) if dtype != torch.float32 else 0.0
    r = unit(dtype)
    t, hq, size = q.shape
    n, hk, _ = k.shape
    group = hq // hk
    scale = size ** -0.5 if scale is None else scale
    q, k, v = (x.detach().cpu().double().movedim(1, 0) for x in (q, k, v))
    kk, vv = k.repeat_interleave(group, 0), v.repeat_interleave(group, 0)
    s = scale * q @ kk.mT
    b = abs(scale) * q.abs() @ kk.abs().mT
    seen = torch.ones(t, n, dtype=torch.bool)
    if causal:
        seen = torch.arange(n) <= torch.arange(t)[:, None] + n - t
    s = torch.where(seen, s, -math.inf)
    b = torch.where(seen, b, 0.0)
    lse = torch.logsumexp(s, -1) if n else torch.full((hq, t), -math.inf, dtype=torch.float64)
    none = ~seen.any(-1)
    p = torch.where(none[:, None], 0.0, (s - torch.where(none, 0.0, lse)[..., None]).exp())
    most = b.amax(-1) if n else torch.zeros_like(lse)
    w = (size + 8) * E * most + (n + 64) * E
    seen_v = torch.where(torch.isfinite(vv), vv, 0.0)
    o = p @ seen_v
    o_bound = (u + 2 * w)[..., None] * (p @ seen_v.abs()) + r * o.abs() + least(dtype)
    out = {"o": (o, o_bound), "lse": (lse, w + 4 * E * torch.where(none, 0.0, lse).abs())}
    if do is not None:
        d = do.detach().cpu().double().movedim(1, 0)
        g = d @ vv.mT
        mean = (d * o).sum(-1)
        mean_abs = (d * o).abs().sum(-1)
        ds = p * (g - mean[..., None])
        ds_bound = p * (2 * w[..., None] * (d.abs() @ vv.abs().mT + mean_abs[..., None])
                        + ((unit(dtype) + (size + 4) * E) * mean_abs)[..., None]) + u * ds.abs()
        fold = lambda x: x.unflatten(0, (hk, group)).sum(1)  # noqa: E731
        ds_low = E * ds.abs().amax(-1, keepdim=True) if n else 0.0
        ds_high = E * ds.abs().amax(-2, keepdim=True) if t else 0.0
        a = abs(scale)
        dq = scale * ds @ kk
        out["dq"] = (dq, a * (ds_bound + n * E * ds.abs() + ds_low) @ kk.abs())
        dk = fold(scale * ds.mT @ q)
        out["dk"] = (dk, fold(a * (ds_bound + t * group * E * ds.abs() + ds_high).mT @ q.abs()))
        dv = fold(p.mT @ d)
        out["dv"] = (dv, fold(((u + 2 * w + t * group * E)[..., None] * p + 2.0 ** -38).mT
                              @ d.abs()))
        for m in ("dq", "dk", "dv"):
            out[m] = (out[m][0], out[m][1] + r * out[m][0].abs() + least(dtype))
    move = lambda x: x.movedim(0, 1) if x.dim() == 3 else x.mT  # noqa: E731
    return {m: (move(x), move(y)) for m, (x, y) in out.items()}


def near(got, want, what=""):
    value, bound = want
    got = got.detach().cpu().double()
    assert got.shape == value.shape, what
    fine = torch.isfinite(value)
    assert torch.equal(got[~fine], value[~fine]), what
    off = (got - value)[fine].abs()
    assert not torch.isnan(off).any(), what
    over = off > bound.expand_as(value)[fine]
    assert not over.any(), (what, int(over.sum()), float((off / bound.expand_as(value)[fine]).max()))
