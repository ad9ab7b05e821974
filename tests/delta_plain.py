"""Plain 64-bit forms of the token mixing operators, for the tests: the
definitions, one token after another, on the CPU."""
import torch


def by_head(x, heads):
    return x.repeat_interleave(heads // x.shape[2], dim=2)


def delta(q, k, v, g, beta, first, scale=None, bounds=None):
    """(o, final states) in float64 by the recurrence; differentiable.  bounds:
    rows of each packed sequence (q, k, ... are then (1, rows, ...))."""
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    if bounds is not None:
        o, last = [], []
        for n, (lo, hi) in enumerate(zip(bounds, bounds[1:])):
            part = [None if x is None else x[:, lo:hi] for x in (q, k, v, g, beta)]
            a, b = delta(*part, None if first is None else first[n:n + 1], scale)
            o.append(a)
            last.append(b)
        return torch.cat(o, 1), torch.cat(last, 0)
    b, t, hv, vs = v.shape
    q, k = by_head(q.double(), hv), by_head(k.double(), hv)
    v = v.double()
    S = torch.zeros(b, hv, q.shape[-1], vs, dtype=torch.float64) if first is None \
        else first.double()
    o = []
    for i in range(t):
        if g is not None:
            S = S * g[:, i].double().exp()[..., None, None]
        u = v[:, i] - (S * k[:, i, :, :, None]).sum(2)
        if beta is not None:
            u = u * beta[:, i].double()[..., None]
        S = S + k[:, i, :, :, None] * u[:, :, None]
        o.append(scale * (S * q[:, i, :, :, None]).sum(2))
    o = torch.stack(o, 1) if t else torch.zeros_like(v)
    return o, S


def delta_gradients(q, k, v, g, beta, do, first, dfinal, scale=None, bounds=None):
    """(dq, dk, dv, dg, dbeta, dinitial) in float64, through the recurrence."""
    names = [q, k, v, g, beta, first]
    x = [None if y is None else y.double().requires_grad_() for y in names]
    n = q.shape[0] if bounds is None else len(bounds) - 1
    if x[5] is None:
        x[5] = torch.zeros(n, v.shape[2], q.shape[-1], v.shape[-1], dtype=torch.float64,
                           requires_grad=True)
    o, last = delta(*x, scale=scale, bounds=bounds)
    outs, grads = [], []
    if o.requires_grad:
        outs, grads = [o], [do.double()]
    if dfinal is not None:
        outs, grads = outs + [last], grads + [dfinal.double()]
    d = torch.autograd.grad(outs, [y for y in x if y is not None], grads, allow_unused=True)
    d = iter(d)
    out = []
    for y in x:
        e = None if y is None else next(d)
        out.append(torch.zeros_like(y) if y is not None and e is None else e)
    return tuple(out)


def rotary(x, cos, sin, positions, interleaved, inverse):
    """The rotation in float64; positions (batch, tokens)."""
    half = cos.shape[1]
    c, s = cos.double()[positions][:, :, None], sin.double()[positions][:, :, None]
    if inverse:
        s = -s
    y = x.double().clone()
    a = slice(0, 2 * half, 2) if interleaved else slice(0, half)
    b = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
    xa, xb = x[..., a].double(), x[..., b].double()
    y[..., a], y[..., b] = xa * c - xb * s, xa * s + xb * c
    return y
