"""Binding of the softmax attention operators.  As in the package's other functions,
everything here marshals arguments; the arithmetic runs in the HIP kernels.

Tensors are (batch, tokens, heads, size); all but the last dimension may have
any strides.  q, k, v, o and their gradients share one type (float32, bfloat16 or float16);
log-sums are float32.  Streams, allocation and autograd are as for the token mixing
operators: a call runs on the current torch stream or on ``stream`` (a hipStream_t handle),
what it allocates belongs to the stream it runs on, and no graph is recorded.
"""
from __future__ import annotations

import struct

import paper_2308_15152_amd as _pkg
from paper_2308_15152_amd.mixing import (
    _NO_VIEW, _device, _launch_on, _like, _new, _packed, _view, _workspace)

# The C argument structs of include/attention_emu.h.
_FORWARD = struct.Struct("=8ifi2q20q2q")
_BACKWARD = struct.Struct("=8ifi2q36q2q")
_STEP = struct.Struct("=9if24q2q2q")

_calls = {}
_dtypes = {}


def _start():
    global _calls
    lib = _pkg.load()
    torch = _pkg._load_torch()
    _dtypes.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
    # whole, and last: other threads take a filled _calls for all of this
    _calls = {name: getattr(lib, name) for name in _pkg.ATTENTION_SYMBOLS}


def _launch(name, dev, stream, args):
    _launch_on(_calls[name], name, dev, stream, args)


def _sizes(q, k):
    """(batch, tokens, keys, query heads, key heads, size)."""
    shape, keys = q.shape, k.shape
    if len(shape) != 4 or len(keys) != 4:
        raise ValueError("q, k and v must be (batch, tokens, heads, size)")
    if q.dtype not in _dtypes:
        raise TypeError(f"q must be float32, bfloat16 or float16, got {q.dtype}")
    return shape[0], shape[1], keys[1], shape[2], keys[2], shape[3]


def _bounds(cu_seqlens, cu_keys, batch):
    """(pointers of both bounds, number of sequences)."""
    if cu_keys is not None and cu_seqlens is None:
        raise ValueError("cu_seqlens_k needs cu_seqlens")
    at, n = _packed(cu_seqlens, batch)
    if cu_keys is None:
        return at, 0, n
    keys_at, m = _packed(cu_keys, batch)
    if m != n:
        raise ValueError("cu_seqlens and cu_seqlens_k must have the same length")
    return at, keys_at, n


def _alike(x, shape, dtype):
    """Whether a (batch, tokens, heads, size) tensor needs no closer look: _view says what is
    wrong with it, at four times the price."""
    return x.dtype is dtype and x.shape == shape and x.stride(3) == 1


def _forward_args(q, k, v, out, lse, causal, scale, cu, cu_k, n):
    b, t, n_keys, hq, hk, size = _sizes(q, k)
    dtype, shape, f32 = q.dtype, q.shape, _pkg._torch.float32
    keys = (b, n_keys, hk, size)
    head = (_dtypes[dtype], n, t, n_keys, hq, hk, size, 1 if causal else 0,
            max(size, 1) ** -0.5 if scale is None else scale, 0, cu, cu_k)
    if out is not None and _alike(q, shape, dtype) and _alike(k, keys, dtype) \
            and _alike(v, keys, dtype) and _alike(out, shape, dtype) and lse.dtype is f32 \
            and lse.shape == (b, t, hq):
        sq, sk, sv, so = q.stride(), k.stride(), v.stride(), out.stride()
        return _FORWARD.pack(
            *head, q.data_ptr(), sq[0], sq[1], sq[2], k.data_ptr(), sk[0], sk[1], sk[2],
            v.data_ptr(), sv[0], sv[1], sv[2], out.data_ptr(), so[0], so[1], so[2],
            lse.data_ptr(), *lse.stride(), 0, 0)
    results = _NO_VIEW * 2 if out is None else (
        *_view(out, "out", shape, dtype), *_view(lse, "lse", (b, t, hq), f32))
    return _FORWARD.pack(*head, *_view(q, "q", shape, dtype), *_view(k, "k", keys, dtype),
                         *_view(v, "v", keys, dtype), *results, 0, 0)


def attention_emu_forward_workspace(q, k, v, *, causal: bool = True, cu_seqlens=None,
                                    cu_seqlens_k=None) -> int:
    """Bytes of workspace that ``attention_emu_forward`` needs for these tensors (a
    host-side query)."""
    if not _calls:
        _start()
    cu, cu_k, n = _bounds(cu_seqlens, cu_seqlens_k, q.shape[0])
    need = _calls["attention_emu_forward_workspace"](
        _forward_args(q, k, v, None, None, causal, None, cu, cu_k, n))
    if need < 0:
        raise _pkg.SgemmEmuError(need, "attention_emu_forward_workspace")
    return need


def attention_emu_forward(q, k, v, *, causal: bool = True, scale=None, cu_seqlens=None,
                          cu_seqlens_k=None, out=None, lse=None, workspace=None, stream=None):
    """(o, lse) of softmax attention over whole sequences: for token i
        s_j = scale q_i k_j,  lse_i = log sum_j e^s_j,  o_i = sum_j e^(s_j - lse_i) v_j
    over the keys that it sees.

    q, o: (batch, tokens, query heads, size <= 128); k, v: (batch, keys, key heads, size),
    query head h with key head h // (query heads / key heads); lse: (batch, tokens, query
    heads) float32.  causal: token i of t sees keys 0 to i + keys - t (the last one all), else
    every token sees all; a token that sees none has zeros and -infinity.  scale: size ** -0.5
    by default.  cu_seqlens: int32 bounds of packed sequences (then batch is 1; rows of no
    sequence are not written, and hold anything in tensors made here); cu_seqlens_k: those of
    the keys, if they are others.  out, lse and workspace (uint8,
    ``attention_emu_forward_workspace`` bytes) are allocated if None."""
    if not _calls:
        _start()
    cu, cu_k, n = _bounds(cu_seqlens, cu_seqlens_k, q.shape[0])
    device = q.device
    if out is None:
        out = _like(q, stream)
    if lse is None:
        lse = _new(stream, q.shape[:3], _pkg._torch.float32, device)
    args = _forward_args(q, k, v, out, lse, causal, scale, cu, cu_k, n)
    dev = _device(q, k, v, cu_seqlens, cu_seqlens_k, out, lse, workspace)
    need = _calls["attention_emu_forward_workspace"](args)
    if need < 0:
        raise _pkg.SgemmEmuError(need, "attention_emu_forward")
    if need > 0 or workspace is not None:
        workspace, at, size = _workspace(need, workspace, device, stream)
        args = args[:-16] + struct.pack("=2q", at, size)
    _launch("attention_emu_forward", dev, stream, args)
    return out, lse


def _backward_args(q, k, v, o, lse, do, grads, causal, scale, cu, cu_k, n):
    b, t, n_keys, hq, hk, size = _sizes(q, k)
    dtype, shape, f32 = q.dtype, q.shape, _pkg._torch.float32
    keys = (b, n_keys, hk, size)
    head = (_dtypes[dtype], n, t, n_keys, hq, hk, size, 1 if causal else 0,
            max(size, 1) ** -0.5 if scale is None else scale, 0, cu, cu_k)
    if grads is not None:
        dq, dk, dv = grads
        if all(_alike(x, shape, dtype) for x in (q, o, do, dq)) \
                and all(_alike(x, keys, dtype) for x in (k, v, dk, dv)) \
                and lse.dtype is f32 and lse.shape == (b, t, hq):
            views = []
            for x in (q, k, v, o, lse, do, dq, dk, dv):
                views.append(x.data_ptr())
                views += x.stride()[:3]
            return _BACKWARD.pack(*head, *views, 0, 0)
    rest = _NO_VIEW * 6 if grads is None else (
        *_view(o, "o", shape, dtype), *_view(lse, "lse", (b, t, hq), f32),
        *_view(do, "do", shape, dtype), *_view(grads[0], "dq", shape, dtype),
        *_view(grads[1], "dk", keys, dtype), *_view(grads[2], "dv", keys, dtype))
    return _BACKWARD.pack(*head, *_view(q, "q", shape, dtype), *_view(k, "k", keys, dtype),
                          *_view(v, "v", keys, dtype), *rest, 0, 0)


def attention_emu_backward_workspace(q, k, v, *, causal: bool = True, cu_seqlens=None,
                                     cu_seqlens_k=None) -> int:
    """Bytes of workspace that ``attention_emu_backward`` needs for these tensors (a
    host-side query)."""
    if not _calls:
        _start()
    cu, cu_k, n = _bounds(cu_seqlens, cu_seqlens_k, q.shape[0])
    need = _calls["attention_emu_backward_workspace"](
        _backward_args(q, k, v, None, None, None, None, causal, None, cu, cu_k, n))
    if need < 0:
        raise _pkg.SgemmEmuError(need, "attention_emu_backward_workspace")
    return need


def attention_emu_backward(q, k, v, o, lse, do, *, causal: bool = True, scale=None,
                           cu_seqlens=None, cu_seqlens_k=None, out=None, workspace=None,
                           stream=None):
    """(dq, dk, dv): the gradients of ``attention_emu_forward`` with these inputs, from its
    results o and lse (which may be of more keys than are given) and from do (like o).  out:
    the three tensors to write to; rows of no packed sequence are not written, so tensors made
    here start as zeros there.  workspace: uint8, ``attention_emu_backward_workspace`` bytes,
    allocated if None."""
    if not _calls:
        _start()
    cu, cu_k, n = _bounds(cu_seqlens, cu_seqlens_k, q.shape[0])
    if out is None:
        out = [_like(x, stream) if cu_seqlens is None else
               _new(stream, x.shape, x.dtype, q.device, zero=True) for x in (q, k, v)]
    dev = _device(q, k, v, o, lse, do, cu_seqlens, cu_seqlens_k, workspace, *out)
    args = _backward_args(q, k, v, o, lse, do, out, causal, scale, cu, cu_k, n)
    need = _calls["attention_emu_backward_workspace"](args)
    if need < 0:
        raise _pkg.SgemmEmuError(need, "attention_emu_backward")
    workspace, at, size = _workspace(need, workspace, q.device, stream)
    _launch("attention_emu_backward", dev, stream, args[:-16] + struct.pack("=2q", at, size))
    return tuple(out)


def _step_args(q, k, v, lengths, prefix_k, prefix_v, slots, scale, out):
    b, t, capacity, hq, hk, size = _sizes(q, k)
    dtype, caches = q.dtype, k.shape[:3] + q.shape[3:]
    if (prefix_k is None) != (prefix_v is None):
        raise ValueError("prefix_k and prefix_v come together")
    prefix, views = 0, _NO_VIEW * 2
    if prefix_k is not None:
        if prefix_k.dim() != 4:
            raise ValueError("prefix_k and prefix_v must be (1, prefix, key heads, size)")
        prefix = prefix_k.shape[1]
        shape = (1, prefix, hk, size)
        if _alike(prefix_k, shape, dtype) and _alike(prefix_v, shape, dtype):
            sk, sv = prefix_k.stride(), prefix_v.stride()
            views = (prefix_k.data_ptr(), sk[0], sk[1], sk[2],
                     prefix_v.data_ptr(), sv[0], sv[1], sv[2])
        else:
            views = (*_view(prefix_k, "prefix_k", shape, dtype),
                     *_view(prefix_v, "prefix_v", shape, dtype))
    for name, x in (("lengths", lengths), ("slots", slots)):
        if x is not None and (x.dtype is not _pkg._torch.int32 or x.shape != (b,)
                              or not x.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous int32 vector of the batch")
    head = (_dtypes[dtype], b, t, prefix, capacity, k.shape[0], hq, hk, size,
            max(size, 1) ** -0.5 if scale is None else scale)
    tail = (0 if lengths is None else lengths.data_ptr(), 0 if slots is None else slots.data_ptr(),
            0, 0)
    if out is not None and _alike(q, q.shape, dtype) and _alike(k, caches, dtype) \
            and _alike(v, caches, dtype) and _alike(out, q.shape, dtype):
        sq, sk, sv, so = q.stride(), k.stride(), v.stride(), out.stride()
        return _STEP.pack(
            *head, q.data_ptr(), sq[0], sq[1], sq[2], *views, k.data_ptr(), sk[0], sk[1], sk[2],
            v.data_ptr(), sv[0], sv[1], sv[2], out.data_ptr(), so[0], so[1], so[2], *tail)
    return _STEP.pack(*head, *_view(q, "q", q.shape, dtype), *views, *_view(k, "k", caches, dtype),
                      *_view(v, "v", caches, dtype),
                      *(_NO_VIEW if out is None else _view(out, "out", q.shape, dtype)), *tail)


def attention_emu_step_workspace(q, k, v, prefix_k=None, prefix_v=None, *, slots=None) -> int:
    """Bytes of workspace that ``attention_emu_step`` needs for these tensors (a host-side
    query)."""
    if not _calls:
        _start()
    need = _calls["attention_emu_step_workspace"](
        _step_args(q, k, v, None, prefix_k, prefix_v, slots, None, None))
    if need < 0:
        raise _pkg.SgemmEmuError(need, "attention_emu_step_workspace")
    return need


def attention_emu_step(q, k, v, lengths, prefix_k=None, prefix_v=None, *, slots=None, scale=None,
                       out=None, workspace=None, stream=None):
    """o of attention for the newest tokens of a batch of sequences, whose keys and values
    are a prefix that all share, read once for all of them, and a cache of each one's own.

    q: (batch, tokens, query heads, size <= 128), usually one token, or a few drafted
    ones; k, v: caches (slots, capacity, key heads, size) that hold the new tokens' keys and
    values already; lengths: int32 (batch,), how many positions of its cache each sequence
    has, the new ones among them; prefix_k, prefix_v: (1, prefix, key heads, size) or None;
    slots: int32 (batch,), which cache each sequence has (default: its own number).  Token i
    of t sees the prefix and positions 0 to lengths - t + i.  A slot outside the caches leaves
    its sequence out: zeros for o.  workspace: uint8, ``attention_emu_step_workspace`` bytes,
    allocated if None."""
    if not _calls:
        _start()
    if lengths is None:
        raise ValueError("lengths must be a contiguous int32 vector of the batch")
    if out is None:
        out = _like(q, stream)
    args = _step_args(q, k, v, lengths, prefix_k, prefix_v, slots, scale, out)
    dev = _device(q, k, v, lengths, prefix_k, prefix_v, slots, out, workspace)
    need = _calls["attention_emu_step_workspace"](args)
    if need < 0:
        raise _pkg.SgemmEmuError(need, "attention_emu_step")
    if need > 0 or workspace is not None:
        workspace, at, size = _workspace(need, workspace, q.device, stream)
        args = args[:-16] + struct.pack("=2q", at, size)
    _launch("attention_emu_step", dev, stream, args)
    return out
