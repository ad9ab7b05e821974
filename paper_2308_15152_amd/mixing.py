"""Binding of the token mixing operators: rotary positions and the gated delta
rule.  As in the package's other functions, everything here marshals arguments;
the arithmetic runs in the HIP kernels.

Tensors are (batch, tokens, heads, size); all but the last dimension may have
any strides.  q, k, v, o and their gradients share one type (float32, bfloat16
or float16); decays, strengths, states and tables are float32.

A call runs on the current torch stream or on ``stream`` (a hipStream_t handle).
What it allocates (outputs and a workspace that are not given) is allocated, and
filled where it is, on the stream it runs on; the outputs are kept from reuse
until the stream that is current in the call is through with them, too.  No autograd
graph is recorded, as by the package's other functions: the gradients have
entries of their own.
"""
from __future__ import annotations

import struct

import paper_2308_15152_amd as _pkg

# The C argument structs of include/mixing_emu.h.  A view is a pointer and the
# element strides of batch, token and head.
_ROTARY = struct.Struct("=10i16q3q3q2i")
_FORWARD = struct.Struct("=7if" + "q" + "24q" + "2q" + "2q")
_BACKWARD = struct.Struct("=7if" + "q" + "44q" + "3q" + "2q")
_STEP = struct.Struct("=7if" + "24q" + "3q" + "2i")
_NO_VIEW = (0, 0, 0, 0)

_calls = {}
_dtypes = {}


def _start():
    global _calls
    lib = _pkg.load()
    torch = _pkg._load_torch()
    _dtypes.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
    # whole, and last: other threads take a filled _calls for all of this
    _calls = {name: getattr(lib, name) for name in (
        "rotary_emu", "delta_emu_forward", "delta_emu_backward", "delta_emu_step",
        "delta_emu_forward_workspace", "delta_emu_backward_workspace")}


def _launch(name, dev, stream, args):
    _launch_on(_calls[name], name, dev, stream, args)


def _launch_on(fn, name, dev, stream, args):
    """Calls an entry point of that name with device dev as the current one."""
    torch = _pkg._torch
    if dev == torch._C._cuda_getDevice():
        rc = fn(args, torch._C._cuda_getCurrentRawStream(dev) if stream is None else int(stream))
    else:
        with torch.cuda.device(dev):
            rc = fn(args, torch._C._cuda_getCurrentRawStream(dev) if stream is None
                    else int(stream))
    if rc != 0:
        raise _pkg.SgemmEmuError(rc, name)


def _side(stream, device):
    """The torch stream of a handle, None if it is the current one's."""
    torch = _pkg._torch
    if device.type != "cuda":
        return None
    index = torch.cuda.current_device() if device.index is None else device.index
    if int(stream) == torch._C._cuda_getCurrentRawStream(index):
        return None
    return torch.cuda.ExternalStream(int(stream), device=device)


def _new(stream, shape, dtype, device, zero=False):
    """A new tensor, made and filled on the stream that the call runs on: memory that
    the current stream is still to read or write is not given out, and the fill comes before
    the kernels.  The caller has it on the current stream, so its memory waits for
    that one too."""
    torch = _pkg._torch
    make = torch.zeros if zero else torch.empty
    side = None if stream is None else _side(stream, device)
    if side is None:
        return make(shape, dtype=dtype, device=device)
    current = torch.cuda.current_stream(device)
    with torch.cuda.stream(side):
        t = make(shape, dtype=dtype, device=device)
    t.record_stream(current)
    return t


def _device(*ts):
    """Index of the one device that every tensor given (None skipped) is on."""
    dev = ts[0].get_device()
    for t in ts:
        if t is not None and t.get_device() != dev or dev < 0:
            return _pkg._device_index(*ts)  # says what is wrong
    return dev


def _view(t, name, shape, dtype):
    """(pointer, batch, token and head stride) of a tensor of that shape and
    type whose last dimension is contiguous."""
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    st = t.stride()
    if len(st) == 4:  # (three: per token and head, no inner dimension)
        if st[3] != 1 and shape[3] > 1:
            raise ValueError(f"{name} must be contiguous along its last dimension")
        return (t.data_ptr(), st[0], st[1], st[2])
    return (t.data_ptr(), *st)


def _like(t, stream):
    """A new contiguous tensor like t."""
    if stream is None and t.is_contiguous():
        return _pkg._torch.empty_like(t)
    return _new(stream, t.shape, t.dtype, t.device)


def _sizes(q, k, v):
    """(batch, tokens, key heads, value heads, key size, value size)."""
    if q.dim() != 4 or k.dim() != 4 or v.dim() != 4:
        raise ValueError("q, k and v must be (batch, tokens, heads, size)")
    if q.dtype not in _dtypes:
        raise TypeError(f"q must be float32, bfloat16 or float16, got {q.dtype}")
    b, t, hk, ks = q.shape
    return b, t, hk, v.shape[2], ks, v.shape[3]


def _scale(scale, k_size):
    """The outputs' scale (a key size of 0 is the library's to refuse)."""
    return max(k_size, 1) ** -0.5 if scale is None else scale


def _states(t, name, shape):
    """Pointer of a contiguous float32 tensor of that shape, or 0."""
    if t is None:
        return 0
    if t.dtype is not _pkg._torch.float32:
        raise TypeError(f"{name} must be float32, got {t.dtype}")
    if tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous with shape {shape}, got {tuple(t.shape)}")
    return t.data_ptr()


def _packed(cu_seqlens, batch):
    """(pointer, number of sequences) of the packed sequences' bounds."""
    if cu_seqlens is None:
        return 0, batch
    if cu_seqlens.dtype is not _pkg._torch.int32 or cu_seqlens.dim() != 1 \
            or not cu_seqlens.is_contiguous() or cu_seqlens.shape[0] < 1:
        raise ValueError("cu_seqlens must be a contiguous int32 vector of the sequences + 1")
    if batch != 1:
        raise ValueError("packed sequences come as one batch")
    return cu_seqlens.data_ptr(), cu_seqlens.shape[0] - 1


def _workspace(need, given, device, stream):
    """(tensor, pointer, bytes) of a call's workspace."""
    torch = _pkg._torch
    if given is None:
        if need == 0:
            return None, 0, 0
        given = _new(stream, need, torch.uint8, device)
    elif not given.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return given, given.data_ptr(), given.numel() * given.element_size()


def rotary_emu(q, k, cos, sin, *, positions=None, offset: int = 0, interleaved: bool = False,
               inverse: bool = False, out=None, stream=None):
    """(q, k) with the first ``2 * cos.shape[1]`` elements of every head turned
    by their token's position, in one launch.

    q: (batch, tokens, heads, size); k: the same with its own number of heads,
    or None; cos, sin: contiguous float32 tables (positions, rot / 2), as
    ``rotary_emu_table`` makes them; positions: int32 or int64 (batch,
    tokens) or (tokens,), default 0, 1, ... plus ``offset``.  Pairs are (2i, 2i + 1)
    if ``interleaved``, else (i, i + rot / 2).  ``inverse`` turns back: applied to
    the outputs' gradients it gives the inputs'.  out: (q, k) to write to,
    which may be the inputs themselves.  A position outside the tables gives NaN."""
    if not _calls:
        _start()
    torch = _pkg._torch
    if q.dim() != 4 or q.dtype not in _dtypes:
        raise ValueError("q must be a (batch, tokens, heads, size) tensor of float32, bfloat16 "
                         "or float16")
    b, t, hq, size = q.shape
    dtype = q.dtype
    if out is None:
        oq, ok = _like(q, stream), None if k is None else _like(k, stream)
    else:
        oq, ok = out
    xq, yq = _view(q, "q", q.shape, dtype), _view(oq, "out", q.shape, dtype)
    hk, xk, yk = 0, _NO_VIEW, _NO_VIEW
    if k is not None:
        if k.dim() != 4:
            raise ValueError("k must be (batch, tokens, heads, size)")
        hk = k.shape[2]
        shape = (b, t, hk, size)
        if ok is None:
            raise ValueError("out must hold a tensor for k")
        xk, yk = _view(k, "k", shape, dtype), _view(ok, "out", shape, dtype)
    for name, table in (("cos", cos), ("sin", sin)):
        if table.dtype is not torch.float32 or table.dim() != 2 or not table.is_contiguous():
            raise ValueError(f"{name} must be a contiguous (positions, rot / 2) float32 tensor")
    if cos.shape != sin.shape:
        raise ValueError("cos and sin must have the same shape")
    at, at_batch, at_token, at_bytes = 0, 0, 0, 0
    if positions is not None:
        if positions.dtype is torch.int32:
            at_bytes = 4
        elif positions.dtype is torch.int64:
            at_bytes = 8
        else:
            raise TypeError(f"positions must be int32 or int64, got {positions.dtype}")
        if positions.shape == (b, t):
            at_batch, at_token = positions.stride()
        elif positions.shape == (t,):
            at_token = positions.stride(0)
        else:
            raise ValueError("positions must be (batch, tokens) or (tokens,)")
        at = positions.data_ptr()
        offset = 0
    args = _ROTARY.pack(_dtypes[dtype], b, t, size, 2 * cos.shape[1], 1 if interleaved else 0,
                        1 if inverse else 0, cos.shape[0], hq, hk, *xq, *xk, *yq, *yk,
                        cos.data_ptr(), sin.data_ptr(), at, at_batch, at_token, int(offset),
                        at_bytes, 0)
    _launch("rotary_emu", _device(q, k, cos, sin, positions, oq, ok), stream, args)
    return oq, ok


def rotary_emu_table(rows: int, rot: int, *, base: float = 10000.0, factor: float = 1.0,
                     original: float = 0.0, ramp=None, amplitude: float = 1.0, device=None,
                     stream=None):
    """(cos, sin) tables of ``rotary_emu`` for positions 0 to rows - 1: two
    (rows, rot / 2) float32 tensors of the frequencies base^(-2i / rot).  factor > 1
    divides the frequencies (longer contexts); with ramp = (low, high) the
    pairs that turn more than ``high`` times over ``original`` positions keep theirs
    and those between ``low`` and ``high`` are joined linearly."""
    if not _calls:
        _start()
    torch = _pkg._torch
    low, high = (0.0, 0.0) if ramp is None else ramp
    rows, rot = int(rows), int(rot)
    device = torch.device("cuda" if device is None else device)
    c, s = (_new(stream, (max(rows, 0), max(rot, 0) // 2), torch.float32, device)
            for _ in range(2))
    with _pkg._on_device(c, s):
        rc = _pkg.load().rotary_emu_table(rows, rot, base, factor, original, low, high, amplitude,
                                          c.data_ptr(), s.data_ptr(), _pkg._stream(stream))
    _pkg._check(rc, "rotary_emu_table")
    return c, s


def _forward_args(q, k, v, g, beta, o, initial, final, scale, cu, n, ws, ws_bytes):
    torch = _pkg._torch
    b, t, hk, hv, ks, vs = _sizes(q, k, v)
    dtype, f32 = q.dtype, torch.float32
    values, gates = (b, t, hv, vs), (b, t, hv)
    states = (n, hv, ks, vs)
    return _FORWARD.pack(
        _dtypes[dtype], n, t, hk, hv, ks, vs, _scale(scale, ks), cu,
        *_view(q, "q", q.shape, dtype), *_view(k, "k", q.shape, dtype),
        *_view(v, "v", values, dtype),
        *(_NO_VIEW if g is None else _view(g, "g", gates, f32)),
        *(_NO_VIEW if beta is None else _view(beta, "beta", gates, f32)),
        *(_NO_VIEW if o is None else _view(o, "out", values, dtype)),
        _states(initial, "initial_state", states), _states(final, "final_state", states),
        ws, ws_bytes)


def delta_emu_forward_workspace(q, k, v, g=None, beta=None, *, cu_seqlens=None) -> int:
    """Bytes of workspace that ``delta_emu_forward`` needs for these tensors (a
    host-side query)."""
    if not _calls:
        _start()
    cu, n = _packed(cu_seqlens, q.shape[0])
    need = _calls["delta_emu_forward_workspace"](
        _forward_args(q, k, v, g, beta, None, None, None, None, cu, n, 0, 0))
    if need < 0:
        raise _pkg.SgemmEmuError(need, "delta_emu_forward_workspace")
    return need


def delta_emu_forward(q, k, v, g=None, beta=None, initial_state=None, *, scale=None,
                      cu_seqlens=None, out=None, final_state=None, workspace=None, stream=None):
    """(o, final_state) of the gated delta rule
        S_t = e^g_t S_{t-1} + k_t u_t^T,  u_t = beta_t (v_t - e^g_t S_{t-1}^T k_t),
        o_t = scale S_t^T q_t.

    q, k: (batch, tokens, key heads, key size <= 128); v, o: (batch, tokens, value
    heads, value size), value head h with key head h // (value heads / key
    heads); g (log decays <= 0), beta: (batch, tokens, value heads) float32, or
    None (no decay, beta = 1); states: (batch, value heads, key size, value
    size) float32, contiguous.  scale: key size ** -0.5 by default.
    cu_seqlens: int32 bounds of packed sequences (then batch is 1 and the states
    are per sequence; rows of no sequence are not written, and hold anything in an
    out made here).  out, final_state (may be initial_state) and workspace
    (uint8, ``delta_emu_forward_workspace`` bytes) are allocated if None."""
    if not _calls:
        _start()
    torch = _pkg._torch
    b, t, hk, hv, ks, vs = _sizes(q, k, v)
    cu, n = _packed(cu_seqlens, b)
    device = q.device
    if out is None:
        out = _new(stream, (b, t, hv, vs), q.dtype, device)
    if final_state is None:
        final_state = _new(stream, (n, hv, ks, vs), torch.float32, device)
    dev = _device(q, k, v, g, beta, initial_state, cu_seqlens, out, final_state, workspace)
    args = _forward_args(q, k, v, g, beta, out, initial_state, final_state, scale, cu, n, 0, 0)
    need = _calls["delta_emu_forward_workspace"](args)
    if need < 0:
        raise _pkg.SgemmEmuError(need, "delta_emu_forward")
    if need > 0 or workspace is not None:
        workspace, at, size = _workspace(need, workspace, device, stream)
        args = args[:-16] + struct.pack("=2q", at, size)
    _launch("delta_emu_forward", dev, stream, args)
    return out, final_state


def _backward_args(q, k, v, g, beta, do, grads, initial, dfinal, dinitial, scale, cu, n):
    torch = _pkg._torch
    b, t, hk, hv, ks, vs = _sizes(q, k, v)
    dtype, f32 = q.dtype, torch.float32
    values, gates = (b, t, hv, vs), (b, t, hv)
    states = (n, hv, ks, vs)
    if grads is None:
        out = _NO_VIEW * 5
    else:
        dq, dk, dv, dg, dbeta = grads
        out = (*_view(dq, "dq", q.shape, dtype), *_view(dk, "dk", q.shape, dtype),
               *_view(dv, "dv", values, dtype),
               *(_NO_VIEW if dg is None else _view(dg, "dg", gates, f32)),
               *(_NO_VIEW if dbeta is None else _view(dbeta, "dbeta", gates, f32)))
    return _BACKWARD.pack(
        _dtypes[dtype], n, t, hk, hv, ks, vs, _scale(scale, ks), cu,
        *_view(q, "q", q.shape, dtype), *_view(k, "k", q.shape, dtype),
        *_view(v, "v", values, dtype),
        *(_NO_VIEW if g is None else _view(g, "g", gates, f32)),
        *(_NO_VIEW if beta is None else _view(beta, "beta", gates, f32)),
        *(_NO_VIEW if do is None else _view(do, "do", values, dtype)), *out,
        _states(initial, "initial_state", states), _states(dfinal, "dfinal", states),
        _states(dinitial, "dinitial", states), 0, 0)


def delta_emu_backward_workspace(q, k, v, g=None, beta=None, *, cu_seqlens=None) -> int:
    """Bytes of workspace that ``delta_emu_backward`` needs for these tensors (a
    host-side query)."""
    if not _calls:
        _start()
    cu, n = _packed(cu_seqlens, q.shape[0])
    need = _calls["delta_emu_backward_workspace"](
        _backward_args(q, k, v, g, beta, None, None, None, None, None, None, cu, n))
    if need < 0:
        raise _pkg.SgemmEmuError(need, "delta_emu_backward_workspace")
    return need


def delta_emu_backward(q, k, v, g, beta, do, initial_state=None, dfinal=None, *, scale=None,
                       cu_seqlens=None, out=None, workspace=None, stream=None):
    """(dq, dk, dv, dg, dbeta, dinitial): the gradients of ``delta_emu_forward``
    with these inputs, from do (like o) and dfinal (gradient of the final
    states, or None).  dg and dbeta are None where g or beta is.  out: the six
    tensors to write to (dinitial may be dfinal itself); rows of no packed
    sequence are not written, so tensors made here start as zeros there."""
    if not _calls:
        _start()
    torch = _pkg._torch
    b, t, hk, hv, ks, vs = _sizes(q, k, v)
    cu, n = _packed(cu_seqlens, b)
    if out is None:
        out = [None if x is None else _new(stream, x.shape, x.dtype, q.device,
                                           zero=cu_seqlens is not None)
               for x in (q, k, v, g, beta)]
        out.append(_new(stream, (n, hv, ks, vs), torch.float32, q.device))
    *grads, dinitial = out
    dev = _device(q, k, v, g, beta, do, initial_state, dfinal, cu_seqlens, workspace, *out)
    args = _backward_args(q, k, v, g, beta, do, grads, initial_state, dfinal, dinitial, scale, cu,
                          n)
    need = _calls["delta_emu_backward_workspace"](args)
    if need < 0:
        raise _pkg.SgemmEmuError(need, "delta_emu_backward")
    workspace, at, size = _workspace(need, workspace, q.device, stream)
    args = args[:-16] + struct.pack("=2q", at, size)
    _launch("delta_emu_backward", dev, stream, args)
    return (*grads, dinitial)


def delta_emu_step(q, k, v, g, beta, state, *, slots=None, scale=None, out=None, stream=None):
    """o of the gated delta rule's recurrent form: the tokens of q, k, v, g,
    beta (shapes as for ``delta_emu_forward``; usually one token) on states that
    are updated in place.  state: (slots, value heads, key size, value size)
    float32, contiguous per slot; slots: int32 (batch,), which state each
    sequence has, all different (default: its own number).  A slot outside the
    states leaves its sequence out: zeros for o."""
    if not _calls:
        _start()
    torch = _pkg._torch
    b, t, hk, hv, ks, vs = _sizes(q, k, v)
    dtype, f32 = q.dtype, torch.float32
    values, gates = (b, t, hv, vs), (b, t, hv)
    if out is None:
        out = _new(stream, values, dtype, q.device)
    if state.dtype is not f32 or state.dim() != 4 or state.shape[1:] != (hv, ks, vs):
        raise ValueError(f"state must be a float32 tensor (slots, {hv}, {ks}, {vs})")
    n_slots, stride = state.shape[0], state.stride()
    if stride[1:] != (ks * vs, vs, 1) and state.numel() > 0:
        if not state[0].is_contiguous():
            raise ValueError("each state must be contiguous")
    at = 0
    if slots is not None:
        if slots.dtype is not torch.int32 or slots.shape != (b,) or not slots.is_contiguous():
            raise ValueError("slots must be a contiguous int32 vector of the batch")
        at = slots.data_ptr()
    args = _STEP.pack(
        _dtypes[dtype], b, t, hk, hv, ks, vs, _scale(scale, ks),
        *_view(q, "q", q.shape, dtype), *_view(k, "k", q.shape, dtype),
        *_view(v, "v", values, dtype),
        *(_NO_VIEW if g is None else _view(g, "g", gates, f32)),
        *(_NO_VIEW if beta is None else _view(beta, "beta", gates, f32)),
        *_view(out, "out", values, dtype),
        state.data_ptr(), stride[0] if n_slots > 1 else hv * ks * vs, at, n_slots, 0)
    _launch("delta_emu_step", _device(q, k, v, g, beta, state, slots, out), stream,
            args)
    return out
