"""The token mixing entries on the host: every invalid argument is refused
with its documented code before any HIP call, empty calls do nothing, and the
binding's names, constants and checks match the header (no GPU needed: the
pointers below are never dereferenced)."""
import ctypes
import os
import re
import struct

import pytest
import torch

import paper_2308_15152_amd as pkg
from paper_2308_15152_amd import mixing

HEADER = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "include", "mixing_emu.h")
OK, DIM, NULL, STRIDE, ALIAS, UNSUPPORTED = 0, -1, -3, -4, -5, -6
MB = 1 << 20


def text():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def test_header_binding_and_library_name_the_same_functions():
    names = re.findall(r"^\s*(?:int|int64_t)\s+(\w+)\s*\(", text(), flags=re.M)
    assert sorted(names) == sorted(pkg.MIXING_SYMBOLS)
    lib = pkg.load()
    for name in names:
        assert hasattr(lib, name) and callable(getattr(pkg, name)) and name in pkg.__all__


def test_constants():
    found = dict(re.findall(r"^#define\s+SGEMM_EMU_(\w+)\s+(\d+)", open(HEADER).read(), flags=re.M))
    assert {k: int(v) for k, v in found.items()} == {"F32": pkg.F32, "BF16": pkg.BF16,
                                                     "F16": pkg.F16}


def fields(name):
    """Names and C types of a struct's members, arrays and lists taken apart."""
    body = re.search(r"typedef struct \{([^}]*)\}\s*" + name + ";", text()).group(1)
    out = []
    for line in body.split(";"):
        line = line.strip()
        if not line:
            continue
        kind, rest = re.match(r"((?:const\s+)?\w+\s*\**)\s*(.*)", line, flags=re.S).groups()
        for item in rest.split(","):
            n = re.search(r"\[(\d+)\]", item)
            out += [(item.strip(), kind.strip())] * (int(n.group(1)) if n else 1)
    return out


@pytest.mark.parametrize("name,packed", [
    ("rotary_emu_t", mixing._ROTARY), ("delta_emu_forward_t", mixing._FORWARD),
    ("delta_emu_backward_t", mixing._BACKWARD), ("delta_emu_step_t", mixing._STEP)])
def test_packed_structs_are_the_headers(name, packed):
    code = ""
    for _, kind in fields(name):
        code += {"int32_t": "i", "float": "f", "int64_t": "q", "sgemm_emu_view_t": "qqqq"}.get(
            kind, "q" if kind.endswith("*") else "?")
    assert struct.calcsize("=" + code) == struct.calcsize("@" + code)  # no padding
    flat = re.sub(r"(\d+)([a-z])", lambda m: m.group(2) * int(m.group(1)), packed.format[1:])
    assert flat == code


def call(name, packed, values):
    lib = pkg.load()
    args = [values] if name.endswith("workspace") else [values, None]
    return getattr(lib, name)(*[packed.pack(*args[0])] + args[1:])


# ---- rotary ---------------------------------------------------------------

def rotary(dtype=1, batch=2, tokens=3, size=64, rot=32, inter=0, inverse=0, rows=10, heads=(4, 2),
           q=(MB, 768, 256, 64), k=(2 * MB, 384, 128, 64), yq=(3 * MB, 768, 256, 64),
           yk=(4 * MB, 384, 128, 64), cos=5 * MB, sin=6 * MB, at=7 * MB, at_strides=(3, 1),
           offset=0, at_bytes=4):
    return call("rotary_emu", mixing._ROTARY,
                (dtype, batch, tokens, size, rot, inter, inverse, rows, *heads, *q, *k, *yq, *yk,
                 cos, sin, at, *at_strides, offset, at_bytes, 0))


@pytest.mark.parametrize("kw,code", [
    (dict(batch=-1), DIM), (dict(tokens=-1), DIM), (dict(heads=(-1, 2)), DIM),
    (dict(offset=-1), DIM), (dict(rows=-1), DIM),
    (dict(dtype=3), UNSUPPORTED), (dict(rot=31), UNSUPPORTED), (dict(rot=66), UNSUPPORTED),
    (dict(at_bytes=2), UNSUPPORTED), (dict(batch=1 << 16, tokens=1 << 16), UNSUPPORTED),
    (dict(heads=(1 << 25, 2)), UNSUPPORTED),
    (dict(q=(0, 768, 256, 64)), NULL), (dict(yk=(0, 384, 128, 64)), NULL), (dict(cos=0), NULL),
    (dict(q=(MB, -1, 256, 64)), STRIDE), (dict(yq=(3 * MB, 768, 256, 63)), STRIDE),
    (dict(yq=(3 * MB, 768, 0, 64)), STRIDE), (dict(at_strides=(-3, 1)), STRIDE),
    (dict(yq=(MB + 2, 768, 256, 64)), ALIAS), (dict(yq=(2 * MB, 768, 256, 64)), ALIAS),
    (dict(yk=(5 * MB, 384, 128, 64)), ALIAS), (dict(yk=(7 * MB, 384, 128, 64)), ALIAS),
    (dict(batch=0), OK), (dict(tokens=0), OK), (dict(heads=(0, 0)), OK)])
def test_rotary_arguments(kw, code):
    assert rotary(**kw) == code


@pytest.mark.parametrize("args,code", [
    ((-1, 8, 1e4, 1, 0, 0, 0, 1, MB, 2 * MB), DIM), ((4, 7, 1e4, 1, 0, 0, 0, 1, MB, 2 * MB), DIM),
    ((4, 8, 0.0, 1, 0, 0, 0, 1, MB, 2 * MB), UNSUPPORTED),
    ((4, 8, 1e4, 0, 0, 0, 0, 1, MB, 2 * MB), UNSUPPORTED),
    ((4, 8, 1e4, 1, 0, 2, 1, 1, MB, 2 * MB), UNSUPPORTED),
    ((4, 8, float("inf"), 1, 0, 0, 0, 1, MB, 2 * MB), UNSUPPORTED),
    ((4, 8, 1e4, 1, 0, 0, 0, float("nan"), MB, 2 * MB), UNSUPPORTED),
    ((4, 8, 1e4, 1, 0, 0, 0, 1, None, 2 * MB), NULL),
    ((4, 8, 1e4, 1, 0, 0, 0, 1, MB, MB + 32), ALIAS),
    ((0, 8, 1e4, 1, 0, 0, 0, 1, None, None), OK)])
def test_rotary_table_arguments(args, code):
    assert pkg.load().rotary_emu_table(*args, None) == code


# ---- the delta rule ---------------------------------------------------------

def shape(**kw):
    s = dict(dtype=1, batch=2, tokens=100, k_heads=2, v_heads=4, k_size=64, v_size=32, scale=0.125)
    s.update(kw)
    return s


def view(at, s, heads, size):
    return (at * MB, s["tokens"] * heads * size, heads * size, size)


def tensors(s, cu):
    """Well separated q, k, v, g, beta, o."""
    hk, hv = s["k_heads"], s["v_heads"]
    v = {"q": view(1, s, hk, s["k_size"]), "k": view(2, s, hk, s["k_size"]),
         "v": view(3, s, hv, s["v_size"]), "g": view(4, s, hv, 1), "beta": view(5, s, hv, 1),
         "o": view(6, s, hv, s["v_size"])}
    return v


def forward(query=False, cu=0, initial=8 * MB, final=9 * MB, ws=1 << 30, ws_bytes=1 << 40,
            views=None, **kw):
    s = shape(**kw)
    t = tensors(s, cu)
    t.update(views or {})
    values = (*s.values(), cu, *(x for v in t.values() for x in v), initial, final, ws, ws_bytes)
    return call("delta_emu_forward" + ("_workspace" if query else ""), mixing._FORWARD, values)


SIZES = [
    (dict(dtype=7), UNSUPPORTED), (dict(batch=-1), DIM), (dict(tokens=-1), DIM),
    (dict(v_size=-1), DIM), (dict(v_size=65537), UNSUPPORTED), (dict(k_size=0), UNSUPPORTED),
    (dict(k_size=129), UNSUPPORTED),
    (dict(k_heads=0), UNSUPPORTED), (dict(k_heads=3), UNSUPPORTED),
    (dict(batch=1 << 20, tokens=65), UNSUPPORTED),  # more than 2^21 (chunk, head) pairs
]


@pytest.mark.parametrize("kw,code", SIZES + [
    (dict(batch=0), OK), (dict(v_size=0), OK),
    (dict(views={"q": (0, 1, 1, 1)}), NULL), (dict(views={"o": (0, 1, 1, 1)}), NULL),
    (dict(ws=0), NULL), (dict(ws_bytes=1000), DIM), (dict(ws=(1 << 30) + 16), DIM),
    (dict(views={"k": (2 * MB, -1, 128, 64)}), STRIDE),
    (dict(views={"k": (2 * MB, 1, 1 << 23, 64)}), UNSUPPORTED),
    (dict(views={"o": (6 * MB, 12800, 128, 31)}), STRIDE),
    (dict(views={"o": (6 * MB, 0, 128, 32)}), STRIDE),
    (dict(views={"o": (MB, 12800, 128, 32)}), ALIAS), (dict(final=MB), ALIAS),
    (dict(final=8 * MB + 64), ALIAS), (dict(ws=8 << 20), ALIAS), (dict(ws=6 << 20), ALIAS),
    (dict(cu=6 * MB), ALIAS)])
def test_forward_arguments(kw, code):
    assert forward(**kw) == code


def test_forward_workspace():
    assert forward(query=True, tokens=16) == 0  # token by token
    one = forward(query=True, tokens=64, batch=1)
    assert one > 0 and one % 256 == 0
    assert forward(query=True, tokens=65, batch=1) == 2 * one
    # packed sequences may each leave a chunk partly used
    assert forward(query=True, tokens=64, batch=3, cu=MB) == 4 * one
    for kw, code in SIZES:
        assert forward(query=True, **kw) == code


def backward(query=False, cu=0, initial=20 * MB, dfinal=21 * MB, dinitial=22 * MB, ws=1 << 32,
             ws_bytes=1 << 40, views=None, **kw):
    s = shape(**kw)
    t = tensors(s, cu)
    for i, n in enumerate(("q", "k", "v", "g", "beta")):
        t["d" + n] = (t[n][0] + 10 * MB, *t[n][1:])
    t.update(views or {})
    values = (*s.values(), cu, *(x for v in t.values() for x in v), initial, dfinal, dinitial, ws,
              ws_bytes)
    return call("delta_emu_backward" + ("_workspace" if query else ""), mixing._BACKWARD, values)


@pytest.mark.parametrize("kw,code", SIZES + [
    (dict(batch=0), OK), (dict(views={"o": (0, 1, 1, 1)}), NULL),
    (dict(views={"dk": (0, 1, 1, 1)}), NULL), (dict(ws=0), NULL), (dict(ws_bytes=1000), DIM),
    (dict(views={"dq": (11 * MB, 12800, 128, 63)}), STRIDE),
    (dict(views={"dv": (3 * MB, 12800, 128, 32)}), ALIAS),
    (dict(views={"dg": (5 * MB, 400, 4, 1)}), ALIAS), (dict(dinitial=20 * MB), ALIAS),
    (dict(dinitial=21 * MB + 4), ALIAS), (dict(ws=(20 << 20)), ALIAS)])
def test_backward_arguments(kw, code):
    assert backward(**kw) == code


def step(state=8 * MB, stride=4 * 64 * 32, slots=10 * MB, n_slots=8, views=None, **kw):
    s = shape(**{"tokens": 1, **kw})
    t = tensors(s, 0)
    t.update(views or {})
    values = (*s.values(), *(x for v in t.values() for x in v), state, stride, slots, n_slots, 0)
    return call("delta_emu_step", mixing._STEP, values)


@pytest.mark.parametrize("kw,code", SIZES[:-1] + [
    (dict(n_slots=-1), DIM), (dict(slots=0, n_slots=1), DIM), (dict(stride=8191), STRIDE),
    (dict(state=0), NULL), (dict(views={"v": (0, 1, 1, 1)}), NULL),
    (dict(state=6 * MB), ALIAS), (dict(state=MB), ALIAS), (dict(state=10 * MB), ALIAS),
    (dict(views={"o": (MB, 128, 128, 32)}), ALIAS), (dict(batch=0), OK), (dict(tokens=0), OK)])
def test_step_arguments(kw, code):
    assert step(**kw) == code


@pytest.mark.parametrize("name", [n for n in pkg.MIXING_SYMBOLS if n != "rotary_emu_table"])
def test_null_struct(name):
    fn = getattr(pkg.load(), name)
    assert fn(*[None] * len(fn.argtypes)) == NULL


# ---- the binding's own checks -----------------------------------------------

def delta_inputs(dtype=torch.bfloat16):
    q = torch.zeros(2, 20, 2, 16, dtype=dtype)
    v = torch.zeros(2, 20, 4, 8, dtype=dtype)
    g = torch.zeros(2, 20, 4)
    return q, q.clone(), v, g, g.clone()


def test_tensors_must_be_on_a_device():
    q, k, v, g, beta = delta_inputs()
    state = torch.zeros(2, 4, 16, 8)
    cos = torch.zeros(32, 4)
    with pytest.raises(ValueError):
        pkg.delta_emu_forward(q, k, v, g, beta)
    with pytest.raises(ValueError):
        pkg.delta_emu_backward(q, k, v, g, beta, v)
    with pytest.raises(ValueError):
        pkg.delta_emu_step(q, k, v, g, beta, state)
    with pytest.raises(ValueError):
        pkg.rotary_emu(q, k, cos, cos.clone())


@pytest.mark.parametrize("change", [
    dict(k=torch.zeros(2, 20, 2, 17, dtype=torch.bfloat16)),
    dict(v=torch.zeros(2, 21, 4, 8, dtype=torch.bfloat16)), dict(g=torch.zeros(2, 20, 3)),
    dict(q=torch.zeros(20, 2, 16, dtype=torch.bfloat16)),
    dict(q=torch.zeros(2, 20, 16, 2, dtype=torch.bfloat16).transpose(2, 3))])
def test_shapes_are_checked(change):
    x = dict(zip(("q", "k", "v", "g", "beta"), delta_inputs()), **change)
    with pytest.raises(ValueError):
        pkg.delta_emu_forward(**x)


@pytest.mark.parametrize("change", [
    dict(k=torch.zeros(2, 20, 2, 16)), dict(q=torch.zeros(2, 20, 2, 16, dtype=torch.float64)),
    dict(g=torch.zeros(2, 20, 4, dtype=torch.bfloat16)),
    dict(initial_state=torch.zeros(2, 4, 16, 8, dtype=torch.bfloat16))])
def test_types_are_checked(change):
    x = dict(zip(("q", "k", "v", "g", "beta"), delta_inputs()), **change)
    with pytest.raises((TypeError, ValueError)):
        pkg.delta_emu_forward(**x)


def test_other_arguments_are_checked():
    q, k, v, g, beta = delta_inputs()
    with pytest.raises(ValueError):  # packed sequences come as one batch
        pkg.delta_emu_forward(q, k, v, g, beta, cu_seqlens=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        pkg.delta_emu_forward(q[:1], k[:1], v[:1], g[:1], beta[:1],
                              cu_seqlens=torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError):
        pkg.delta_emu_forward(q, k, v, g, beta, torch.zeros(2, 4, 8, 16))
    state = torch.zeros(5, 4, 16, 8)
    with pytest.raises(ValueError):
        pkg.delta_emu_step(q, k, v, g, beta, state[:, :3])
    with pytest.raises(ValueError):
        pkg.delta_emu_step(q, k, v, g, beta, state, slots=torch.zeros(3, dtype=torch.int32))
    cos = torch.zeros(32, 4)
    with pytest.raises(ValueError):
        pkg.rotary_emu(q, k, cos, torch.zeros(32, 5))
    with pytest.raises(ValueError):
        pkg.rotary_emu(q, k, cos, cos.clone(), positions=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(TypeError):
        pkg.rotary_emu(q, k, cos, cos.clone(), positions=torch.zeros(20))


def test_workspace_queries_through_the_binding():
    q, k, v, g, beta = delta_inputs()
    assert pkg.delta_emu_forward_workspace(q, k, v, g, beta) > 0
    assert pkg.delta_emu_backward_workspace(q, k, v, g, beta) > \
        pkg.delta_emu_forward_workspace(q, k, v, g, beta)
    with pytest.raises(pkg.SgemmEmuError):
        big = torch.zeros(1, 1, 1, 200)
        pkg.delta_emu_forward_workspace(big, big, big)
    assert ctypes.sizeof(ctypes.c_void_p) == 8
