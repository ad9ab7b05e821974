"""The attention entries on the host: every invalid argument is refused with its
documented code before any HIP call, empty calls do nothing, and the binding's names and
checks match the header (no GPU needed: the pointers below are never dereferenced)."""
import os
import re
import struct

import pytest
import torch

import paper_2308_15152_amd as pkg
from paper_2308_15152_amd import attention

HEADER = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "include",
                      "attention_emu.h")
OK, DIM, NULL, STRIDE, ALIAS, UNSUPPORTED = 0, -1, -3, -4, -5, -6
MB = 1 << 20
BIG = 2 ** 31 - 1


def text():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def test_header_binding_and_library_name_the_same_functions():
    names = re.findall(r"^\s*(?:int|int64_t)\s+(\w+)\s*\(", text(), flags=re.M)
    assert sorted(names) == sorted(pkg.ATTENTION_SYMBOLS)
    lib = pkg.load()
    for name in names:
        assert hasattr(lib, name) and callable(getattr(pkg, name)) and name in pkg.__all__


@pytest.mark.parametrize("name,packed", [
    ("attention_emu_forward_t", attention._FORWARD),
    ("attention_emu_backward_t", attention._BACKWARD), ("attention_emu_step_t", attention._STEP)])
def test_packed_structs_are_the_headers(name, packed):
    body = re.search(r"typedef struct \{([^}]*)\}\s*" + name + ";", text()).group(1)
    code = ""
    for line in filter(None, (x.strip() for x in body.split(";"))):
        kind, names = re.match(r"((?:const\s+)?\w+\s*\**)\s*(.*)", line, flags=re.S).groups()
        kind = kind.strip()
        code += len(names.split(",")) * {
            "int32_t": "i", "float": "f", "int64_t": "q", "sgemm_emu_view_t": "qqqq"}.get(
                kind, "q" if kind.endswith("*") else "?")
    assert struct.calcsize("=" + code) == struct.calcsize("@" + code)  # no padding
    flat = re.sub(r"(\d+)([a-z])", lambda m: m.group(2) * int(m.group(1)), packed.format[1:])
    assert flat == code


def call(name, packed, values, query):
    lib = pkg.load()
    if query:
        return getattr(lib, name + "_workspace")(packed.pack(*values))
    return getattr(lib, name)(packed.pack(*values), None)


def view(at, tokens, heads, size):
    return (at * MB, tokens * heads * size, heads * size, size)


def shape(**kw):
    s = dict(dtype=1, batch=2, tokens=100, keys=100, q_heads=4, k_heads=2, size=64, causal=1,
             scale=0.125, reserved=0)
    if "tokens" in kw:
        s["keys"] = kw["tokens"]
    s.update(kw)
    return s


def forward(query=False, cu=0, cu_k=0, ws=1 << 32, ws_bytes=1 << 40, views=None, **kw):
    s = shape(**kw)
    t, n, hq, hk, d = (s[x] for x in ("tokens", "keys", "q_heads", "k_heads", "size"))
    x = {"q": view(1, t, hq, d), "k": view(2, n, hk, d), "v": view(3, n, hk, d),
         "o": view(4, t, hq, d), "lse": view(5, t, hq, 1)}
    x.update(views or {})
    return call("attention_emu_forward", attention._FORWARD,
                (*s.values(), cu, cu_k, *(y for z in x.values() for y in z), ws, ws_bytes), query)


SIZES = [
    (dict(dtype=3), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED), (dict(batch=-1), DIM),
    (dict(tokens=-1), DIM), (dict(keys=-1), DIM), (dict(q_heads=-4), DIM), (dict(size=-1), DIM),
    (dict(q_heads=0), UNSUPPORTED), (dict(k_heads=0), UNSUPPORTED), (dict(k_heads=3), UNSUPPORTED),
    (dict(q_heads=2, k_heads=4), UNSUPPORTED), (dict(size=0), UNSUPPORTED),
    (dict(size=129), UNSUPPORTED), (dict(scale=0.0), UNSUPPORTED),
    (dict(scale=float("inf")), UNSUPPORTED), (dict(scale=float("nan")), UNSUPPORTED),
    (dict(cu=0, cu_k=30 * MB), NULL), (dict(cu=30 * MB, keys=101), DIM),
    (dict(tokens=BIG, keys=1), UNSUPPORTED), (dict(keys=BIG), UNSUPPORTED),
    (dict(tokens=1 << 29, keys=1), UNSUPPORTED),
    (dict(tokens=1 << 20, batch=1 << 15), UNSUPPORTED),
    (dict(keys=1 << 20, batch=1 << 15), UNSUPPORTED),
    (dict(batch=BIG, tokens=1), UNSUPPORTED)]


WIDE = [(dict(dtype=0, q_heads=16386, size=8), UNSUPPORTED),  # planes too far apart
        (dict(dtype=0, q_heads=16384, size=8, batch=0), OK),
        (dict(dtype=1, q_heads=16386, size=8, batch=0), OK)]


@pytest.mark.parametrize("kw,code", SIZES + WIDE + [
    (dict(batch=0), OK), (dict(tokens=0), OK), (dict(tokens=0, keys=7), OK),
    (dict(views={"q": (0, 1, 1, 1)}), NULL), (dict(views={"k": (0, 1, 1, 1)}), NULL),
    (dict(views={"v": (0, 1, 1, 1)}), NULL), (dict(views={"o": (0, 1, 1, 1)}), NULL),
    (dict(tokens=16, keys=8192, batch=1, ws=0), NULL),
    (dict(tokens=16, keys=8192, batch=1, ws_bytes=256), DIM),
    (dict(tokens=16, keys=8192, batch=1, ws=(1 << 32) + 16), DIM),
    (dict(tokens=16, keys=8192, batch=1, ws=MB), ALIAS),
    (dict(tokens=16, keys=8192, batch=1, ws=4 * MB), ALIAS),
    (dict(views={"k": (2 * MB, -1, 128, 64)}), STRIDE),
    (dict(views={"q": (MB, 1, -256, 64)}), STRIDE),
    (dict(views={"k": (2 * MB, 1, (1 << 22) + 1, 64)}), UNSUPPORTED),
    (dict(views={"k": (2 * MB, 1 << 62, 128, 64)}), ALIAS),  # 2^63 bytes, the outputs in them
    (dict(views={"k": (2 * MB, (1 << 63) - 1, 128, 64)}), STRIDE),  # past 2^64
    (dict(views={"o": (4 * MB, 25600, 256, 63)}), STRIDE),
    (dict(views={"o": (4 * MB, 0, 256, 64)}), STRIDE),
    (dict(views={"lse": (5 * MB, 400, 0, 1)}), STRIDE),
    (dict(views={"o": (MB, 25600, 256, 64)}), ALIAS),
    (dict(views={"o": (3 * MB + 128, 25600, 256, 64)}), ALIAS),
    (dict(views={"lse": (2 * MB, 400, 4, 1)}), ALIAS),
    (dict(views={"lse": (4 * MB, 400, 4, 1)}), ALIAS),
    (dict(cu=4 * MB), ALIAS), (dict(cu=30 * MB, cu_k=5 * MB), ALIAS)])
def test_forward_arguments(kw, code):
    assert forward(**kw) == code


def test_forward_workspace():
    for kw, code in SIZES:
        assert forward(query=True, **kw) == code
    # enough rows for the device, and few rows behind many keys
    assert forward(query=True, tokens=8192, q_heads=32, k_heads=32) == 0
    few = forward(query=True, tokens=16, keys=8192, batch=1)
    assert few > 0 and few % 256 == 0
    # FP32 operands are taken apart once
    assert forward(query=True, dtype=0, tokens=2000, q_heads=32, k_heads=32) >= 3 * 2 * 2000 * 32 * 256


def backward(query=False, cu=0, cu_k=0, ws=1 << 32, ws_bytes=1 << 40, views=None, **kw):
    s = shape(**kw)
    t, n, hq, hk, d = (s[x] for x in ("tokens", "keys", "q_heads", "k_heads", "size"))
    x = {"q": view(1, t, hq, d), "k": view(2, n, hk, d), "v": view(3, n, hk, d),
         "o": view(4, t, hq, d), "lse": view(5, t, hq, 1), "do": view(6, t, hq, d),
         "dq": view(7, t, hq, d), "dk": view(8, n, hk, d), "dv": view(9, n, hk, d)}
    x.update(views or {})
    return call("attention_emu_backward", attention._BACKWARD,
                (*s.values(), cu, cu_k, *(y for z in x.values() for y in z), ws, ws_bytes), query)


@pytest.mark.parametrize("kw,code", SIZES + WIDE + [(dict(batch=0), OK)] + [
    (dict(views={name: (0, 1, 1, 1)}), NULL)
    for name in ("q", "k", "v", "o", "lse", "do", "dq", "dk", "dv")] + [
    (dict(ws=0), NULL), (dict(ws_bytes=256), DIM), (dict(ws=(1 << 32) + 128), DIM),
    (dict(views={"do": (6 * MB, 1, 1 << 23, 64)}), UNSUPPORTED),
    (dict(views={"dk": (8 * MB, 12800, 128, 63)}), STRIDE),
    (dict(views={"lse": (5 * MB, 400, -4, 1)}), STRIDE),
    (dict(views={"dq": (6 * MB, 25600, 256, 64)}), ALIAS),
    (dict(views={"dv": (8 * MB, 12800, 128, 64)}), ALIAS),
    (dict(ws=6 * MB), ALIAS), (dict(ws=9 * MB), ALIAS), (dict(cu=7 * MB), ALIAS)])
def test_backward_arguments(kw, code):
    assert backward(**kw) == code


def test_gradients_may_be_slices_of_one_projection():
    """(Taken as far as the workspace, which is missing.)"""
    row = 8 * 64
    at = 7 * MB
    views = {n: (at + 2 * x, 100 * row, row, 64) for n, x in (("dq", 0), ("dk", 256), ("dv", 384))}
    assert backward(views=views, ws=0) == NULL
    assert backward(views={**views, "dv": (at + 2 * 383, 100 * row, row, 64)}) == ALIAS


def test_backward_workspace():
    for kw, code in SIZES:
        assert backward(query=True, **kw) == code
    assert backward(query=True) >= 2 * 100 * 4 * 4  # a number for each row


def step(query=False, ws=1 << 32, ws_bytes=1 << 40, views=None, lengths=20 * MB, slots=0, **kw):
    s = dict(dtype=1, batch=4, tokens=1, prefix=2000, capacity=128, n_slots=6, q_heads=4, k_heads=2,
             size=64, scale=0.125)
    s.update(kw)
    hq, hk, d = s["q_heads"], s["k_heads"], s["size"]
    x = {"q": view(1, s["tokens"], hq, d), "prefix_k": view(2, s["prefix"], hk, d),
         "prefix_v": view(3, s["prefix"], hk, d), "k": view(4, s["capacity"], hk, d),
         "v": view(5, s["capacity"], hk, d), "o": view(6, s["tokens"], hq, d)}
    x.update(views or {})
    return call("attention_emu_step", attention._STEP,
                (*s.values(), *(y for z in x.values() for y in z), lengths, slots, ws, ws_bytes),
                query)


STEP_SIZES = [x for x in SIZES if not x[0].keys() & {"keys", "cu", "batch"}
              and x[0].get("tokens", 0) < 1 << 20] + [
    (dict(batch=-1), DIM), (dict(prefix=-1), DIM), (dict(capacity=-1), DIM), (dict(n_slots=-1), DIM),
    (dict(batch=7), DIM), (dict(tokens=1 << 28), UNSUPPORTED), (dict(prefix=BIG), UNSUPPORTED),
    (dict(capacity=BIG), UNSUPPORTED), (dict(batch=1 << 28, slots=30 * MB), UNSUPPORTED)]


@pytest.mark.parametrize("kw,code", STEP_SIZES + [
    (dict(batch=0), OK), (dict(tokens=0), OK), (dict(lengths=0), NULL), (dict(ws=0), NULL),
    (dict(ws_bytes=256), DIM), (dict(ws=(1 << 32) + 8), DIM)] + [
    (dict(views={name: (0, 1, 1, 1)}), NULL)
    for name in ("q", "prefix_k", "prefix_v", "k", "v", "o")] + [
    (dict(views={"prefix_k": (2 * MB, 0, 1 << 23, 64)}), UNSUPPORTED),
    (dict(views={"v": (5 * MB, 0, -128, 64)}), STRIDE),
    (dict(views={"o": (6 * MB, 0, 256, 64)}), STRIDE),
    (dict(views={"o": (MB, 256, 256, 64)}), ALIAS), (dict(views={"o": (5 * MB, 256, 256, 64)}), ALIAS),
    (dict(lengths=6 * MB), ALIAS), (dict(slots=6 * MB), ALIAS), (dict(ws=20 * MB), ALIAS),
    (dict(ws=2 * MB), ALIAS)])
def test_step_arguments(kw, code):
    assert step(**kw) == code


def test_step_workspace():
    for kw, code in STEP_SIZES:
        assert step(query=True, **kw) == code
    assert step(query=True) > 0
    assert step(query=True, prefix=0) == 0  # one short part


@pytest.mark.parametrize("name", pkg.ATTENTION_SYMBOLS)
def test_null_struct(name):
    fn = getattr(pkg.load(), name)
    assert fn(*[None] * len(fn.argtypes)) == NULL


# ---- the binding's own checks -----------------------------------------------

BF16 = torch.bfloat16


def inputs():
    q = torch.zeros(2, 20, 4, 16, dtype=BF16)
    k = torch.zeros(2, 20, 2, 16, dtype=BF16)
    return {"q": q, "k": k, "v": k.clone()}


def gradient(**change):
    x = inputs()
    x.update(o=x["q"].clone(), lse=torch.zeros(2, 20, 4), do=x["q"].clone())
    x.update(change)
    return pkg.attention_emu_backward(**x)


def one_step(**change):
    x = inputs()
    x.update(lengths=torch.zeros(2, dtype=torch.int32))
    x.update(change)
    return pkg.attention_emu_step(**x)


def test_tensors_must_be_on_a_device():
    for call_ in (lambda: pkg.attention_emu_forward(**inputs()), gradient, one_step):
        with pytest.raises(ValueError):
            call_()


def zeros(*shape, dtype=BF16):
    return torch.zeros(*shape, dtype=dtype)


@pytest.mark.parametrize("call_", [
    lambda **c: pkg.attention_emu_forward(**{**inputs(), **c}), gradient, one_step])
@pytest.mark.parametrize("change", [
    dict(q=zeros(20, 4, 16)), dict(k=zeros(20, 2, 16)), dict(v=zeros(20, 2, 16)),
    dict(k=zeros(2, 20, 2, 17)), dict(v=zeros(2, 20, 1, 16)), dict(v=zeros(2, 19, 2, 16)),
    dict(q=zeros(2, 20, 16, 4).transpose(2, 3)), dict(k=zeros(2, 20, 2, 32)[..., ::2]),
    dict(k=zeros(2, 20, 2, 16, dtype=torch.float16)), dict(v=zeros(2, 20, 2, 16, dtype=torch.float32)),
    dict(q=zeros(2, 20, 4, 16, dtype=torch.float64))])
def test_inputs_are_checked(call_, change):
    with pytest.raises((TypeError, ValueError)):
        call_(**change)


@pytest.mark.parametrize("change", [
    dict(lse=zeros(2, 20, 4)), dict(lse=zeros(2, 4, 20, dtype=torch.float32)),
    dict(o=zeros(2, 20, 4, 15)), dict(do=zeros(2, 20, 4, 16, dtype=torch.float16)),
    dict(out=[zeros(2, 20, 4, 16), zeros(2, 20, 4, 16), zeros(2, 20, 2, 16)])])
def test_gradient_arguments(change):
    with pytest.raises((TypeError, ValueError)):
        gradient(**change)


@pytest.mark.parametrize("change", [
    dict(out=zeros(2, 20, 2, 16)), dict(out=zeros(2, 20, 4, 16, dtype=torch.float32)),
    dict(lse=zeros(2, 20, 4)), dict(cu_seqlens=zeros(3, dtype=torch.int32)),
    dict(cu_seqlens_k=zeros(3, dtype=torch.int32))])
def test_forward_results_and_bounds(change):
    with pytest.raises((TypeError, ValueError)):
        pkg.attention_emu_forward(**inputs(), **change)


def test_packed_bounds():
    x = {m: y[:1] for m, y in inputs().items()}
    three = zeros(3, dtype=torch.int32)
    for bad in (dict(cu_seqlens=three.long()), dict(cu_seqlens=three, cu_seqlens_k=three[:2]),
                dict(cu_seqlens=zeros(3, 1, dtype=torch.int32)), dict(cu_seqlens=three[:0]),
                dict(cu_seqlens=zeros(6, dtype=torch.int32)[::2])):
        with pytest.raises((TypeError, ValueError)):
            pkg.attention_emu_forward(**x, **bad)


@pytest.mark.parametrize("change", [
    dict(lengths=None), dict(lengths=zeros(3, dtype=torch.int32)),
    dict(lengths=zeros(2, dtype=torch.int64)), dict(lengths=zeros(4, dtype=torch.int32)[::2]),
    dict(slots=zeros(1, dtype=torch.int32)), dict(slots=zeros(2)),
    dict(prefix_k=zeros(1, 5, 2, 16)), dict(prefix_v=zeros(1, 5, 2, 16)),
    dict(prefix_k=zeros(2, 5, 2, 16), prefix_v=zeros(2, 5, 2, 16)),
    dict(prefix_k=zeros(5, 2, 16), prefix_v=zeros(5, 2, 16)),
    dict(prefix_k=zeros(1, 5, 2, 16), prefix_v=zeros(1, 6, 2, 16)),
    dict(prefix_k=zeros(1, 5, 2, 16), prefix_v=zeros(1, 5, 2, 16, dtype=torch.float16)),
    dict(out=zeros(2, 20, 4, 15))])
def test_step_tensors(change):
    with pytest.raises((TypeError, ValueError)):
        one_step(**change)


def test_workspace_queries_through_the_binding():
    x = inputs()
    assert pkg.attention_emu_forward_workspace(**x) == 0
    assert pkg.attention_emu_backward_workspace(**x) >= 2 * 20 * 4 * 4
    assert pkg.attention_emu_step_workspace(**x) == 0
    one = zeros(1, 4000, 2, 16)
    assert pkg.attention_emu_step_workspace(**x, prefix_k=one, prefix_v=one) > 0
    big = zeros(1, 1, 1, 200)
    for name in pkg.ATTENTION_SYMBOLS:
        if name.endswith("_workspace"):
            with pytest.raises(pkg.SgemmEmuError):
                getattr(pkg, name)(big, big, big)


def test_first_use_is_whole(monkeypatch):
    """Another thread sees the looked up functions all or not at all."""
    lib = pkg.load()
    seen = []

    class Library:
        def __getattr__(self, name):
            seen.append((len(attention._calls), len(attention._dtypes)))
            return getattr(lib, name)

    monkeypatch.setattr(attention, "_calls", {})
    monkeypatch.setattr(pkg, "load", Library)
    attention._start()
    assert len(seen) == len(attention._calls) == len(pkg.ATTENTION_SYMBOLS)
    assert all(calls == 0 and types == 3 for calls, types in seen)
