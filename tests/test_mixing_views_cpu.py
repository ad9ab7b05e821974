"""Outputs of one call that share elements: refused by the entries, and the check behind it
against sets of bytes."""
import importlib.util
import os
import random
import subprocess

import pytest

from test_mixing_cpu import ALIAS, MB, backward, rotary

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# (The entries' own arguments here always end in a refusal: nothing is launched.)
Q, K = (768, 256, 64), (384, 128, 64)  # strides of rotary's tensors of 4 and 2 heads


@pytest.mark.parametrize("kw", [
    dict(yk=(3 * MB, *K)),  # both outputs in one place
    dict(yq=(3 * MB, *Q), yk=(3 * MB + 64, *K)),
    dict(heads=(4, 4), q=(MB, *Q), k=(MB, *Q), yq=(MB, *Q), yk=(MB, *Q)),  # both in place
    dict(heads=(4, 4), q=(MB, *Q), k=(MB + 128, *Q), yq=(MB, *Q), yk=(MB + 128, *Q))])
def test_rotary(kw):
    assert rotary(**kw) == ALIAS


@pytest.mark.parametrize("views", [
    {"dk": (11 * MB, 12800, 128, 64)},           # dq's place
    {"dbeta": (14 * MB, 400, 4, 1)},             # dg's place
    {"dv": (12 * MB + 2, 12800, 128, 32)},       # across dk
    {"dbeta": (13 * MB + 400, 400, 4, 1)},       # inside dv, in another type
])
def test_backward(views):
    assert backward(views=views) == ALIAS


# ---- the check itself -------------------------------------------------------

MAIN = """
#include <cstdio>
#include "views.h"
int main() {
    long long x[18];
    while (true) {
        for (long long& v : x)
            if (std::scanf("%lld", &v) != 1) return 0;
        using namespace sgemm_emu;
        const Tensor a{{(void*)x[0], x[1], x[2], x[3]}, x[4], x[5], x[6], x[7], x[8]};
        const Tensor b{{(void*)x[9], x[10], x[11], x[12]}, x[13], x[14], x[15], x[16], x[17]};
        std::printf("%d%d%d\\n", apart(a), apart(b), meet(a, b));
    }
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    spec = importlib.util.spec_from_file_location(
        "product_build", os.path.join(ROOT, "paper_2308_15152_amd", "build.py"))
    build = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(build)
    at = tmp_path_factory.mktemp("views")
    (at / "main.hip").write_text(MAIN)
    subprocess.run([build.HIPCC, *build.DEVICE_FLAGS, str(at / "main.hip"), "-o", str(at / "main")],
                   check=True, capture_output=True)
    return str(at / "main")


def elements(x):
    at, sb, st, sh, b, t, h, size, elem = x
    return {at + (i * sb + j * st + k * sh) * elem + e
            for i in range(b) for j in range(t) for k in range(h) for e in range(size * elem)}


def ask(program, pairs):
    text = "\n".join(" ".join(map(str, (*a, *b))) for a, b in pairs)
    out = subprocess.run([program], input=text, capture_output=True, text=True, check=True).stdout
    return [tuple(c == "1" for c in line) for line in out.split()]


def test_slices_of_one_buffer_are_told_apart(program):
    """Same strides, two places in a row (or in heads or batches): exactly the elements
    that are shared."""
    r = random.Random(3)
    pairs = []
    for _ in range(3000):
        n = [r.randint(1, 3) for _ in range(3)]
        row = 24
        order = r.sample(range(3), 3)
        strides, step = [0] * 3, row
        for i in order:
            strides[i], step = step, step * max(n[i], r.randint(1, 3))
        def piece():
            return (4096 + r.choice([0, r.randint(0, row), r.randint(0, 2 * step)]) * 2, *strides,
                    *(r.randint(1, k) for k in n), r.randint(1, 12), 2)
        pairs.append((piece(), piece()))
    got = ask(program, pairs)
    seen = {True: 0, False: 0}
    for (a, b), (apart_a, apart_b, met) in zip(pairs, got):
        assert apart_a and apart_b
        shared = bool(elements(a) & elements(b))
        # a dimension of one entry has no stride, which may leave blocks that are not told apart
        if all(i == j for i, j in zip(a[4:7], b[4:7])):
            assert met == shared, (a, b)
            seen[shared] += 1
        assert met or not shared, (a, b)
    assert min(seen.values()) > 100


def test_what_is_shared_is_always_seen(program):
    r = random.Random(4)
    pairs = []
    for _ in range(20000):
        def piece():
            return (4096 + r.randint(0, 60), *(r.randint(0, 40) for _ in range(3)),
                    *(r.randint(0, 3) for _ in range(3)), r.randint(0, 5), r.choice([1, 2, 4]))
        pairs.append((piece(), piece()))
    seen = 0
    for (a, b), (apart_a, apart_b, met) in zip(pairs, ask(program, pairs)):
        if apart_a and apart_b:
            seen += 1
            assert met or not elements(a) & elements(b), (a, b)
    assert seen > 1000
