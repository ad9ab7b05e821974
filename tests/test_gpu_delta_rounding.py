"""16-bit outputs of the gated delta rule are FP32 results rounded once.

Tolerance.  With x the result in 64 bits and c = 2^-22 (4 + sqrt(chunks)) the bound of
what is computed in FP32 (test_gpu_delta_forward.py), an output is the rounding of x + e,
|e| <= c |x| in the 2-norm.  It differs from the rounding of x where an edge between two
roundings lies between the two, which is so for a share |e| / ulp of the elements, and
then by one ulp <= 2 u |x| (u = 2^-8 for bfloat16, 2^-11 for float16): the squares of
the differences add up to 2 u c |x|^2 on average.  Twice the root of that is allowed.  An
operand rounded to 11 bits on the way (2^-12 on average) is off by about 2^-10."""
import math

import pytest
import torch

import paper_2308_15152_amd as emu
from delta_plain import delta
from test_gpu_delta_forward import UNIT
from test_gpu_delta_step import dev, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("t,ks,vs,copies", [
    (10, 64, 96, 1), (200, 64, 96, 1), (200, 128, 96, 1), (333, 96, 36, 1),
    (200, 64, 96, 70), (200, 128, 96, 70)])
def test_outputs_are_rounded_once(dtype, t, ks, vs, copies):
    """copies: of the sequence in the batch; many fill the device, which takes other
    kernels than few."""
    x = inputs(1, t, 2, 2, ks, vs, dtype, seed=t, decay=0.2)
    first = torch.randn(1, 2, ks, vs, generator=torch.Generator().manual_seed(5))
    want, _ = delta(*x, first)
    y = [z.expand(copies, *z.shape[1:]) for z in dev(*x)]
    o, _ = emu.delta_emu_forward(*y, first.to("cuda:0").repeat(copies, 1, 1, 1))
    assert torch.equal(o, o[:1].expand_as(o))
    off = float((o[:1].cpu().double() - want.to(dtype).double()).norm() / want.norm())
    c = 2.0 ** -22 * (4 + math.sqrt(t / 64))
    assert off <= 2 * math.sqrt(2 * UNIT[dtype] * c), off
