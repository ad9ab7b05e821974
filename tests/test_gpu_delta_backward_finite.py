"""Gradients that are not finite: what comes in at a token reaches the tokens that the reversed
recurrence takes it to, in 64 bits as well, and no later ones.  What stays finite keeps the
bounds of test_gpu_delta_backward.py."""
import pytest
import torch

from delta_plain import delta_gradients
from test_gpu_delta_backward import NAMES, check, gradients
from test_gpu_delta_step import inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def seeded():
    torch.manual_seed(11)


def compare(got, x, do, first, dfinal, clean, tokens, dtype):
    """Finite where the recurrence's gradient is, and there what it is without the value that
    is not (which has no part in it).  clean: those gradients, and their do."""
    want = delta_gradients(*x, do, first, dfinal)
    good = []
    for name, a, b, c in zip(NAMES, got, want, clean[0]):
        keep = b.isfinite()
        assert torch.equal(a.cpu().isfinite(), keep), name
        assert float((b - c)[keep].norm()) <= 1e-12 * float(c.norm())
        # the others as they should be, so that the norms are those of whole tensors
        good.append(torch.where(keep, a.cpu().double(), c))
    check(good, clean[0], x, clean[1], tokens, dtype)


def copied(y, n):
    return None if y is None else y.repeat(n, *[1] * (y.dim() - 1))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("copies", [1, 18])
@pytest.mark.parametrize("t,at", [(10, 4), (150, 0), (150, 21), (150, 63), (150, 64), (150, 149)])
def test_of_an_output(dtype, copies, t, at):
    """copies: of the sequence in the batch, of which the last has the value; many take kernels
    of their own."""
    x = inputs(1, t, 1, 2, 64, 112, dtype, seed=at, decay=0.2)
    do = torch.randn(1, t, 2, 112).to(dtype)
    first, dfinal = torch.randn(1, 2, 64, 112), torch.randn(1, 2, 64, 112)
    clean = delta_gradients(*x, do, first, dfinal), do
    many = [copied(y, copies) for y in (*x, do, first, dfinal)]
    for value in (torch.nan, torch.inf):
        many[5][-1, at, -1, 7] = value
        got = gradients(many[:5], *many[5:])
        compare([y[-1:] for y in got], x, many[5][-1:], first, dfinal, clean, t, dtype)
        if copies > 1:
            assert all(torch.equal(y[:-1], y[:1].expand_as(y[:-1])) for y in got)
            check([y[:1] for y in got], clean[0], x, do, t, dtype)


@pytest.mark.parametrize("t", [10, 150])
def test_of_a_final_state(t):
    x = inputs(2, t, 1, 2, 64, 48, torch.float32, seed=t, decay=0.2)
    do, dfinal = torch.randn(2, t, 2, 48), torch.randn(2, 2, 64, 48)
    clean = delta_gradients(*x, do, None, dfinal), do
    bad = dfinal.clone()
    bad[1, 0, 5, 7] = torch.nan
    compare(gradients(x, do, None, bad), x, do, None, bad, clean, t, torch.float32)


@pytest.mark.parametrize("at", [100, 2500, 4400])
def test_in_parts(at):
    x = inputs(1, 4500, 1, 1, 64, 32, torch.float32, seed=1, decay=0.05)
    do = torch.randn(1, 4500, 1, 32)
    clean = delta_gradients(*x, do, None, None), do
    bad = do.clone()
    bad[0, at, 0, 3] = torch.nan
    compare(gradients(x, bad, None, None), x, bad, None, None, clean, 4 * 4500, torch.float32)
