"""The bounds of tests/window_bounds.py on the CPU: results that are rounded as the kernels round them are inside, mistakes in rows of small values are not."""
import pytest
import torch

from tests import window_bounds
from tests.window_ref import attend, window_attention


def _rounded(seed, b, h, kvh, n, d, c, window, sinks):
    """Inputs, and results with P, dS and the results rounded to bf16."""
    gen = torch.Generator()
    gen.manual_seed(seed)
    inputs = [torch.randn(b, x, n, d, generator=gen).bfloat16() for x in (h, kvh, kvh, h)]
    r = lambda t: t.bfloat16().double()
    Q, K, V, dO = (t.double() for t in inputs)
    O, dQ, dK, dV = (torch.zeros_like(t) for t in (Q, Q, K, K))
    LSE = torch.zeros(b, h, n, dtype=torch.float64)
    for x in range(b):
        for y in range(h):
            z = y // (h // kvh)
            _, LSE[x, y], f = attend(Q[x, y], K[x, z], V[x, z], 0, c, window, sinks)
            O[x, y] = r(r(f) @ V[x, z])
            ds = r(f * (dO[x, y] @ V[x, z].t() - (dO[x, y] * O[x, y]).sum(1, keepdim=True)))
            dQ[x, y] = c * (ds @ K[x, z])
            dK[x, z] += c * (ds.t() @ Q[x, y])
            dV[x, z] += r(f).t() @ dO[x, y]
    return inputs, [O.bfloat16(), LSE.float(), dQ.bfloat16(), dK.bfloat16(), dV.bfloat16()]


@pytest.mark.parametrize("window,sinks", [(0, 0), (30, 2)])
def test_rounded_results_are_inside(window, sinks):
    inputs, got = _rounded(1, 2, 4, 2, 150, 40, 0.2, window, sinks)
    assert window_bounds.check_step(inputs, got, 0.2, window, sinks, None, "bf16") <= 1.0


@pytest.mark.parametrize("which,at", [(0, (0, 3, 395)), (2, (0, 1, 390)), (3, (0, 0, 399)), (4, (0, 1, 380))])
def test_a_row_that_is_off_by_a_fifth_is_not(which, at):
    inputs, got = _rounded(2, 1, 4, 2, 400, 64, 0.125, 0, 0)
    row = got[which][at]
    got[which][at] = row * 1.2
    with pytest.raises(AssertionError, match="beyond their bounds"):
        window_bounds.check_step(inputs, got, 0.125, 0, 0, None, "bf16")


def test_a_key_that_should_be_hidden_is_seen():
    """The definition with a window of one key more."""
    inputs, _ = _rounded(3, 1, 2, 1, 300, 32, 0.2, 100, 0)
    O, LSE, *_ = window_attention(*inputs, 0.2, 101, 0)
    got = [O.bfloat16(), LSE.float(), *(t.bfloat16() for t in window_attention(*inputs, 0.2, 101, 0, given=(O.bfloat16(), LSE.float()))[2:])]
    with pytest.raises(AssertionError, match="beyond their bounds"):
        window_bounds.check_step(inputs, got, 0.2, 100, 0, None, "bf16")
