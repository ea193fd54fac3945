"""How exact windowed attention is, by the norm of the error over the norm of the result, beside the calls without a window.

Rounding to bf16 moves a value x by up to 2^-8 of its binade's lower end, evenly on both sides: 2^-7 / sqrt(12) = 2.26e-3 of x at the lower end, half of that at
the upper one.  A tensor that is rounded once (O or a gradient, when it is stored) is therefore off by at most 2.26e-3 of its norm.  Rounding the
weights P or dS as well adds as much again, independently: the terms of a sum over keys with values of both signs add up in squares
as the sum itself does.  At most sqrt(2) 2.26e-3 = 3.19e-3 together.  The windowed kernels round both at every head dimension; attn_fwd and
attn_bwd do at 64, 128 and 256 and keep the weights in 32 bits at the others."""
import pytest

from tests import window_ref
from tests.test_gpu_window import _inputs, _step

pytestmark = pytest.mark.gpu
ONCE = 2.0 ** -7 / 12 ** 0.5
TWICE = ONCE * 2 ** 0.5


def _errors(inputs, got, window=0, sinks=0):
    """Of O, dQ, dK and dV; the gradients' reference takes O and LSE as the backward got them."""
    Q, K, V, dO = inputs
    want = window_ref.window_attention(Q, K, V, dO, Q.shape[3] ** -0.5, window, sinks, given=got[:2])
    return [float((x.double() - y).norm() / y.norm()) for i, (x, y) in enumerate(zip(got, want)) if i != 1]


@pytest.mark.parametrize("d", [24, 72, 96, 136, 248])
def test_causal_attention_at_head_dimensions_between_the_widths(d):
    from paper_2410_09397_amd import attn
    print("case precision", d, flush=True)
    inputs = _inputs("bf16", 1, 4, 4, 700, d, seed=41)
    Q, K, V, dO = inputs
    O, LSE = attn.attn_fwd(Q, K, V, d ** -0.5, causal=True)
    full = _errors(inputs, (O, LSE) + tuple(attn.attn_bwd(Q, K, V, O, dO, LSE, d ** -0.5, causal=True)))
    here = _errors(inputs, _step(Q, K, V, dO, d ** -0.5, 0, 0))
    print("without a window %s, windowed entry points %s" % (" ".join("%.2e" % e for e in full), " ".join("%.2e" % e for e in here)), flush=True)
    assert max(full) <= ONCE and max(here) <= TWICE


@pytest.mark.parametrize("d", [40, 64, 104, 128, 192, 256])
@pytest.mark.parametrize("heads,kv_heads", [(6, 2), (3, 3)])
def test_windows_and_shared_heads(d, heads, kv_heads):
    print("case precision window", d, heads, kv_heads, flush=True)
    inputs = _inputs("bf16", 2, heads, kv_heads, 500, d, seed=42)
    here = _errors(inputs, _step(*inputs, d ** -0.5, 130, 3), 130, 3)
    print(" ".join("%.2e" % e for e in here), flush=True)
    assert max(here) <= TWICE
