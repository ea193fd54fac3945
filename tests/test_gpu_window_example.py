"""The example that trains with a window and serves from a paged cache."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("quantised", [False, True])
def test_example_learns_and_serves(quantised):
    """bf16 pages: the served outputs are those of one forward up to bf16 (2 %).  Quantised: keys and values are off by up to 2^-4 of each
    value, a score (a sum of 64 products of both signs) by a few per cent of its size, so outputs by some per cent: the gate is 15 %."""
    from paper_2410_09397_amd import example_window_cache
    losses, far, cache = example_window_cache.main(steps=40, n=128, quantised=quantised)
    assert losses[-1] < 0.9 * losses[0]
    assert max(far) <= (0.15 if quantised else 0.02)
    assert cache <= (2.0 ** -4 if quantised else 0.0)
