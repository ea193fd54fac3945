"""Every single value of windowed attention, its gradients and the attention over pages within the bound of its own (tests/window_bounds.py), at
the shapes of both sides of the rules and at random ones."""
import random

import pytest

from tests import window_bounds
from tests.test_gpu_paged import CASES as FEW_PAGED
from tests.test_gpu_paged import _paged_case
from tests.test_gpu_window import CASES as FEW_TRAIN
from tests.test_gpu_window import _inputs, _step
from tests.window_shapes import PAGED, TRAIN

pytestmark = pytest.mark.gpu


def _train(case, seed):
    import torch
    dtype, b, h, kvh, n, d, window, sinks, lens = case
    inputs = _inputs(dtype, b, h, kvh, n, d, seed=seed)
    dev = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    got = _step(*inputs, d ** -0.5, window, sinks, dev)
    print("share of the bound %.2f" % window_bounds.check_step(inputs, got, d ** -0.5, window, sinks, lens, dtype), flush=True)


def _pages(case, seed):
    dtype, kind, lens, new, h, kvh, d, page, window, sinks = case
    c, Q, O, _ = _paged_case(*case, seed=seed)
    starts = [sum(new[:b]) for b in range(len(new) + 1)]
    print("share of the bound %.2f" % window_bounds.check_pages(Q, O, c.keys, c.values, starts, lens, d ** -0.5, window, sinks, dtype), flush=True)


@pytest.mark.parametrize("case", FEW_TRAIN + [case for case, _ in TRAIN])
def test_training_steps(case):
    print("case train", *case, flush=True)
    _train(case, 51)


@pytest.mark.parametrize("case", FEW_PAGED + [case for case, _ in PAGED])
def test_attention_over_pages(case):
    print("case pages", *case, flush=True)
    _pages(case, 52)


@pytest.mark.parametrize("seed", range(24))
def test_training_steps_of_random_sizes(seed):
    rng = random.Random(seed)
    for _ in range(4):
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        kvh = rng.choice([1, 1, 2, 3, 5])
        h, b, n = kvh * rng.choice([1, 1, 2, 3, 4, 7, 8]), rng.choice([1, 1, 2, 3]), rng.randint(1, rng.choice([70, 300, 1300]))
        d = 8 * rng.randint(1, 32) if dtype == "bf16" and rng.random() < 0.5 else rng.choice([64, 128, 256]) if dtype == "bf16" else rng.randint(1, 256)
        window = rng.choice([0, rng.randint(1, n), rng.randint(1, 64)])
        sinks = rng.choice([0, 0, 1, 4, rng.randint(0, 150)])
        lens = rng.choice([None, [rng.randint(0, n) for _ in range(b)]])
        case = (dtype, b, h, kvh, n, d, window, sinks, lens)
        print("case train", seed, *case, flush=True)
        _train(case, seed)


@pytest.mark.parametrize("seed", range(24))
def test_attention_over_pages_of_random_sizes(seed):
    rng = random.Random(1000 + seed)
    for _ in range(4):
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        kind, kvh = rng.choice(["plain", "fp8"]), rng.choice([1, 2, 3, 5])
        h, b = kvh * rng.choice([1, 2, 3, 4, 8, 17]), rng.choice([1, 2, 3, 7])
        lens = [rng.randint(0, rng.choice([40, 600, 3000])) for _ in range(b)]
        most = rng.choice([1, 1, 3, 20, 200])
        new = [min(x, rng.randint(0, most)) if rng.random() < 0.9 else rng.randint(0, most) for x in lens]
        d = rng.choice([64, 128, 256, 8 * rng.randint(1, 32)]) if dtype == "bf16" or kind == "fp8" else rng.randint(1, 256)
        page, window = 8 << rng.randint(0, 5), rng.choice([0, rng.randint(1, 64), rng.randint(1, 2000)])
        case = (dtype, kind, lens, new, h, kvh, d, page, window, rng.choice([0, 1, 4, 70, 200]))
        if sum(new) == 0:
            continue
        print("case pages", seed, *case, flush=True)
        _pages(case, seed)
