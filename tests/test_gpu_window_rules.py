"""Windowed attention and the paged cache on the far side of the rules that choose their kernels by the size of the call (tests/window_shapes.py;
which side each shape is on is held by tests/test_window_rules.py), against 64 bits with the tolerances of the small cases."""
import pytest

from tests import window_ref
from tests.test_gpu_paged import Cache, _paged_case
from tests.test_gpu_window import _check, _inputs, _step
from tests.window_shapes import CACHE, CACHE_LINE, PAGED, TRAIN

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", [case for case, _ in TRAIN])
def test_training_steps(case):
    import torch
    print("case train", *case, flush=True)
    dtype, b, h, kvh, n, d, window, sinks, lens = case
    inputs = _inputs(dtype, b, h, kvh, n, d, seed=31)
    dev = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    _check("train", inputs, d ** -0.5, window, sinks, lens, _step(*inputs, d ** -0.5, window, sinks, dev), dtype)


@pytest.mark.parametrize("case", [case for case, _ in PAGED])
def test_attention_over_pages(case):
    print("case pages", *case, flush=True)
    dtype, kind, lens, new, h, kvh, d, page, window, sinks = case
    _paged_case(dtype, kind, lens, new, h, kvh, d, page, window, sinks, seed=32)


def _write_and_read(dtype, kind, new, kvh, d, page):
    """Rows that are written come back as they are (quantised and back, to the bit), and nothing else in the cache changes."""
    import torch
    from paper_2410_09397_amd import attn
    lens = [q + (7 * i) % 40 for i, q in enumerate(new)]
    c = Cache(dtype, kind, lens, kvh, d, page, seed=33)
    starts = [sum(new[:b]) for b in range(len(new) + 1)]
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    gen = torch.Generator()
    gen.manual_seed(34)
    x = [torch.randn(starts[-1], kvh, d, generator=gen).mul(2.0).to(dt) for _ in range(2)]
    codes = [window_ref.quantise(y) if kind == "fp8" else (y, None) for y in x]
    raw = lambda t: t.view(torch.uint8) if t.dtype is torch.float8_e4m3fn else t
    want = [raw(t).clone() for t in (c.K, c.V)]
    want_exp = [None if e is None else e.clone() for e in (c.K_exp, c.V_exp)]
    pos = torch.cat([torch.arange(l - q, l) for l, q in zip(lens, new)]).cuda()
    seq = torch.repeat_interleave(torch.arange(len(new)), torch.tensor(new)).cuda()
    at, slot = c.table[seq, pos // page].long(), pos % page
    for which in range(2):
        want[which][at, :, slot] = raw(codes[which][0]).cuda()
        if kind == "fp8":
            want_exp[which][at, :, slot] = codes[which][1].cuda()
    kw = dict(q_ptr=torch.tensor(starts, dtype=torch.int32, device="cuda"), max_q=max(new), **c.exps())
    attn.attn_cache_write(x[0].cuda(), x[1].cuda(), *c.args(), **kw)
    bits = lambda t: t if t.dtype is torch.uint8 else t.view(torch.int16 if t.dtype is torch.bfloat16 else torch.int32)
    for which in range(2):
        assert torch.equal(bits(raw((c.K, c.V)[which])), bits(want[which]))
        if kind == "fp8":
            assert torch.equal((c.K_exp, c.V_exp)[which], want_exp[which])
    for got, y in zip(attn.attn_cache_read(*c.args(), dt, starts[-1], **kw), codes):
        assert torch.equal(got, window_ref.values(*y).to(dt).cuda())


@pytest.mark.parametrize("case", CACHE)
def test_writing_and_reading_back_large_calls(case):
    print("case cache", *case, flush=True)
    _write_and_read(*case)


@pytest.mark.parametrize("total,kvh,d,rows", CACHE_LINE)
@pytest.mark.parametrize("kind", ["plain", "fp8"])
def test_writing_and_reading_back_around_the_line(kind, total, kvh, d, rows):
    print("case cache line", kind, total, kvh, d, flush=True)
    _write_and_read("bf16", kind, [total - 3, 3], kvh, d, 16)
