"""Windowed attention with shared heads (attn_win_fwd, attn_win_bwd) against its definition in 64 bits.

The gradients' reference takes O and LSE as the backward gets them.  Tolerance: that of the parity tests, max |x - ref| / max |ref| per tensor.  bf16: P, dS, O and the outputs are rounded to 8
bits (2^-9 of the value each); four such roundings that all err one way are 0.8 % of the largest value, and the gate is 2 %.
fp32: sums of up to a few thousand products, each off by 2^-24 of the largest partial sum; the gate is 1e-4.  Where dP - delta is a difference of
equal numbers (a query that sees one key), dQ and dK are what rounding leaves of two sums of d products: up to
2 d 2^-24 max |dO| max |O| max |K or Q| |scale|, and `group` times that for a key."""
import math

import pytest

from tests import window_ref
from tests.helpers import LSE_TOL, TOL

pytestmark = pytest.mark.gpu


def _inputs(dtype, b, h, kvh, n, d, seed=0, layout="bhnd"):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]

    def draw(heads):
        x = torch.randn(b, heads, n, d, generator=gen, device="cuda").to(dt)
        if layout == "bnhd":
            return x.transpose(1, 2).contiguous().transpose(1, 2)
        if layout == "padded":  # rows with a gap behind them, as a view of a wider tensor has
            wide = torch.full((b, heads, n + 3, d + 16), math.nan, device="cuda", dtype=dt)
            wide[:, :, :n, :d] = x
            return wide[:, :, :n, :d]
        return x
    return draw(h), draw(kvh), draw(kvh), draw(h)


def _check(name, inputs, scale, window, sinks, lens, got, dtype):
    import torch
    Q, K, V, dO = inputs
    want = window_ref.window_attention(Q, K, V, dO, scale, window, sinks, lens, given=got[:2])
    O, LSE, dQ, dK, dV = want
    top = lambda t: float(t.double().abs().max())
    left = 2 * Q.shape[3] * 2.0 ** -24 * top(dO) * top(O) * abs(scale)
    floors = (0.0, left * top(K), left * top(Q) * Q.shape[1] / K.shape[1], 0.0)
    for what, x, ref, floor in zip(("O", "dQ", "dK", "dV"), (got[0],) + tuple(got[2:]), (O, dQ, dK, dV), floors):
        err = top(x.double() - ref)
        print("%s %s %.3e of %.3e" % (name, what, err, top(ref)), flush=True)
        assert err <= TOL[dtype] * top(ref) + floor, (name, what, err, top(ref), floor)
    none = LSE == -math.inf
    assert torch.equal(got[1] == -math.inf, none), name
    if bool((~none).any()):
        err = float((got[1].double() - LSE)[~none].abs().max())
        assert err <= LSE_TOL[dtype] * max(1.0, float(LSE[~none].abs().max())), (name, "LSE", err)
    for x in (got[0], got[2]):  # a query that sees nothing: exact zeros
        assert not bool(x[none].any()), name


def _step(Q, K, V, dO, scale, window, sinks, lens=None, **kw):
    from paper_2410_09397_amd import attn
    O, LSE = attn.attn_win_fwd(Q, K, V, scale, window=window, sinks=sinks, lens=lens, **kw)
    return (O, LSE) + tuple(attn.attn_win_bwd(Q, K, V, O, dO, LSE, scale, window=window, sinks=sinks, lens=lens, **kw))


CASES = [
    # dtype, b, h, kvh, n, d, window, sinks, lens
    ("f32", 1, 1, 1, 1, 1, 0, 0, None),
    ("f32", 1, 2, 1, 33, 7, 5, 0, None),
    ("f32", 2, 6, 2, 197, 80, 32, 3, None),
    ("f32", 1, 5, 1, 130, 128, 0, 0, None),
    ("f32", 3, 3, 3, 95, 96, 31, 40, [95, 0, 17]),
    ("f32", 1, 2, 2, 70, 200, 20, 1, None),
    ("f32", 1, 4, 2, 64, 256, 64, 0, None),
    ("f32", 1, 2, 1, 1200, 33, 16, 5, None),   # sink keys shared out over workgroups
    ("bf16", 1, 1, 1, 1, 64, 1, 0, None),
    ("bf16", 1, 1, 1, 2, 128, 1, 1, None),
    ("bf16", 2, 3, 1, 63, 64, 7, 2, None),
    ("bf16", 1, 4, 4, 64, 128, 0, 0, None),
    ("bf16", 1, 8, 2, 65, 128, 64, 64, None),
    ("bf16", 2, 4, 1, 300, 128, 100, 70, [300, 131]),
    ("bf16", 1, 8, 1, 517, 64, 128, 4, None),
    ("bf16", 4, 6, 3, 257, 128, 33, 0, [0, 1, 257, 200]),
    ("bf16", 1, 2, 2, 384, 256, 130, 1, None),
    ("bf16", 2, 5, 1, 190, 256, 0, 0, [190, 64]),
    ("bf16", 1, 10, 2, 1031, 64, 1, 0, None),
    ("bf16", 1, 4, 1, 2111, 128, 257, 130, None),  # sink keys in three tiles, shared out over workgroups
    ("bf16", 1, 3, 1, 1500, 64, 60, 4, [-3]),      # a length below zero counts as zero
    ("bf16", 2, 2, 1, 130, 128, 50, 200, [1000, 129]),  # a length above n counts as n; sinks >= n: no window
    ("bf16", 2, 6, 2, 150, 96, 40, 3, [150, 77]),
    ("bf16", 1, 3, 1, 100, 136, 30, 0, None),
    ("bf16", 1, 2, 1, 90, 8, 13, 2, None),
    ("bf16", 1, 2, 1, 70, 240, 30, 33, None),
]


@pytest.mark.parametrize("dtype,b,h,kvh,n,d,window,sinks,lens", CASES)
def test_window_attention_and_its_gradients(dtype, b, h, kvh, n, d, window, sinks, lens):
    import torch
    print("case window", dtype, b, h, kvh, n, d, window, sinks, lens, flush=True)
    Q, K, V, dO = _inputs(dtype, b, h, kvh, n, d)
    dev = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    _check("window", (Q, K, V, dO), d ** -0.5, window, sinks, lens, _step(Q, K, V, dO, d ** -0.5, window, sinks, dev), dtype)


@pytest.mark.parametrize("dtype,d", [("f32", 48), ("bf16", 64), ("bf16", 128), ("bf16", 72)])
@pytest.mark.parametrize("layout", ["bnhd", "padded"])
def test_other_layouts(dtype, d, layout):
    print("case layout", dtype, d, layout, flush=True)
    Q, K, V, dO = _inputs(dtype, 2, 4, 2, 150, d, layout=layout)
    import torch
    from paper_2410_09397_amd import attn
    like = lambda x: _inputs(dtype, 2, x.shape[1], x.shape[1], 150, d, seed=9, layout=layout)[0]
    O = like(Q)
    LSE = torch.empty(Q.shape[:3], dtype=torch.float32, device="cuda")
    attn.attn_win_fwd(Q, K, V, 0.1, window=60, sinks=5, out=(O, LSE))
    grads = (like(Q), like(K), like(K))
    attn.attn_win_bwd(Q, K, V, O, dO, LSE, 0.1, window=60, sinks=5, out=grads)
    _check("layout", (Q, K, V, dO), 0.1, 60, 5, None, (O, LSE) + grads, dtype)
    if layout == "padded":  # nothing is written into the gaps
        for x in (O,) + grads:
            assert bool(torch.isnan(x.as_strided((x.shape[0], x.shape[1], x.shape[2], 16), x.stride(), x.storage_offset() + d)).all())


@pytest.mark.parametrize("scale", [0.0, -0.7, 3.0])
@pytest.mark.parametrize("dtype,d", [("f32", 32), ("bf16", 64), ("bf16", 128), ("bf16", 256)])
def test_scales_of_either_sign_and_zero(dtype, d, scale):
    print("case scale", dtype, d, scale, flush=True)
    Q, K, V, dO = _inputs(dtype, 1, 2, 1, 140, d, seed=3)
    Q, K = Q * 0.3, K * 0.3
    _check("scale", (Q, K, V, dO), scale, 50, 3, None, _step(Q, K, V, dO, scale, 50, 3), dtype)


@pytest.mark.parametrize("dtype,d", [("f32", 40), ("bf16", 64), ("bf16", 128), ("bf16", 256)])
def test_padding_may_hold_anything(dtype, d):
    """NaN and infinities in rows at and beyond a sequence's length change nothing, down to the bits."""
    import torch
    print("case padding", dtype, d, flush=True)
    n, lens = 333, [200, 0, 64, 333, 129]
    Q, K, V, dO = _inputs(dtype, 5, 4, 2, n, d, seed=4)
    dev = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for x in (Q, K, V, dO):
        for i, l in enumerate(lens):
            x[i, :, l:] = 0
    clean = _step(Q, K, V, dO, 0.1, 90, 5, dev)
    for x, bad in zip((Q, K, V, dO), (math.nan, math.inf, math.nan, -math.inf)):
        for i, l in enumerate(lens):
            x[i, :, l:] = bad
    dirty = _step(Q, K, V, dO, 0.1, 90, 5, dev)
    for a, c in zip(clean, dirty):
        assert torch.equal(a, c)


@pytest.mark.parametrize("window,sinks,lens", [(0, 0, None), (9, 0, None), (9, 3, [41, 26])])
def test_gradients_against_differences_of_the_forward(window, sinks, lens):
    """dL/dx . u for L = sum O o dO against (L(x + e u) - L(x - e u)) / 2e with the fp32 forward.  Error: e^2 / 6 times the third
    derivative (of the order of L's own size with unit-variance inputs: 2e-5 at e = 1e-2) and 2^-24 |O o dO|_1 / e, about 2e-4."""
    import torch
    from paper_2410_09397_amd import attn
    print("case differences", window, sinks, lens, flush=True)
    Q, K, V, dO = _inputs("f32", 2, 4, 2, 41, 24, seed=5)
    dev = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    _, _, *grads = _step(Q, K, V, dO, 24 ** -0.5, window, sinks, dev)

    def loss(q, k, v):
        O, _ = attn.attn_win_fwd(q, k, v, 24 ** -0.5, window=window, sinks=sinks, lens=dev)
        return float((O.double() * dO.double()).sum())

    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)
    e = 1e-2
    for which, g in enumerate(grads):
        x = [Q, K, V]
        u = torch.randn(x[which].shape, generator=gen, device="cuda")
        u /= u.norm()
        x[which] = x[which] + e * u
        up = loss(*x)
        x[which] = x[which] - 2 * e * u
        down = loss(*x)
        want, got = (up - down) / (2 * e), float((g.double() * u.double()).sum())
        assert abs(want - got) <= 5e-3 * max(1.0, abs(want)), (which, want, got)


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 64), ("bf16", 128), ("bf16", 256)])
def test_without_a_window_it_is_causal_attention(dtype, d):
    from paper_2410_09397_amd import attn
    print("case causal", dtype, d, flush=True)
    Q, K, V, dO = _inputs(dtype, 1, 4, 4, 300, d, seed=7)
    O, LSE = attn.attn_fwd(Q, K, V, d ** -0.5, causal=True)
    want = (O, LSE) + tuple(attn.attn_bwd(Q, K, V, O, dO, LSE, d ** -0.5, causal=True))
    for window in (0, 300, 5000):
        got = _step(Q, K, V, dO, d ** -0.5, window, 0)
        for a, c in zip(got, want):
            assert float((a.double() - c.double()).abs().max()) <= TOL[dtype] * max(1.0, float(c.double().abs().max()))


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 64), ("bf16", 128), ("bf16", 256)])
def test_same_bits_again_on_another_stream_and_in_a_graph(dtype, d):
    """The second replay onwards as well, with eager work and new inputs in between."""
    import torch
    from paper_2410_09397_amd import attn
    print("case stream and graph", dtype, d, flush=True)
    n, window, sinks = 700, 65, 3
    Q, K, V, dO = _inputs(dtype, 2, 4, 2, n, d, seed=8)
    lens = torch.tensor([700, 350], dtype=torch.int32, device="cuda")
    want = _step(Q, K, V, dO, 0.1, window, sinks, lens)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = _step(Q, K, V, dO, 0.1, window, sinks, lens, stream=side)
    side.synchronize()
    for a, c in zip(got, want):
        assert torch.equal(a, c)
    out = tuple(torch.empty_like(x) for x in want)
    desc = attn._win_desc(Q, K, 0.1, window, sinks)
    workspace = torch.empty(max(256, attn.attn_win_workspace_bytes(desc)), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        attn.attn_win_fwd(Q, K, V, 0.1, window=window, sinks=sinks, lens=lens, out=out[:2])
        attn.attn_win_bwd(Q, K, V, out[0], dO, out[1], 0.1, window=window, sinks=sinks, lens=lens, out=out[2:], workspace=workspace)
    for seed in (11, 12, 13):
        for x, y in zip((Q, K, V, dO), _inputs(dtype, 2, 4, 2, n, d, seed=seed)):
            x.copy_(y)
        lens.copy_(torch.tensor([700 - seed, 20 * seed], dtype=torch.int32))
        want = _step(Q, K, V, dO, 0.1, window, sinks, lens)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(out, want):
            assert torch.equal(a, c), seed


def test_empty_calls():
    import torch
    from paper_2410_09397_amd import attn
    for b, h, n in ((0, 2, 5), (1, 2, 0)):
        x = torch.empty(b, h, n, 64, dtype=torch.bfloat16, device="cuda")
        O, LSE = attn.attn_win_fwd(x, x, x, 1.0, window=3)
        assert O.shape == x.shape and LSE.shape == x.shape[:3]
        attn.attn_win_bwd(x, x, x, O, x, LSE, 1.0, window=3)
