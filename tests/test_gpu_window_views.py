"""Queries, keys and values that are views of one fused tensor, as a projection makes them: the results are those of separate tensors, down to
the bits, and have the views' strides.  (The kernels take the same steps whatever the strides are.)"""
import pytest

from paper_2410_09397_amd import attn


def _views(x, heads, kv_heads):
    """Q, K and V of a fused [..., heads + 2 kv_heads, d]."""
    return x[..., :heads, :], x[..., heads:heads + kv_heads, :], x[..., heads + kv_heads:, :]


@pytest.mark.parametrize("shape,cut", [((10, 12, 64), (slice(None), slice(0, 8))), ((7, 12, 64), (slice(None), slice(8, 9))), ((5, 3, 12, 64), (slice(None), slice(None), slice(2, 4)))])
def test_an_image_of_a_view_has_its_strides(shape, cut):
    import torch
    for x in (torch.zeros(shape)[cut], torch.zeros(shape)[cut].transpose(-2, -3)):
        y = attn._empty_as(x)
        assert y.shape == x.shape and y.stride() == x.stride() and y.dtype == x.dtype
        y.zero_()
        for i in range(y.numel()):
            y[tuple(int(v) for v in torch.unravel_index(torch.tensor(i), y.shape))] += 1  # an entry that shared memory would be counted twice
        assert bool((y == 1).all())


def test_views_whose_entries_share_memory_have_no_image():
    import torch
    x = torch.zeros(4, 8, 16)
    for bad in (x[:1].expand(4, -1, -1), x.as_strided((4, 8, 16), (64, 16, 1)), x.as_strided((4, 8, 16), (127, 16, 1)), x.as_strided((4, 8, 16), (128, 8, 1))):
        with pytest.raises(ValueError):
            attn._empty_as(bad)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [("f32", 33), ("bf16", 64), ("bf16", 128), ("bf16", 256), ("bf16", 96)])
@pytest.mark.parametrize("n", [1, 150])
def test_a_training_step_on_views(dtype, d, n):
    import torch
    print("case views", dtype, d, n, flush=True)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    fused = torch.randn(2, n, 8, d, device="cuda").to(dt)
    lens = torch.tensor([n, max(1, n - 31)], dtype=torch.int32, device="cuda")
    views = [t.transpose(1, 2) for t in _views(fused, 4, 2)]
    O, LSE = attn.attn_win_fwd(*views, 0.1, window=60, sinks=5, lens=lens)
    assert O.stride() == views[0].stride()
    dO = attn._empty_as(O).copy_(torch.randn(O.shape, device="cuda"))
    grads = attn.attn_win_bwd(*views, O, dO, LSE, 0.1, window=60, sinks=5, lens=lens)
    Q, K, V = (t.contiguous() for t in views)
    wO, wL = attn.attn_win_fwd(Q, K, V, 0.1, window=60, sinks=5, lens=lens)
    want = attn.attn_win_bwd(Q, K, V, wO, dO.contiguous(), wL, 0.1, window=60, sinks=5, lens=lens)
    for got, ref in zip((O, LSE, *grads), (wO, wL, *want)):
        assert torch.equal(got, ref)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,d", [("plain", 64), ("plain", 128), ("fp8", 128), ("plain", 40)])
@pytest.mark.parametrize("new", [1, 5, 90])
def test_a_serving_step_on_views(kind, d, new):
    import torch
    print("case serving views", kind, d, new, flush=True)
    batch, kvh, page, n = 3, 2, 16, 200
    fused = torch.randn(batch * new, 12, d, device="cuda").to(torch.bfloat16)
    pages = attn.attn_cache_pages(batch * -(-n // page), kvh, page, d, torch.bfloat16 if kind == "plain" else torch.float8_e4m3fn)
    exps = dict(K_exp=pages[2], V_exp=pages[3])
    table = torch.arange(batch * -(-n // page), dtype=torch.int32, device="cuda").view(batch, -1)
    lens = torch.tensor([n, new, n - 7], dtype=torch.int32, device="cuda")
    results = []
    for Q, K, V in (_views(fused, 8, 2), [t.contiguous() for t in _views(fused, 8, 2)]):
        for x in pages:
            if x is not None:
                x.view(torch.uint8).zero_()
        attn.attn_cache_write(K, V, *pages[:2], table, lens, **exps)
        O, LSE = attn.attn_paged_fwd(Q, *pages[:2], table, lens, 0.1, **exps)
        assert O.stride() == Q.stride()
        results.append((O, LSE, *(x.view(torch.uint8).clone() for x in pages if x is not None)))
    for got, ref in zip(*results):
        assert torch.equal(got, ref)
