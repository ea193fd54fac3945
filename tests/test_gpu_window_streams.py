"""Results of a call on a stream of its own are not put into memory that was freed on the current one, where earlier work may still use it."""
import pytest

pytestmark = pytest.mark.gpu


def _freed(*tensors):
    """Addresses of blocks of these tensors' sizes that the current stream has free."""
    import torch
    blocks = [torch.empty_like(x) for x in tensors for _ in range(2)]
    return {x.data_ptr() for x in blocks}


def test_windowed_attention_takes_its_results_from_the_pool_of_its_stream():
    import torch
    from paper_2410_09397_amd import attn
    Q = torch.randn(2, 8, 1024, 128, device="cuda").to(torch.bfloat16)
    K, V, dO = Q[:, :4].contiguous(), Q[:, 4:].contiguous(), Q.flip(2).contiguous()
    want_O, want_LSE = attn.attn_win_fwd(Q, K, V, 0.1, window=100)
    want = attn.attn_win_bwd(Q, K, V, want_O, dO, want_LSE, 0.1, window=100)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    free = _freed(Q, want_LSE, K)
    O, LSE = attn.attn_win_fwd(Q, K, V, 0.1, window=100, stream=side)
    grads = attn.attn_win_bwd(Q, K, V, O, dO, LSE, 0.1, window=100, stream=side)
    side.synchronize()
    for got, ref in zip((O, LSE, *grads), (want_O, want_LSE, *want)):
        assert got.data_ptr() not in free
        assert torch.equal(got, ref)


def test_the_paged_cache_takes_its_results_from_the_pool_of_its_stream():
    import torch
    from paper_2410_09397_amd import attn
    B, new, page = 4, 512, 16
    K, V = (torch.randn(B * new, 4, 128, device="cuda").to(torch.bfloat16) for _ in range(2))
    Q = torch.randn(B * new, 8, 128, device="cuda").to(torch.bfloat16)
    pages = attn.attn_cache_pages(B * new // page, 4, page, 128, torch.bfloat16)[:2]
    table = torch.arange(B * new // page, dtype=torch.int32, device="cuda").view(B, -1)
    lens = torch.full((B,), new, dtype=torch.int32, device="cuda")
    attn.attn_cache_write(K, V, *pages, table, lens)
    want_O, want_LSE = attn.attn_paged_fwd(Q, *pages, table, lens, 0.1)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    free = _freed(Q, want_LSE, K)
    O, LSE = attn.attn_paged_fwd(Q, *pages, table, lens, 0.1, stream=side)
    back = attn.attn_cache_read(*pages, table, lens, torch.bfloat16, B * new, stream=side)
    side.synchronize()
    for got, ref in zip((O, LSE, *back), (want_O, want_LSE, K, V)):
        assert got.data_ptr() not in free
        assert torch.equal(got, ref)
