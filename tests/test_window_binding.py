"""What the binding of windowed attention and the paged cache turns down before the library is called: tensors whose addresses mean nothing on
the GPU."""
import pytest

from paper_2410_09397_amd import attn


def _tensors(device):
    import torch
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=device)
    pages = [bf(4, 2, 16, 64), bf(4, 2, 16, 64)]
    table, lens = torch.arange(4, dtype=torch.int32, device=device).view(2, 2), torch.full((2,), 20, dtype=torch.int32, device=device)
    return bf(2, 4, 20, 64), bf(2, 2, 20, 64), pages, table, lens, bf(2, 4, 64), bf(2, 2, 64), torch.zeros(2, 4, 20, device=device)


def test_host_tensors_are_refused():
    import torch
    Q, K, pages, table, lens, q, k, LSE = _tensors("cpu")
    for call in (lambda: attn.attn_win_fwd(Q, K, K, 1.0, out=(Q, LSE)), lambda: attn.attn_win_bwd(Q, K, K, Q, Q, LSE, 1.0, out=(Q, K, K)),
                 lambda: attn.attn_cache_write(k, k, *pages, table, lens), lambda: attn.attn_cache_read(*pages, table, lens, torch.bfloat16, 2),
                 lambda: attn.attn_paged_fwd(q, *pages, table, lens, 1.0, out=(q, LSE[:, :, 0].contiguous()))):
        with pytest.raises(ValueError, match="on a GPU"):
            call()


def test_tensors_to_read_into_agree_with_the_call():
    """More rows than `total` would be filled with earlier tokens, and another type would go unnoticed."""
    import torch
    pages = [torch.zeros(4, 2, 16, 64) for _ in range(2)]
    table, lens = torch.arange(4, dtype=torch.int32).view(2, 2), torch.full((2,), 20, dtype=torch.int32)
    for shape, dtype in (((6, 2, 64), torch.float32), ((2, 2, 64), torch.float32), ((4, 3, 64), torch.float32), ((4, 2, 32), torch.float32)):
        with pytest.raises(ValueError, match="out must hold"):
            attn.attn_cache_read(*pages, table, lens, dtype, 4, out=tuple(torch.zeros(shape) for _ in range(2)))
    with pytest.raises(ValueError, match="out must hold"):
        attn.attn_cache_read(*pages, table, lens, torch.bfloat16, 4, out=tuple(torch.zeros(4, 2, 64) for _ in range(2)))


@pytest.mark.gpu
def test_workspaces_elsewhere_are_refused():
    import torch
    Q, K, pages, table, lens, q, k, LSE = _tensors("cuda")
    size = 1 << 20
    for bad in (torch.zeros(size, dtype=torch.uint8), torch.zeros(1, dtype=torch.uint8, device="cuda").expand(size),
                torch.zeros(2 * size, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError, match="workspace"):
            attn.attn_win_bwd(Q, K, K, Q, Q, LSE, 1.0, workspace=bad)
        with pytest.raises(ValueError, match="workspace"):
            attn.attn_paged_fwd(q, *pages, table, lens, 1.0, workspace=bad)
    attn.attn_paged_fwd(q, *pages, table, lens, 1.0, workspace=torch.zeros(size, dtype=torch.uint8, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("side", [False, True])
def test_keys_that_no_head_reads_have_gradients_of_zero(side):
    import torch
    Q, K = torch.zeros(2, 0, 30, 64, device="cuda"), torch.randn(2, 3, 30, 64, device="cuda")
    LSE, stream = torch.zeros(2, 0, 30, device="cuda"), torch.cuda.Stream() if side else None
    out = (torch.empty_like(Q), torch.full_like(K, 7.0), torch.full_like(K, 7.0))
    torch.cuda.synchronize()
    attn.attn_win_bwd(Q, K, K, Q, Q, LSE, 1.0, stream=stream, out=out)
    torch.cuda.synchronize()
    assert not bool(out[1].any()) and not bool(out[2].any())
    assert attn.attn_win_fwd(Q, K, K, 1.0, stream=stream)[0].shape == Q.shape
