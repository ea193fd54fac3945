"""Weights and eviction of a cache by calls without query heads: every token of the cache is worked on all the same, as by a call without new tokens."""
import ctypes

import pytest

from paper_2410_09397_amd import attn
from tests.test_keep_abi import BAD, OK, evict, weigh
from tests.test_window_abi import paged


def test_only_a_call_without_key_heads_has_nothing_to_do():
    for kw in (dict(heads=0, kv_heads=0), dict(batch=0, heads=0), dict(max_len=0, heads=0)):
        assert weigh(paged(**kw), None, None, None) == OK and evict(paged(**kw), None, ws=None, size=0) == OK
    d = paged(heads=0)  # two key heads: there is a cache to work on, and here none is given
    assert weigh(d, None, None, None) == BAD and evict(d, None) == BAD
    assert attn.lib().attn_weigh_workspace_bytes(ctypes.byref(d)) == 256
    long = paged(heads=0, max_len=400, max_pages=30, table_stride=30)
    assert attn.lib().attn_evict_workspace_bytes(ctypes.byref(long), 200) == attn.lib().attn_evict_workspace_bytes(
        ctypes.byref(paged(max_len=400, max_pages=30, table_stride=30)), 200) > 256


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind,d", [("bf16", "plain", 64), ("bf16", "fp8", 128), ("bf16", "fp8", 72), ("f32", "plain", 33)])
def test_weights_decay_without_query_heads(dtype, kind, d):
    import torch
    from tests.test_gpu_paged import DTYPES, Cache
    print("case weigh without heads", dtype, kind, d, flush=True)
    c = Cache(dtype, kind, [5, 90], 2, d, 16)
    t = getattr(torch, DTYPES[dtype])
    for new in (0, 3):
        Q, LSE = torch.empty(2 * new, 0, d, dtype=t, device="cuda"), torch.empty(2 * new, 0, device="cuda")
        w = torch.rand(2, 2, 96, device="cuda")
        want = w.clone()
        for b, l in enumerate(c.host_lens):
            want[b, :, :l - new] *= 0.5
            want[b, :, l - new:l] = 0.0
        assert attn.attn_cache_weigh(Q, LSE, *c.args(), 1.0, weight=w, decay=0.5, **c.exps()) is w
        assert torch.equal(w, want)


@pytest.mark.gpu
@pytest.mark.parametrize("budget", [20, 300])
def test_evicting_without_query_heads(budget):
    import torch
    from tests.test_gpu_paged import Cache
    from tests.test_gpu_tree import _raw
    print("case evict without heads", budget, flush=True)
    lens = [1000, 100, 7]
    a, b = (Cache("bf16", "plain", lens, 2, 64, 16, seed=3) for _ in range(2))
    slots = a.table.shape[1] * 16
    w = torch.rand(3, 2, slots, device="cuda")
    want = attn.attn_cache_evict(w.clone(), *a.args(), budget, recent=5)
    got, lens_out, scratch = w.clone(), torch.full((3,), -1, dtype=torch.int32, device="cuda"), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    desc, cache = attn._on_pages("evict", 0, 0, 128, 64, torch.bfloat16, b.K.device, *b.args(), None, 0, None, None, None)
    args = attn._EVICTION.pack(budget, 0, 5, 0, got.data_ptr(), 0, 0, 0, got.data_ptr(), 0, lens_out.data_ptr(), 2 * slots, slots, 2 * slots, slots)
    assert attn.lib().attn_cache_evict(desc, cache, args, scratch.data_ptr(), scratch.numel(), torch.cuda.current_stream().cuda_stream) == OK
    assert torch.equal(lens_out, want[2]) and torch.equal(got, want[0])
    assert torch.equal(_raw(a.K), _raw(b.K)) and torch.equal(_raw(a.V), _raw(b.V))


@pytest.mark.gpu
def test_new_lengths_of_a_cache_without_tokens_are_written_where_they_are_wanted():
    """No key heads, or max_len = 0: nothing moves, and the new lengths come back in `out` as they do without it."""
    import torch
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    lens, table = ints([5, 9]), torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    for kvh, max_len, want in ((0, None, [5, 7]), (2, 0, [0, 0])):
        pages = torch.zeros(2, kvh, 16, 64, dtype=torch.bfloat16, device="cuda")
        w = torch.ones(2, kvh, 16, device="cuda")
        side = torch.cuda.Stream()
        for stream in (None, side):
            out = w.clone(), None, ints([-1, -1])
            torch.cuda.synchronize()
            got = attn.attn_cache_evict(w, pages, pages.clone(), table, lens, 7, max_len=max_len, out=out, stream=stream)
            torch.cuda.synchronize()
            assert got is out and out[2].tolist() == want
            made = attn.attn_cache_evict(w, pages, pages.clone(), table, lens, 7, max_len=max_len, stream=stream)
            torch.cuda.synchronize()
            assert made[2].tolist() == want
