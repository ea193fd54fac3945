"""Refusals of windowed attention and the paged cache: every bad argument is turned down on the host, before anything is launched."""
import ctypes

import pytest

from paper_2410_09397_amd import attn

P = 0x1000  # a non-null, 16-byte aligned fake device address: never dereferenced by a rejected call
BAD, UNSUPPORTED, WORKSPACE = attn.ATTN_ERR_INVALID_ARG, attn.ATTN_ERR_UNSUPPORTED, attn.ATTN_ERR_WORKSPACE


def win(**kw):
    d, n = kw.get("d", 64), kw.get("n", 100)
    base = dict(batch=2, heads=4, kv_heads=2, n=n, d=d, scale=0.1, window=8, sinks=1, dtype=attn.ATTN_BF16, reserved=0, q_stride_b=4 * n * d,
                q_stride_h=n * d, q_stride_n=d, kv_stride_b=2 * n * d, kv_stride_h=n * d, kv_stride_n=d)
    base.update(kw)
    return attn.attn_win_desc(**base)


def win_fwd(d, ptrs=(P,) * 5):
    return attn.lib().attn_win_fwd(ctypes.byref(d) if d is not None else None, None, *ptrs, None)


def win_bwd(d, ptrs=(P,) * 9, ws=P, ws_bytes=1 << 40):
    return attn.lib().attn_win_bwd(ctypes.byref(d) if d is not None else None, None, *ptrs, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), BAD), (dict(n=-1), BAD), (dict(heads=-4), BAD), (dict(kv_heads=-1), BAD), (dict(d=0, q_stride_n=8, kv_stride_n=8), BAD),
    (dict(heads=3), BAD),                                  # not a multiple of the key heads
    (dict(kv_heads=0), BAD), (dict(window=-1), BAD), (dict(sinks=-1), BAD), (dict(reserved=1), BAD),
    (dict(scale=float("inf")), BAD), (dict(scale=float("nan")), BAD),
    (dict(q_stride_n=32), BAD), (dict(kv_stride_n=56), BAD), (dict(q_stride_n=68), BAD), (dict(kv_stride_h=6404), BAD),
    (dict(q_stride_h=0), BAD), (dict(kv_stride_b=0), BAD), (dict(kv_stride_h=-6400), BAD),  # rows that overlap
    (dict(dtype=2), UNSUPPORTED), (dict(d=264), UNSUPPORTED), (dict(d=60), UNSUPPORTED),
    (dict(q_stride_n=1 << 22), UNSUPPORTED), (dict(kv_stride_n=1 << 22), UNSUPPORTED),
    (dict(n=1 << 30), UNSUPPORTED), (dict(batch=1 << 24), UNSUPPORTED),
])
def test_bad_window_descriptors(kw, status):
    d = win(**kw)
    assert win_fwd(d) == status and win_bwd(d) == status
    assert attn.lib().attn_win_workspace_bytes(ctypes.byref(d)) == 0


def test_window_pointers_and_workspace():
    d = win()
    need = attn.lib().attn_win_workspace_bytes(ctypes.byref(d))
    assert need >= 2 * 4 * 100 * 4
    assert win_fwd(None) == BAD and win_bwd(None) == BAD
    for i in range(5):
        assert win_fwd(d, tuple(None if j == i else P for j in range(5))) == BAD
    for i in range(9):
        assert win_bwd(d, tuple(None if j == i else P for j in range(9))) == BAD
    for i in (0, 1, 2, 3):
        assert win_fwd(d, tuple(P + 8 if j == i else P for j in range(5))) == BAD
    assert win_bwd(d, (P,) * 8 + (P + 2,)) == BAD
    assert win_bwd(d, ws=None) == WORKSPACE and win_bwd(d, ws_bytes=need - 1) == WORKSPACE and win_bwd(d, ws=P + 4) == WORKSPACE
    for kw in (dict(batch=0), dict(n=0), dict(heads=0), dict(heads=0, kv_heads=0)):
        assert win_fwd(win(**kw), (None,) * 5) == attn.ATTN_OK and win_bwd(win(**kw), (None,) * 9, None, 0) == attn.ATTN_OK


def paged(**kw):
    d = kw.get("d", 64)
    base = dict(batch=2, heads=4, kv_heads=2, d=d, total_q=6, max_q=3, max_len=100, page_size=16, num_pages=9, max_pages=7, scale=0.1, window=0,
                sinks=0, dtype=attn.ATTN_BF16, kind=attn.ATTN_CACHE_FP8, reserved=0, q_stride_n=4 * d, q_stride_h=d, kv_stride_n=2 * d, kv_stride_h=d,
                page_stride_p=32 * d, page_stride_h=16 * d, page_stride_n=d, table_stride=7)
    base.update(kw)
    return attn.attn_paged_desc(**base)


def cache(**kw):
    base = dict(K=P, V=P, K_exp=P, V_exp=P, table=P, lens=P, q_ptr=P)
    base.update(kw)
    return attn.attn_cache(**base)


def calls(d, c=None, a=P, b=P):
    L = attn.lib()
    d = ctypes.byref(d) if d is not None else None
    c = ctypes.byref(cache() if c is None else c)
    return (L.attn_cache_write(d, c, a, b, None), L.attn_cache_read(d, c, a, b, None), L.attn_paged_fwd(d, c, a, b, P, P, 1 << 40, None))


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), BAD), (dict(total_q=-1), BAD), (dict(max_q=-1), BAD), (dict(max_len=-1), BAD), (dict(num_pages=-1), BAD),
    (dict(max_pages=-1), BAD), (dict(reserved=3), BAD), (dict(heads=5), BAD), (dict(scale=float("nan")), BAD), (dict(window=-2), BAD),
    (dict(max_len=113), BAD),                              # longer than a row of the table can hold
    (dict(table_stride=6), BAD), (dict(num_pages=0), BAD),
    (dict(q_stride_n=60), BAD), (dict(kv_stride_h=4), BAD), (dict(page_stride_n=32), BAD), (dict(page_stride_n=72), BAD),
    (dict(page_stride_h=0), BAD), (dict(page_stride_p=-1024), BAD),
    (dict(page_size=24), UNSUPPORTED), (dict(page_size=4), UNSUPPORTED), (dict(page_size=8192), UNSUPPORTED), (dict(page_size=0), UNSUPPORTED),
    (dict(dtype=9), UNSUPPORTED), (dict(kind=2), UNSUPPORTED), (dict(d=512), UNSUPPORTED),
    (dict(d=60, dtype=attn.ATTN_F32, kind=attn.ATTN_CACHE_FP8), UNSUPPORTED),
    (dict(batch=65536), UNSUPPORTED), (dict(max_q=1 << 29), UNSUPPORTED),
])
def test_bad_cache_descriptors(kw, status):
    d = paged(**kw)
    assert calls(d) == (status,) * 3
    if "num_pages" not in kw or kw["num_pages"] < 0:
        assert attn.lib().attn_paged_workspace_bytes(ctypes.byref(d)) == 0


@pytest.mark.parametrize("kw", [dict(K=None), dict(V=None), dict(table=None), dict(lens=None), dict(K_exp=None), dict(V_exp=None), dict(K=P + 8),
                                dict(V=P + 4)])
def test_bad_caches(kw):
    assert calls(paged(), cache(**kw)) == (BAD,) * 3


def test_cache_pointers_and_workspace():
    L, d = attn.lib(), paged()
    assert calls(None) == (BAD,) * 3
    assert calls(d, a=None) == (BAD,) * 3 and calls(d, b=None) == (BAD,) * 3 and calls(d, a=P + 2) == (BAD,) * 3
    c = cache()
    assert L.attn_paged_fwd(ctypes.byref(d), None, P, P, P, P, 1 << 40, None) == BAD
    assert L.attn_paged_fwd(ctypes.byref(d), ctypes.byref(c), P, P, None, P, 1 << 40, None) == BAD
    assert calls(paged(total_q=5), cache(q_ptr=None)) == (BAD,) * 3  # 2 sequences of 3 rows need 6
    long = paged(max_len=4000, max_pages=300, table_stride=300)  # few rows, a long cache: the work is split
    need = L.attn_paged_workspace_bytes(ctypes.byref(long))
    assert need > 256
    for ws, size in ((None, need), (P, need - 256), (P + 8, need)):
        assert L.attn_paged_fwd(ctypes.byref(long), ctypes.byref(c), P, P, P, ws, size, None) == WORKSPACE
    for kw in (dict(batch=0), dict(total_q=0), dict(max_q=0), dict(heads=0)):
        empty = paged(**kw)
        assert L.attn_paged_fwd(ctypes.byref(empty), None, None, None, None, None, 0, None) == attn.ATTN_OK
        assert L.attn_cache_write(ctypes.byref(empty), None, None, None, None) == attn.ATTN_OK


def test_the_binding_checks_what_it_passes_on():
    import torch
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    q, k = bf(1, 4, 10, 64), bf(1, 2, 10, 64)
    for args in ((bf(1, 4, 9, 64), k, k), (q, k, bf(1, 2, 10, 32)), (q, k.float(), k.float()), (q[..., ::2], k, k), (q.half(), k.half(), k.half())):
        with pytest.raises(ValueError):
            attn.attn_win_fwd(*args, 1.0)
    with pytest.raises(ValueError):
        attn.attn_win_fwd(q, k, k, 1.0, lens=torch.zeros(1, dtype=torch.int64))
    with pytest.raises(ValueError):
        attn.attn_win_bwd(q, k, k, q, q, torch.zeros(1, 4, 9), 1.0)
    pages, exps = torch.zeros(3, 2, 16, 64, dtype=torch.float8_e4m3fn), torch.zeros(3, 2, 16, dtype=torch.uint8)
    table, lens, rows = torch.zeros(2, 3, dtype=torch.int32), torch.ones(2, dtype=torch.int32), bf(2, 4, 64)
    ok = dict(K_exp=exps, V_exp=exps)
    for a, kw in (((rows, pages, pages, table, lens), dict(K_exp=exps)),                            # no exponents for V
                  ((rows, pages, pages, table.long(), lens), ok), ((rows, pages, pages, table, lens[:1]), ok),
                  ((rows.float(), bf(3, 2, 16, 64), bf(3, 2, 16, 64), table, lens), {}),            # pages of another type
                  ((bf(3, 4, 64), pages, pages, table, lens), ok),                                  # 3 rows, 2 sequences
                  ((rows, pages, pages, table, lens), dict(ok, q_ptr=torch.zeros(3, dtype=torch.int32)))):  # no max_q
        with pytest.raises(ValueError):
            attn.attn_paged_fwd(*a, 1.0, **kw)
    with pytest.raises(ValueError):
        attn.attn_cache_write(rows, rows, pages, pages, table, lens, **ok)  # 4 heads, pages of 2
