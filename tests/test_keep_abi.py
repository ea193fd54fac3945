"""Refusals of trees, weights and eviction: every bad argument is turned down on the host, before anything is launched."""
import ctypes

import pytest

from paper_2410_09397_amd import attn
from tests.test_window_abi import BAD, P, UNSUPPORTED, WORKSPACE, cache, paged

OK = attn.ATTN_OK
A, B, C = 0x10000, 0x20000, 0x30000  # more addresses that no rejected call dereferences


def ref(x):
    return None if x is None else ctypes.byref(x)


def tree_fwd(d, c="cache", mask=P, stride=1, q=P, o=P, lse=P, ws=P, size=1 << 40):
    return attn.lib().attn_tree_fwd(ref(d), ref(cache() if c == "cache" else c), mask, stride, q, o, lse, ws, size, None)


def commit(d, c="cache", mask=P, stride=1, leaf=A, new=B):
    return attn.lib().attn_tree_commit(ref(d), ref(cache() if c == "cache" else c), mask, stride, leaf, new, None)


def weights(**kw):
    base = dict(in_=A, out=B, in_stride_b=200, in_stride_h=100, out_stride_b=200, out_stride_h=100, decay=1.0, reserved=0)
    base.update(kw)
    return attn.attn_weights(**base)


def weigh(d, c="cache", q=P, lse=P, w="weights", ws=P, size=1 << 40):
    return attn.lib().attn_cache_weigh(ref(d), ref(cache() if c == "cache" else c), q, lse, ref(weights() if w == "weights" else w), ws, size, None)


def eviction(**kw):
    base = dict(budget=50, first=2, recent=3, reserved=0, weight=A, pos=B, kept=P, seen=P, weight_out=A, pos_out=B, new_lens=C, stride_b=200, stride_h=100,
                out_stride_b=200, out_stride_h=100)
    base.update(kw)
    return attn.attn_eviction(**base)


def evict(d, c="cache", e="eviction", ws=P, size=1 << 40):
    return attn.lib().attn_cache_evict(ref(d), ref(cache() if c == "cache" else c), ref(eviction() if e == "eviction" else e), ws, size, None)


CALLS = [tree_fwd, commit, weigh, evict]


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), BAD), (dict(total_q=-1), BAD), (dict(max_q=-1), BAD), (dict(max_len=-1), BAD), (dict(num_pages=-1), BAD), (dict(reserved=3), BAD),
    (dict(heads=5), BAD), (dict(scale=float("nan")), BAD), (dict(window=-2), BAD), (dict(max_len=113), BAD), (dict(table_stride=6), BAD),
    (dict(num_pages=0), BAD), (dict(page_stride_n=32), BAD), (dict(page_stride_n=72), BAD), (dict(page_stride_h=0), BAD),
    (dict(page_size=24), UNSUPPORTED), (dict(dtype=9), UNSUPPORTED), (dict(kind=2), UNSUPPORTED), (dict(d=512), UNSUPPORTED),
    (dict(d=60, dtype=attn.ATTN_F32, kind=attn.ATTN_CACHE_FP8), UNSUPPORTED), (dict(batch=65536), UNSUPPORTED), (dict(max_q=1 << 29), UNSUPPORTED),
])
def test_bad_cache_descriptors(kw, status):
    d = paged(**kw)
    assert [call(d) for call in CALLS] == [status] * 4
    if "num_pages" not in kw or kw["num_pages"] < 0:
        assert attn.lib().attn_tree_workspace_bytes(ctypes.byref(d)) == 0
        assert attn.lib().attn_evict_workspace_bytes(ctypes.byref(d), 50) == attn.lib().attn_weigh_workspace_bytes(ctypes.byref(d)) == 0


@pytest.mark.parametrize("kw", [dict(K=None), dict(V=None), dict(table=None), dict(lens=None), dict(K_exp=None), dict(V_exp=None), dict(K=P + 8),
                                dict(V=P + 4)])
def test_bad_caches(kw):
    assert [call(paged(), cache(**kw)) for call in CALLS] == [BAD] * 4


def test_missing_structures():
    assert [call(None) for call in CALLS] == [BAD] * 4 and [call(paged(), None) for call in CALLS] == [BAD] * 4
    assert weigh(paged(), w=None) == BAD and evict(paged(), e=None) == BAD and evict(None, e=None) == BAD


def test_trees():
    d = paged()
    for bad in (dict(q=None), dict(o=None), dict(lse=None), dict(q=P + 2), dict(o=P + 8), dict(mask=None), dict(stride=-1), dict(stride=0)):
        assert tree_fwd(d, **bad) == BAD
    assert commit(d, mask=None) == BAD and commit(d, stride=0) == BAD and commit(d, leaf=None) == BAD and commit(d, new=None) == BAD
    assert commit(d, new=A) == BAD and commit(d, new=P) == BAD and commit(d, new=A + 4) == BAD  # over leaf, over lens
    wide = paged(max_q=40, total_q=80)
    assert tree_fwd(wide, stride=1) == BAD and commit(wide, stride=1) == BAD  # 40 tokens are two words
    many = paged(max_q=1025, total_q=2050)
    assert tree_fwd(many, stride=33) == UNSUPPORTED and commit(many, stride=33) == UNSUPPORTED
    assert attn.lib().attn_tree_workspace_bytes(ctypes.byref(many)) == 0
    assert tree_fwd(paged(total_q=5), cache(q_ptr=None)) == BAD and commit(paged(total_q=5), cache(q_ptr=None)) == BAD
    assert commit(paged(batch=65535, heads=1 << 16, kv_heads=1 << 16, max_q=1, total_q=65535, q_stride_n=1 << 40)) == UNSUPPORTED
    long = paged(max_len=4000, max_pages=300, table_stride=300)  # few rows, a long cache: the work is split
    need = attn.lib().attn_tree_workspace_bytes(ctypes.byref(long))
    assert need > 256
    for ws, size in ((None, need), (P, need - 256), (P + 8, need)):
        assert tree_fwd(long, ws=ws, size=size) == WORKSPACE
    for kw in (dict(batch=0), dict(total_q=0), dict(max_q=0), dict(heads=0)):
        assert tree_fwd(paged(**kw), None, None, 0, None, None, None, None, 0) == OK and commit(paged(**kw), None, None, 0, None, None) == OK


def test_masks():
    call = attn.lib().attn_tree_mask
    for args in ((2, 6, 3, P, None, P, 1), (-1, 6, 3, P, P, P, 1), (2, -6, 3, P, P, P, 1), (2, 6, -3, P, P, P, 1), (2, 6, 3, P, P, None, 1), (2, 6, 3, P, P, P, 0),
                 (2, 6, 3, P, P, P, -1), (2, 80, 40, P, P, P, 1), (2, 5, 3, None, P, P, 1)):
        assert call(*args, None) == BAD
    assert call(65536, 6, 3, P, P, P, 1, None) == UNSUPPORTED and call(2, 4000, 1025, P, P, P, 40, None) == UNSUPPORTED
    assert call(2, 1 << 30, 3, P, P, P, 1, None) == UNSUPPORTED
    for args in ((0, 6, 3), (2, 0, 3), (2, 6, 0)):
        assert call(*args, None, None, None, 0, None) == OK


@pytest.mark.parametrize("kw", [dict(out=None), dict(reserved=1), dict(decay=float("nan")), dict(decay=float("inf")), dict(out_stride_h=99),
                                dict(out_stride_b=99), dict(in_stride_h=-100), dict(in_stride_b=0), dict(out_stride_h=-100),
                                dict(in_=B, in_stride_b=400), dict(in_=B, in_stride_h=101)])
def test_bad_weights(kw):
    assert weigh(paged(), w=weights(**kw)) == BAD


def test_weigh_pointers_and_sizes():
    d = paged()
    assert weigh(d, q=None) == BAD and weigh(d, lse=None) == BAD and weigh(d, q=P + 2) == BAD
    assert weigh(paged(total_q=5), cache(q_ptr=None)) == BAD
    for kw in (dict(batch=0), dict(heads=0, kv_heads=0), dict(max_len=0)):
        assert weigh(paged(**kw), None, None, None) == OK
    prompt = paged(total_q=4000, max_q=2000, max_len=2000, max_pages=200, table_stride=200)  # many rows for few keys: they are shared out
    need = attn.lib().attn_weigh_workspace_bytes(ctypes.byref(prompt))
    assert need > 256
    slots = weights(in_stride_b=4000, in_stride_h=2000, out_stride_b=4000, out_stride_h=2000)
    for ws, size in ((None, need), (P, need - 1), (P + 8, need)):
        assert weigh(prompt, w=slots, ws=ws, size=size) == WORKSPACE
    big = dict(max_len=1 << 28, max_pages=1 << 24, table_stride=1 << 24)
    huge = dict(in_stride_b=1 << 40, in_stride_h=1 << 30, out_stride_b=1 << 40, out_stride_h=1 << 30)
    assert weigh(paged(batch=64, **big), w=weights(**huge)) == UNSUPPORTED
    assert weigh(paged(batch=65535, heads=1 << 16, kv_heads=1 << 16, max_q=0, q_stride_n=1 << 40, kv_stride_n=1 << 40), w=weights(**huge)) == UNSUPPORTED


@pytest.mark.parametrize("kw", [dict(budget=0), dict(budget=-1), dict(first=-1), dict(recent=-1), dict(first=40, recent=11), dict(reserved=1), dict(weight=None),
                                dict(weight_out=None), dict(new_lens=None), dict(pos_out=None), dict(stride_h=99), dict(stride_b=-1), dict(out_stride_h=49),
                                dict(out_stride_b=0), dict(out_stride_b=300), dict(weight_out=C + 4096, out_stride_h=90), dict(new_lens=P), dict(new_lens=P + 4),
                                dict(first=2 ** 31 - 1, recent=2 ** 31 - 1)])
def test_bad_evictions(kw):
    assert evict(paged(), e=eviction(**kw)) == BAD


def test_evict_workspace():
    L, d = attn.lib(), paged()
    assert L.attn_evict_workspace_bytes(ctypes.byref(d), 50) == 256  # 50 tokens move without one
    long = paged(max_len=400, max_pages=30, table_stride=30)
    need = L.attn_evict_workspace_bytes(ctypes.byref(long), 200)
    assert need >= 2 * 2 * 2 * 200 * 4  # 200 of 400 tokens may move, from and to, for two key heads of two sequences
    slots = eviction(budget=200, stride_b=1000, stride_h=400, out_stride_b=1000, out_stride_h=400)
    for ws, size in ((None, need), (P, need - 1), (P + 4, need)):
        assert evict(long, e=slots, ws=ws, size=size) == WORKSPACE
    assert L.attn_evict_workspace_bytes(ctypes.byref(d), 0) == 0 and L.attn_evict_workspace_bytes(None, 5) == 0
    assert L.attn_evict_workspace_bytes(ctypes.byref(d), 100) == 256 and L.attn_evict_workspace_bytes(ctypes.byref(d), 2 ** 31 - 1) == 256
    for kw in (dict(batch=0), dict(heads=0, kv_heads=0), dict(max_len=0)):
        assert evict(paged(**kw), None, ws=None, size=0) == OK


def _tensors(device="cpu"):
    import torch
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=device)
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32, device=device)
    return dict(q=bf(6, 4, 64), lse=torch.zeros(6, 4, device=device), mask=ints(6, 1), pages=(bf(8, 2, 16, 64), bf(8, 2, 16, 64)), table=ints(2, 4),
                lens=ints(2) + 20, w=torch.zeros(2, 2, 64, device=device), pos=ints(2, 2, 64), leaf=ints(2))


def test_host_tensors_are_refused():
    t = _tensors()
    at = (*t["pages"], t["table"], t["lens"])
    for call in (lambda: attn.attn_tree_mask(t["leaf"], 1), lambda: attn.attn_tree_fwd(t["q"], t["mask"], *at, 1.0), lambda: attn.attn_tree_commit(t["mask"], t["leaf"], *at),
                 lambda: attn.attn_cache_weigh(t["q"], t["lse"], *at, 1.0), lambda: attn.attn_cache_evict(t["w"], *at, 5)):
        with pytest.raises(ValueError, match="on a GPU"):
            call()


@pytest.mark.gpu
def test_the_binding_checks_what_it_passes_on():
    import torch
    t = _tensors("cuda")
    at, q, lse, mask, leaf, w, pos = (*t["pages"], t["table"], t["lens"]), t["q"], t["lse"], t["mask"], t["leaf"], t["w"], t["pos"]
    ptr = torch.tensor([0, 3, 6], dtype=torch.int32, device="cuda")
    bad = [lambda: attn.attn_tree_mask(mask, 3), lambda: attn.attn_tree_mask(leaf.long(), 1), lambda: attn.attn_tree_mask(leaf, 3), lambda: attn.attn_tree_mask(leaf, -1),
           lambda: attn.attn_tree_mask(mask[:, 0].contiguous(), 3, out=mask[:5]), lambda: attn.attn_tree_mask(mask[:, 0].contiguous(), 3, out=mask.long()),
           lambda: attn.attn_tree_mask(mask[:, 0].contiguous(), 3, q_ptr=ptr.long()),
           lambda: attn.attn_tree_fwd(q, mask[:5], *at, 1.0), lambda: attn.attn_tree_fwd(q, mask.long(), *at, 1.0), lambda: attn.attn_tree_fwd(q, mask.cpu(), *at, 1.0),
           lambda: attn.attn_tree_fwd(q, mask, *at, 1.0, q_ptr=ptr, max_q=33), lambda: attn.attn_tree_fwd(q, mask, *at, 1.0, q_ptr=ptr),
           lambda: attn.attn_tree_fwd(q, torch.zeros(6, 8, dtype=torch.int32, device="cuda")[:, ::4], *at, 1.0, q_ptr=ptr, max_q=33),
           lambda: attn.attn_tree_fwd(q, mask, *at, 1.0, workspace=torch.zeros(1 << 20, dtype=torch.uint8)), lambda: attn.attn_tree_fwd(q.float(), mask, *at, 1.0),
           lambda: attn.attn_tree_commit(mask, leaf.long(), *at), lambda: attn.attn_tree_commit(mask, leaf[:1], *at), lambda: attn.attn_tree_commit(mask[:5], leaf, *at),
           lambda: attn.attn_tree_commit(mask, None, *at), lambda: attn.attn_tree_commit(mask, leaf, *at, out=torch.zeros(3, dtype=torch.int32, device="cuda")),
           lambda: attn.attn_cache_weigh(q, lse[:5], *at, 1.0), lambda: attn.attn_cache_weigh(q, lse, *at, 1.0, weight=w[:, :1]),
           lambda: attn.attn_cache_weigh(q, lse, *at, 1.0, weight=w[:, :, :63]), lambda: attn.attn_cache_weigh(q, lse, *at, 1.0, weight=w.double()),
           lambda: attn.attn_cache_weigh(q, lse, *at, 1.0, out=w.transpose(0, 1).contiguous().transpose(0, 1)[:, :, ::2]), lambda: attn.attn_cache_weigh(q, lse, *at, 1.0, weight=w.cpu()),
           lambda: attn.attn_cache_evict(w[:, :, :63], *at, 5), lambda: attn.attn_cache_evict(w, *at, 5, pos=pos.long()), lambda: attn.attn_cache_evict(w, *at, 5, pos=pos[:, :, :60]),
           lambda: attn.attn_cache_evict(w, *at, 5, pos=torch.zeros(2, 2, 65, dtype=torch.int32, device="cuda")), lambda: attn.attn_cache_evict(w, *at, 5, kept=leaf.long()),
           lambda: attn.attn_cache_evict(w, *at, 5, pos=pos, out=(w, None, leaf)), lambda: attn.attn_cache_evict(w, *at, 5, out=(w, pos, None)),
           lambda: attn.attn_cache_evict(w, *at, 5, workspace=torch.zeros(4096, dtype=torch.uint8, device="cuda")[::2])]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, attn.AttnError)):
            call()
            print("not refused:", i)
    with pytest.raises(attn.AttnError):
        attn.attn_tree_commit(mask, leaf, *at, out=t["lens"])
    with pytest.raises(attn.AttnError):
        attn.attn_cache_evict(w, *at, 5, out=(w, None, t["lens"]))
    with pytest.raises(attn.AttnError):
        attn.attn_cache_evict(w, *at, 5, first=3, recent=3)
