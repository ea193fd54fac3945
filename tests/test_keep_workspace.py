"""A workspace of 256 bytes says that a call on trees, weights or eviction keeps nothing there, and the binding then passes none: wherever a call shares its work out
over sums, or lists the tokens that move, its size has to be larger."""
import ctypes
import random
import shutil

import pytest

from paper_2410_09397_amd import attn
from tests.test_keep_rules import _tree, _weigh, lib  # noqa: F401 (the fixture)
from tests.test_window_abi import paged

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


def _desc(bf16, fp8, batch, heads, kv_heads, d, total, max_q, max_len, window=0, sinks=0):
    page, width = 16, -(-max_len // 16)
    return paged(batch=batch, heads=heads, kv_heads=kv_heads, d=d, total_q=total, max_q=max_q, max_len=max_len, page_size=page, num_pages=batch * width,
                 max_pages=width, table_stride=width, window=window, sinks=sinks, dtype=attn.ATTN_BF16 if bf16 else attn.ATTN_F32,
                 kind=attn.ATTN_CACHE_FP8 if fp8 else attn.ATTN_CACHE_PLAIN, q_stride_n=heads * d, q_stride_h=d, kv_stride_n=kv_heads * d, kv_stride_h=d,
                 page_stride_p=kv_heads * page * d, page_stride_h=page * d, page_stride_n=d)


def _check_weigh(lib, bf16, fp8, batch, heads, kv_heads, d, max_q, max_len):
    desc = _desc(bf16, fp8, batch, heads, kv_heads, d, batch * max_q, max_q, max_len)
    parts = _weigh(lib, bf16, fp8, batch, heads, kv_heads, d, max_q, max_len, heads * d, d)[3]
    size = attn.lib().attn_weigh_workspace_bytes(ctypes.byref(desc))
    assert size >= 256 and (size > 256) == (parts > 1) and (parts == 1 or size >= 4 * parts * batch * kv_heads * max_len)
    return parts > 1


@pytest.mark.parametrize("heads,max_q,max_len", [(32, 13, 16), (32, 16, 16), (16, 32, 32), (64, 16, 16)])
def test_sums_of_few_slots(lib, heads, max_q, max_len):  # noqa: F811
    assert _check_weigh(lib, 1, 0, 1, heads, 1, 128, max_q, max_len)


def test_a_workspace_that_is_used_is_larger_than_256_bytes(lib):  # noqa: F811
    rng, split = random.Random(1), 0
    for _ in range(3000):
        bf16, fp8 = rng.choice([(1, 0), (1, 1), (0, 0), (0, 1)])
        batch, kv_heads, group, d = rng.choice([1, 1, 2, 5]), rng.choice([1, 1, 2, 8]), rng.choice([1, 2, 8, 16, 64]), rng.choice([64, 128, 256])
        max_q, max_len = rng.choice([1, 5, 16, 33, 100, 1000]), rng.choice([1, 8, 16, 33, 64, 300, 5000])
        split += _check_weigh(lib, bf16, fp8, batch, kv_heads * group, kv_heads, d, max_q, max_len)
        places = _tree(lib, bf16, fp8, batch, kv_heads * group, kv_heads, d, batch * max_q, max_q, max_len, 0, 0)[3]
        desc = _desc(bf16, fp8, batch, kv_heads * group, kv_heads, d, batch * max_q, max_q, max_len)
        assert (attn.lib().attn_tree_workspace_bytes(ctypes.byref(desc)) > 256) == (places > 0)
        budget = rng.randint(1, max_len)
        assert (attn.lib().attn_evict_workspace_bytes(ctypes.byref(desc), budget) > 256) == (min(budget, max_len - budget) > lib.here())
    assert split > 300


@pytest.mark.gpu
@pytest.mark.parametrize("heads,new", [(32, 13), (32, 16), (16, 32), (64, 16)])
def test_weights_of_few_slots(heads, new):
    from tests.test_gpu_evict import _weigh_case
    print("case weigh few slots", heads, new, flush=True)
    _weigh_case("bf16", "plain", [new], [new], heads, 1, 128, 16)
    _weigh_case("bf16", "fp8", [new], [new], heads, 1, 64, 16, in_place=True)
