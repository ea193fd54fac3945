"""Calls on the far side of the rules that choose a kernel of windowed attention and the paged cache by the size of the call
(csrc/attn_win_rules.hpp): the small cases of the other files take the kernels for few blocks and small calls.  tests/test_window_rules.py holds
on the CPU that each of these takes what it is there for, tests/test_gpu_window_rules.py compares their results with 64 bits."""

# dtype, batch, heads, kv_heads, n, d, window, sinks, lengths; rows of a workgroup (of the bf16 kernels); workgroups of a tile of sinks
# (if there are any) and of another tile of keys
TRAIN = [
    # blocks of 128 rows at every width, whole and padded, with lengths that end inside a tile
    (("bf16", 9, 8, 4, 1403, 64, 200, 5, [1403, 1, 700, 0, 1290, 64, 1402, 333, 129]), (128, 6, 1)),
    (("bf16", 2, 16, 8, 1733, 64, 0, 0, None), (128, 1, 1)),
    (("bf16", 5, 12, 3, 931, 128, 130, 70, [931, 500, 65, 930, 128]), (128, 5, 1)),
    (("bf16", 13, 4, 4, 1000, 256, 300, 3, [1000, 999, 0, 1, 640, 641, 1000, 63, 300, 301, 777, 65, 900]), (128, 3, 1)),
    (("bf16", 4, 9, 3, 1434, 40, 64, 0, [1434, 1000, 33, 1]), (128, 1, 1)),
    (("bf16", 13, 4, 2, 1004, 72, 90, 130, [1000, 999, 0, 1, 640, 641, 1004, 63, 300, 301, 777, 65, 900]), (128, 7, 1)),
    (("bf16", 7, 6, 3, 1250, 200, 0, 0, [1250, 1249, 77, 0, 600, 1000, 1]), (128, 1, 1)),
    # the last call in front of that line and the first beyond it
    (("bf16", 32, 12, 12, 128, 64, 40, 1, [128 - 4 * i for i in range(32)]), (64, 2, 1)),
    (("bf16", 35, 11, 11, 128, 64, 40, 1, [128 - 3 * i for i in range(35)]), (128, 2, 1)),
    # tokens of every key tile shared out over workgroups, with and without sinks
    (("bf16", 1, 8, 1, 1501, 64, 400, 5, [1499]), (64, 16, 4)),
    (("bf16", 1, 8, 2, 1001, 64, 0, 0, None), (64, 5, 5)),
    (("bf16", 1, 6, 1, 1100, 128, 500, 130, [1037]), (64, 8, 4)),
    (("bf16", 1, 8, 1, 1030, 256, 400, 3, [1000]), (64, 12, 4)),
    (("bf16", 2, 6, 1, 900, 256, 0, 0, [900, 513]), (64, 7, 7)),
    (("bf16", 1, 8, 1, 810, 48, 0, 0, [809]), (64, 6, 6)),
    (("bf16", 1, 12, 2, 1010, 96, 300, 66, [1009]), (64, 9, 3)),
    (("bf16", 1, 8, 1, 700, 168, 0, 0, None), (64, 5, 5)),
    (("f32", 1, 6, 1, 611, 80, 200, 3, [600]), (64, 12, 4)),
    (("f32", 2, 4, 2, 500, 144, 0, 0, [500, 33]), (64, 5, 5)),
]

# dtype, kind, lengths, new tokens, heads, kv_heads, d, page size, window, sinks; rows of a workgroup, whether the keys of a block are split
PAGED = [
    # blocks of 128 rows, over pages of values (whole and padded rows) and of codes
    (("bf16", "plain", [900, 1203, 777, 700, 2000, 705], [700, 691, 700, 700, 650, 705], 16, 8, 64, 16, 0, 0), (128, False)),
    (("bf16", "plain", [900, 1203, 777, 700, 2000, 705], [700, 691, 700, 700, 650, 705], 16, 8, 128, 64, 300, 5), (128, False)),
    (("bf16", "plain", [900, 1203, 777, 700, 1000, 705], [700, 691, 700, 700, 650, 705], 16, 8, 256, 16, 130, 70), (128, False)),
    (("bf16", "plain", [900, 1203, 777, 700, 1000, 705], [700, 691, 700, 700, 650, 705], 16, 8, 96, 8, 0, 0), (128, False)),
    (("bf16", "plain", [900, 1203, 777, 700, 1000, 705], [700, 691, 700, 700, 650, 705], 16, 8, 200, 32, 90, 1), (128, False)),
    (("bf16", "fp8", [900, 1203, 777, 700, 2000, 705], [700, 691, 700, 700, 650, 705], 16, 8, 64, 16, 200, 4), (128, False)),
    (("bf16", "fp8", [900, 1203, 777, 700, 2000, 705], [700, 691, 700, 700, 650, 705], 16, 8, 128, 16, 0, 0), (128, False)),
    (("bf16", "fp8", [900, 1203, 777, 700, 1000, 705], [700, 691, 700, 700, 650, 705], 16, 8, 256, 128, 0, 0), (128, False)),
    # 64-row blocks behind a long cache: their keys are split
    (("bf16", "plain", [4507, 3001], [101, 37], 4, 2, 64, 16, 0, 0), (64, True)),
    (("bf16", "plain", [4507, 3001], [101, 37], 4, 2, 128, 64, 2500, 3), (64, True)),
    (("bf16", "plain", [4507, 90], [101, 80], 4, 2, 256, 16, 0, 0), (64, True)),
    (("bf16", "plain", [4507, 3001], [101, 37], 4, 2, 104, 16, 0, 0), (64, True)),
    (("bf16", "fp8", [4507, 3001], [101, 37], 4, 2, 64, 32, 0, 0), (64, True)),
    (("bf16", "fp8", [4507, 20], [101, 37], 4, 2, 128, 16, 0, 0), (64, True)),
    (("bf16", "fp8", [4507, 3001], [101, 37], 4, 2, 256, 16, 3000, 70), (64, True)),
    # 32 rows and fp32 arithmetic, split
    (("bf16", "plain", [3007, 1000], [13, 9], 6, 2, 256, 16, 0, 0), (32, True)),
    (("bf16", "fp8", [3007, 1000], [1, 9], 6, 2, 80, 16, 0, 0), (32, True)),
    (("f32", "plain", [2101, 1000], [40, 9], 6, 2, 72, 16, 0, 0), (32, True)),
]

# dtype, kind, new tokens, kv_heads, d, page size: several rows of the cache to a thread
CACHE = [
    ("bf16", "plain", [4000, 1, 1503], 3, 64, 16), ("bf16", "fp8", [4000, 1, 1503], 3, 64, 16),
    ("bf16", "plain", [2003, 0, 741], 3, 128, 64), ("bf16", "fp8", [2003, 0, 741], 3, 128, 16),
    ("bf16", "plain", [1371], 3, 256, 8), ("bf16", "fp8", [1300, 70], 3, 200, 32),
    ("f32", "plain", [4000, 1499], 3, 33, 16), ("f32", "fp8", [2003, 741], 3, 104, 16),
]
# the last call with one row to a thread and the first with two
CACHE_LINE = [(1024, 16, 64, 1), (1025, 16, 64, 2), (1024, 8, 128, 1), (1025, 8, 128, 2), (512, 8, 256, 1), (513, 8, 256, 2)]
