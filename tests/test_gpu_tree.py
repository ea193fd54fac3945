"""Trees of drafted tokens (attn_tree_mask, attn_tree_fwd, attn_tree_commit) against their definitions in 64 bits.  Masks, moves and lengths are exact;
every value of O has a bound of its own (tests/keep_ref.py), LSE is within the absolute bound of the other paged calls."""
import math
import random

import pytest

from tests import keep_ref
from tests.helpers import LSE_TOL
from tests.test_gpu_paged import DTYPES, Cache
from tests.window_bounds import check

pytestmark = pytest.mark.gpu


def _bits(style, count, rng):
    import torch
    if style == "chain":
        return keep_ref.ancestors(list(range(-1, count - 1)), count)
    if style == "star":
        return keep_ref.ancestors([-1] * count, count)
    if style == "tree":
        return keep_ref.ancestors([rng.randint(-1, t - 1) for t in range(count)], count)
    bits = torch.tensor([[rng.random() < 0.3 for _ in range(count)] for _ in range(count)], dtype=torch.bool).reshape(count, count)
    bits[::5] = False  # rows that see the context alone
    return bits


def _mask(bits, max_q):
    import torch
    rows = [keep_ref.pack(b[:max_q], -(-max_q // 32)) if b.shape[0] else torch.zeros(0, -(-max_q // 32), dtype=torch.int32) for b in bits]
    return torch.cat(rows).cuda()


def _starts(new):
    return [sum(new[:b]) for b in range(len(new) + 1)]


def _check(c, Q, O, LSE, bits, new, dtype, d, window, sinks):
    import torch
    starts, worst = _starts(new), 0.0
    for b, length in enumerate(c.host_lens):
        r = slice(starts[b], starts[b + 1])
        seen = keep_ref.tree_seen(bits[b], length, new[b], window, sinks).cuda()
        none = ~seen.any(1)
        assert bool((LSE[r][none] == -math.inf).all()) and not bool(O[r][none].any())
        for h in range(Q.shape[1]):
            k, v = (x[b][:, h // (Q.shape[1] // x[b].shape[1])] for x in (c.keys, c.values))
            o, lse, bound = keep_ref.attend(Q[r, h].double(), k, v, seen, d ** -0.5, dtype)
            worst = max(worst, check("sequence %d head %d O" % (b, h), O[r, h], o, bound))
            if bool((~none).any()):
                assert float((LSE[r, h].double() - lse)[~none].abs().max()) <= LSE_TOL[dtype] * max(1.0, float(lse[~none].abs().max()))
    print("share of the bound %.2f" % worst, flush=True)


def _case(dtype, kind, lens, new, h, kvh, d, page, window=0, sinks=0, style="tree", layout="phnd", max_len=None, seed=0):
    import torch
    from paper_2410_09397_amd import attn
    rng = random.Random(seed)
    c = Cache(dtype, kind, lens, kvh, d, page, seed=seed, layout=layout)
    bits, starts, max_q = [_bits(style, q, rng) for q in new], _starts(new), max([1] + new)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 100)
    Q = torch.randn(starts[-1], h, d, generator=gen, device="cuda").to(getattr(torch, DTYPES[dtype]))
    kw = dict(q_ptr=torch.tensor(starts, dtype=torch.int32, device="cuda"), max_q=max_q, window=window, sinks=sinks, max_len=max_len, **c.exps())
    mask = _mask(bits, max_q)
    O, LSE = attn.attn_tree_fwd(Q, mask, *c.args(), d ** -0.5, **kw)
    _check(c, Q, O, LSE, bits, new, dtype, d, window, sinks)
    again = attn.attn_tree_fwd(Q, mask, *c.args(), d ** -0.5, **kw)
    assert torch.equal(O, again[0]) and torch.equal(LSE, again[1])
    return c, Q, mask, kw, O, LSE


CASES = [
    # dtype, kind, lens, new tokens, heads, kv heads, d, page, window, sinks, style
    ("bf16", "plain", [1], [1], 1, 1, 64, 16, 0, 0, "tree"),
    ("bf16", "fp8", [5, 1, 0, 40], [3, 1, 0, 40], 4, 2, 128, 16, 0, 0, "tree"),             # no context; nothing at all
    ("bf16", "plain", [17, 600, 64, 333], [4, 4, 4, 3], 8, 2, 64, 16, 0, 0, "star"),         # 16 rows
    ("bf16", "fp8", [17, 600, 64, 333], [4, 2, 1, 3], 16, 4, 128, 32, 0, 0, "tree"),
    ("bf16", "fp8", [5000, 300, 2000], [4, 2, 3], 8, 2, 128, 16, 0, 0, "tree"),              # the same, shared out over workgroups
    ("bf16", "plain", [2500, 40], [3, 4], 8, 2, 64, 16, 0, 0, "bits"),
    ("bf16", "plain", [3000, 1700], [5, 1], 3, 1, 256, 16, 200, 3, "tree"),
    ("bf16", "plain", [130, 900], [9, 13], 8, 2, 128, 64, 0, 0, "tree"),                     # 32 rows
    ("bf16", "fp8", [5000], [15], 4, 1, 128, 16, 0, 0, "bits"),                              # shared out over workgroups
    ("bf16", "plain", [3000, 30], [31, 30], 10, 5, 256, 128, 0, 0, "tree"),
    ("bf16", "fp8", [700, 431], [64, 33], 8, 2, 128, 16, 0, 0, "tree"),                      # 128 rows
    ("bf16", "plain", [2100, 100], [64, 64], 16, 1, 64, 16, 0, 0, "bits"),
    ("bf16", "fp8", [400] * 24, [64] * 24, 32, 8, 64, 16, 0, 0, "tree"),                     # blocks for all places of the chip
    ("bf16", "plain", [300, 299], [65, 100], 4, 2, 256, 16, 0, 0, "bits"),
    ("bf16", "fp8", [300, 200], [100, 200], 4, 2, 256, 256, 0, 0, "chain"),
    ("bf16", "plain", [400], [90], 15, 3, 96, 16, 0, 0, "tree"),                             # padded widths
    ("bf16", "plain", [400, 33], [7, 2], 6, 3, 200, 16, 0, 0, "bits"),
    ("bf16", "plain", [400, 33], [3, 2], 6, 3, 24, 16, 5, 2, "tree"),
    ("bf16", "plain", [4100, 2000, 100], [5, 3, 1], 8, 2, 128, 16, 100, 4, "tree"),          # windows that end in the context
    ("bf16", "fp8", [4100, 2000, 100], [40, 64, 64], 8, 2, 128, 16, 3, 70, "chain"),         # among the drafted tokens
    ("bf16", "fp8", [150, 64, 90, 3], [37, 64, 1, 3], 6, 2, 64, 64, 20, 65, "bits"),         # sinks that reach into them
    ("bf16", "plain", [900, 40], [70, 40], 4, 2, 256, 8, 1, 0, "tree"),
    ("bf16", "fp8", [2000, 50], [1, 7], 4, 2, 72, 16, 0, 0, "tree"),                         # 32-bit arithmetic
    ("bf16", "fp8", [200, 50], [33, 7], 4, 2, 248, 16, 10, 3, "bits"),
    ("f32", "plain", [1, 40, 2100], [1, 13, 2], 6, 3, 40, 8, 0, 0, "tree"),
    ("f32", "plain", [77, 500], [77, 1], 2, 1, 33, 16, 20, 2, "tree"),
    ("f32", "plain", [300], [100], 4, 1, 256, 16, 0, 0, "bits"),
    ("f32", "fp8", [130, 500], [1, 60], 4, 1, 128, 4096, 7, 1, "chain"),
]


@pytest.mark.parametrize("case", CASES)
def test_attention_of_trees(case):
    print("case tree", *case, flush=True)
    _case(*case)


@pytest.mark.parametrize("seed", range(16))
def test_attention_of_trees_of_random_sizes(seed):
    rng = random.Random(seed)
    for _ in range(3):
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        kind, kvh = rng.choice(["plain", "fp8"]), rng.choice([1, 2, 3, 5])
        h, b = kvh * rng.choice([1, 2, 3, 4, 8, 17]), rng.choice([1, 2, 3, 7])
        most = rng.choice([2, 7, 30, 150])
        new = [rng.randint(0, most) for _ in range(b)]
        lens = [max(q - rng.choice([0, 0, 0, 2]), 0) + rng.choice([0, rng.randint(0, 60), rng.randint(0, 2500)]) for q in new]
        d = rng.choice([64, 128, 256, 8 * rng.randint(1, 32)]) if dtype == "bf16" or kind == "fp8" else rng.randint(1, 256)
        window = rng.choice([0, 0, rng.randint(1, 8), rng.randint(1, 1000)])
        case = (dtype, kind, lens, new, h, kvh, d, 8 << rng.randint(0, 5), window, rng.choice([0, 1, 4, 70]), rng.choice(["tree", "bits", "chain"]))
        if sum(new) == 0:
            continue
        print("case tree", seed, *case, flush=True)
        _case(*case, seed=seed)


def test_new_tokens_in_front_of_slot_0_are_no_keys():
    print("case tree in front", flush=True)
    for style in ("tree", "bits", "chain"):
        _case("bf16", "plain", [3, 0, 70], [9, 4, 100], 4, 2, 128, 16, style=style)
        _case("bf16", "fp8", [3, 40, 70], [40, 41, 100], 4, 2, 64, 16, window=3, sinks=1, style=style)
        _case("f32", "plain", [3, 0], [5, 1], 2, 2, 24, 16, style=style)


@pytest.mark.parametrize("d,kind", [(128, "fp8"), (64, "plain"), (40, "fp8")])
def test_the_longest_trees_and_chains(d, kind):
    print("case longest trees", d, kind, flush=True)
    _case("bf16", kind, [1500, 1024], [1024, 1024], 2, 1, d, 64, style="chain")
    _case("bf16", kind, [1500, 1024], [1000, 1024], 2, 1, d, 64, window=300, sinks=2, style="bits")


@pytest.mark.parametrize("kind", ["plain", "fp8"])
def test_token_major_pages_and_a_tight_bound_on_the_lengths(kind):
    print("case tree layout", kind, flush=True)
    for d in (64, 128, 80):
        _case("bf16", kind, [300, 77, 1000], [3, 20, 40], 4, 2, d, 16, layout="pnhd", max_len=1000)


def test_batches_of_more_than_64_sequences():
    """Sequences are counted 64 at a time; some have no drafted token, and where there are many the work is not shared out."""
    print("case tree many sequences", flush=True)
    lens = [1 + (37 * i) % 300 for i in range(150)]
    new = [min(l, (0, 1, 0, 3, 40, 1)[i % 6]) for i, l in enumerate(lens)]
    _case("bf16", "fp8", lens, new, 4, 1, 64, 16)
    _case("bf16", "plain", [l + 2000 for l in lens], new, 4, 1, 64, 16, window=50, sinks=3)
    _case("bf16", "plain", [l + 1500 for l in lens], [2] * 150, 4, 1, 128, 16)
    _case("bf16", "plain", [40 + (37 * i) % 100 for i in range(1100)], [(0, 2, 20)[i % 3] for i in range(1100)], 8, 4, 64, 16)
    _case("f32", "plain", [40 + (37 * i) % 100 for i in range(1100)], [(0, 2)[i % 2] for i in range(1100)], 8, 4, 24, 16)


def test_a_chain_sees_what_new_tokens_in_order_see():
    """attn_tree_fwd with the mask of a chain against attn_paged_fwd: both within their bounds of the same values."""
    import torch
    from paper_2410_09397_amd import attn
    print("case chain", flush=True)
    c, Q, mask, kw, O, LSE = _case("bf16", "plain", [700, 130, 40], [30, 130, 1], 6, 2, 128, 16, window=50, sinks=3, style="chain")
    o, lse = attn.attn_paged_fwd(Q, *c.args(), 128 ** -0.5, **kw)
    top = max(float(v.abs().max()) for v in c.values)  # each side is off by at most 2^-8 of |O| and of the weighted |V|, and some 2^-24
    assert float((O.float() - o.float()).abs().max()) <= 2.02 * 2.0 ** -8 * 2 * top
    assert float((LSE - lse).abs().max()) <= 2 * LSE_TOL["bf16"]


@pytest.mark.parametrize("kind,d", [("plain", 64), ("fp8", 128), ("plain", 96), ("fp8", 256), ("fp8", 72)])
@pytest.mark.parametrize("new", [3, 50])
def test_pages_behind_the_window_may_be_gone(kind, d, new):
    import torch
    from paper_2410_09397_amd import attn
    print("case tree pages gone", kind, d, new, flush=True)
    window, page, lens = 100, 16, [900, 300, 5000, 120]
    c, Q, mask, kw, O, LSE = _case("bf16", kind, lens, [new] * 4, 4, 2, d, page, window, 4)
    for b, l in enumerate(lens):
        for x in range(1, max(0, l - new - window) // page):  # (the last `window` tokens of the context are read)
            gone = int(c.table[b, x])
            c.table[b, x] = [-1, 10 ** 9, -(10 ** 9)][x % 3]
            for pages, exps in ((c.K, c.K_exp), (c.V, c.V_exp)):
                if exps is None:
                    pages[gone] = math.nan
                else:
                    pages.view(torch.uint8)[gone] = 0x7f
                    exps[gone] = 255
    again = attn.attn_tree_fwd(Q, mask, *c.args(), d ** -0.5, **kw)
    assert torch.equal(again[0], O) and torch.equal(again[1], LSE)


def test_rows_of_no_sequence_are_left_alone():
    import torch
    from paper_2410_09397_amd import attn
    print("case tree gaps in the rows", flush=True)
    c = Cache("bf16", "plain", [40, 70], 2, 128, 16)
    Q = torch.randn(10, 4, 128, device="cuda").to(torch.bfloat16)
    ptr = torch.tensor([2, 3, 9], dtype=torch.int32, device="cuda")  # rows 0, 1 and 9 belong to nobody; max_q cuts the second sequence
    parents = torch.tensor([5, 5, -1, -1, 0, 0, 1, 2, 0, 9], dtype=torch.int32, device="cuda")
    mask = torch.full((10, 3), -7, dtype=torch.int32, device="cuda")
    attn.attn_tree_mask(parents, 4, q_ptr=ptr, out=mask)
    assert mask.tolist() == [[-7] * 3] * 2 + [[x, -7, -7] for x in (1, 1, 3, 5, 11)] + [[-7] * 3] * 3  # (words behind the rows' own too)
    O, LSE = torch.full_like(Q, 7.0), torch.full((10, 4), 7.0, device="cuda")
    attn.attn_tree_fwd(Q, mask, *c.args(), 0.1, q_ptr=ptr, max_q=4, out=(O, LSE))
    assert bool((O[[0, 1, 7, 8, 9]] == 7.0).all()) and bool((LSE[[0, 1, 7, 8, 9]] == 7.0).all())
    seen = torch.zeros(4, 70, dtype=torch.bool)
    seen[:, :64] = True
    for t, row in enumerate(([0], [0, 1], [0, 2], [0, 1, 3])):
        seen[t, [64 + u for u in row]] = True
    for h in range(4):
        o, _, bound = keep_ref.attend(Q[3:7, h].double(), c.keys[1][:, h // 2], c.values[1][:, h // 2], seen.cuda(), 0.1, "bf16")
        check("head %d" % h, O[3:7, h], o, bound)


@pytest.mark.parametrize("kind,d", [("plain", 64), ("fp8", 128), ("fp8", 72)])
def test_rows_of_several_sequences(kind, d):
    """q_ptr has to ascend.  One that does not, and gives a row to several sequences, makes more parts than the workspace has places: what comes out is one
    sequence's or the other's, or nothing of a row's, but nothing else is written and what is behind the workspace is not read."""
    import torch
    from paper_2410_09397_amd import attn
    print("case tree rows of several sequences", kind, d, flush=True)
    lens, rows, batch = [3000] * 6, 200, 6
    c = Cache("bf16", kind, lens, 2, d, 64)
    Q = torch.randn(rows, 4, d, device="cuda").to(torch.bfloat16)
    ptr = torch.tensor([0, rows, 0, rows, 0, rows, 0], dtype=torch.int32, device="cuda")
    mask = _mask([_bits("chain", rows, random.Random(0))], rows)
    kw = dict(q_ptr=ptr, max_q=rows, **c.exps())
    exps = c.exps()
    desc, _ = attn._paged("attn_tree_fwd", Q, *c.args(), ptr, rows, None, exps.get("K_exp"), exps.get("V_exp"), False, 0.1, 0, 0)
    size = attn.attn_tree_workspace_bytes(desc)
    assert size > 256
    workspace = torch.zeros(size + 4096, dtype=torch.uint8, device="cuda")
    out = torch.full((rows + 2, 4, d), 7.0, device="cuda", dtype=torch.bfloat16), torch.full((rows + 2, 4), 7.0, device="cuda")
    attn.attn_tree_fwd(Q, mask, *c.args(), 0.1, out=(out[0][1:-1], out[1][1:-1]), workspace=workspace[:size], **kw)
    for x in out:
        assert bool((x[0] == 7.0).all()) and bool((x[-1] == 7.0).all())
    assert not bool(workspace[size:].any())


@pytest.mark.parametrize("counts,max_q", [([1], 1), ([0, 5, 31, 32, 33], 33), ([64] * 70, 64), ([1024, 1000, 3], 1024), ([300], 512)])
def test_masks_of_parents(counts, max_q):
    import torch
    from paper_2410_09397_amd import attn
    print("case masks", counts, max_q, flush=True)
    rng = random.Random(max_q)
    parents = [[rng.choice([t - 1, rng.randint(-1, t - 1), rng.randint(-1, t - 1)]) for t in range(q)] for q in counts]
    if counts[-1] == 3:
        parents[-1] = [0, 1, 2]                      # themselves: they follow the context
    if len(parents[0]) > 40:
        parents[0][20], parents[0][30], parents[0][35] = 21, 10 ** 9, -(2 ** 31)  # no earlier tokens
    want = torch.cat([keep_ref.pack(keep_ref.ancestors(p, len(p)), -(-max_q // 32)) for p in parents])
    flat = torch.tensor([x for p in parents for x in p], dtype=torch.int32, device="cuda")
    got = attn.attn_tree_mask(flat, max_q, q_ptr=torch.tensor(_starts(counts), dtype=torch.int32, device="cuda"))
    assert torch.equal(got.cpu(), want)
    if len(set(counts)) == 1 and counts[0] == max_q:
        assert torch.equal(attn.attn_tree_mask(flat, max_q).cpu(), want)


def _raw(x):
    import torch
    return x.view(torch.uint8) if x.dtype is torch.float8_e4m3fn else x.view(torch.int16 if x.dtype is torch.bfloat16 else torch.int32) if x.dtype.is_floating_point else x


@pytest.mark.parametrize("dtype,kind,d,page,layout", [("bf16", "plain", 64, 16, "phnd"), ("bf16", "fp8", 128, 16, "pnhd"), ("bf16", "fp8", 72, 8, "phnd"),
                                                      ("f32", "plain", 33, 16, "pnhd"), ("f32", "plain", 256, 32, "phnd"), ("f32", "plain", 255, 64, "phnd"),
                                                      ("bf16", "plain", 40, 16, "pnhd"), ("f32", "fp8", 104, 4096, "phnd"), ("bf16", "fp8", 256, 64, "phnd")])
def test_committing(dtype, kind, d, page, layout):
    """What stays, in its order; everything else in the pages as it was, bit for bit."""
    import torch
    from paper_2410_09397_amd import attn
    print("case commit", dtype, kind, d, page, layout, flush=True)
    rng = random.Random(d)
    new = [5, 64, 1, 33, 0, 300, 20, 9, 9]
    lens = [100, 64, 1, 300, 7, 333, 12, 50, 60]  # the second has no context; of the seventh the first 8 have no slot
    leaf = [4, 63, 0, -1, 0, 299, 19, 9, 2 ** 31 - 1]
    bits = [_bits(s, q, rng) for s, q in zip(["tree", "chain", "tree", "tree", "tree", "bits", "bits", "tree", "tree"], new)]
    bits[5][299, 200:] = True
    c = Cache(dtype, kind, lens, 3, d, page, layout=layout, seed=5)
    if kind == "fp8":
        for e in (c.K_exp, c.V_exp):
            e.copy_(torch.randint(100, 140, e.shape, device="cuda"))
    gone = (lens[0] - new[0]) // page if page < 100 else None  # a page of the first sequence's drafted tokens
    table = c.table.cpu()
    if gone is not None:
        c.table[0, gone] = -1
    arrays = [x for x in (c.K, c.V, c.K_exp, c.V_exp) if x is not None]
    want = [_raw(x).clone() for x in arrays]
    lengths = []
    for b in range(len(new)):
        first = lens[b] - new[b]
        stay = [u for u in range(new[b]) if 0 <= leaf[b] < new[b] and bits[b][leaf[b], u] and first + u >= 0]
        lengths.append(max(first, 0) + len(stay))
        for x, at in enumerate(stay):
            source, target = first + at, max(first, 0) + x
            if b == 0 and gone is not None and gone in (source // page, target // page):
                continue
            for w, a in zip(want, arrays):
                w[int(table[b, target // page]), :, target % page] = _raw(a)[int(table[b, source // page]), :, source % page]
    got = attn.attn_tree_commit(_mask(bits, 300), torch.tensor(leaf, dtype=torch.int32, device="cuda"), *c.args(),
                                q_ptr=torch.tensor(_starts(new), dtype=torch.int32, device="cuda"), max_q=300, **c.exps())
    assert got.tolist() == lengths
    for a, w in zip(arrays, want):
        assert torch.equal(_raw(a), w)


def test_committing_a_thousand_tokens_that_move_by_one():
    """Every row is overwritten by the next one: rows are read before they are overwritten."""
    import torch
    from paper_2410_09397_amd import attn
    print("case commit overlap", flush=True)
    for d, dt in ((256, torch.float32), (64, torch.bfloat16)):
        K, V = (torch.randn(40, 2, 32, d, device="cuda").to(dt) for _ in range(2))
        table = torch.randperm(40)[:33][None].to(device="cuda", dtype=torch.int32)
        lens = torch.tensor([1030], dtype=torch.int32, device="cuda")
        bits = torch.zeros(1024, 1024, dtype=torch.bool)
        bits[1023, 1:] = True
        rows = [x[table[0].long()].permute(1, 0, 2, 3).flatten(1, 2).clone() for x in (K, V)]
        got = attn.attn_tree_commit(_mask([bits], 1024), torch.tensor([1023], dtype=torch.int32, device="cuda"), K, V, table, lens)
        assert got.tolist() == [1029]
        for x, was in zip((K, V), rows):
            now = x[table[0].long()].permute(1, 0, 2, 3).flatten(1, 2)
            assert torch.equal(now[:, :6], was[:, :6]) and torch.equal(now[:, 6:1029], was[:, 7:1030]) and torch.equal(now[:, 1029:], was[:, 1029:])


@pytest.mark.parametrize("kind", ["plain", "fp8"])
def test_queries_that_are_a_view(kind):
    """Queries of a fused projection, with gaps between their rows: the result has their strides, the gaps are left alone."""
    import torch
    from paper_2410_09397_amd import attn
    print("case tree views", kind, flush=True)
    c = Cache("bf16", kind, [60, 200], 2, 64, 16)
    fused = torch.randn(12, 8, 64, device="cuda").to(torch.bfloat16)
    mask = attn.attn_tree_mask(torch.tensor([-1, 0, 0, 1, 1, 2] * 2, dtype=torch.int32, device="cuda"), 6)
    view, plain = fused[:, :4], fused[:, :4].contiguous()
    O, LSE = attn.attn_tree_fwd(view, mask, *c.args(), 0.125, **c.exps())
    o, lse = attn.attn_tree_fwd(plain, mask, *c.args(), 0.125, **c.exps())
    assert O.stride() == view.stride() and torch.equal(O, o) and torch.equal(LSE, lse)


def test_offsets_beyond_32_bits():
    import torch
    from paper_2410_09397_amd import attn
    kvh, page, n, d = 8, 64, 300, 128
    num = (1 << 32) // (kvh * page * d) + 100
    for kind in ("plain", "fp8"):
        print("case tree large cache", kind, flush=True)
        small = Cache("bf16", kind, [n], kvh, d, page, spare=0)
        used = small.K.shape[0]
        K, V = (torch.empty(num, kvh, page, d, dtype=small.K.dtype, device="cuda") for _ in range(2))
        _raw(K)[-used:], _raw(V)[-used:] = _raw(small.K), _raw(small.V)
        exps = {}
        if kind == "fp8":
            exps = {x: torch.empty(num, kvh, page, dtype=torch.uint8, device="cuda") for x in ("K_exp", "V_exp")}
            for x in exps:
                exps[x][-used:] = small.exps()[x]
        table = small.table + (num - used)
        for new in (3, 60):
            Q = torch.randn(new, 16, d, device="cuda").to(torch.bfloat16)
            mask = _mask([_bits("tree", new, random.Random(new))], new)
            far = attn.attn_tree_fwd(Q, mask, K, V, table, small.lens, 0.1, **exps)
            near = attn.attn_tree_fwd(Q, mask, *small.args(), 0.1, **small.exps())
            assert torch.equal(far[0], near[0]) and torch.equal(far[1], near[1])
        leaf = torch.tensor([57], dtype=torch.int32, device="cuda")
        a = attn.attn_tree_commit(mask, leaf, K, V, table, small.lens, **exps)
        b = attn.attn_tree_commit(mask, leaf, *small.args(), **small.exps())
        assert torch.equal(a, b)
        for x, y in ((K, small.K), (V, small.V)):
            assert torch.equal(_raw(x)[-used:], _raw(y))
        del K, V, far, exps


def test_calls_without_work():
    import torch
    from paper_2410_09397_amd import attn
    c = Cache("bf16", "plain", [5, 9], 2, 64, 16)
    x, none = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(0, 0, dtype=torch.int32, device="cuda")
    leaf = torch.zeros(2, dtype=torch.int32, device="cuda")
    assert attn.attn_tree_mask(none[:, 0] if none.shape[1] else none.flatten(), 0).shape == (0, 0)
    assert attn.attn_tree_fwd(x, none, *c.args(), 1.0)[0].shape == x.shape
    assert attn.attn_tree_commit(none, leaf, *c.args()).tolist() == [5, 9]
    out = torch.zeros_like(leaf)
    assert attn.attn_tree_commit(none, leaf, *c.args(), out=out) is out and out.tolist() == [5, 9]
