"""Attention weights of cached tokens (attn_cache_weigh) and eviction by them (attn_cache_evict) against their definitions in 64 bits: every weight has a
bound of its own (tests/keep_ref.py), what stays, moves and is left is exact."""
import math
import random

import pytest

from tests import keep_ref
from tests.helpers import LSE_TOL
from tests.test_gpu_paged import DTYPES, Cache
from tests.test_gpu_tree import _raw, _starts
from tests.window_bounds import F, check

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------------------- weights
def _weigh_case(dtype, kind, lens, new, h, kvh, d, page, window=0, sinks=0, layout="phnd", max_len=None, old=True, in_place=False, seed=0, max_q=None,
                scale=None):
    import torch
    from paper_2410_09397_amd import attn
    c = Cache(dtype, kind, lens, kvh, d, page, seed=seed, layout=layout)
    starts, c_scale = _starts(new), d ** -0.5 if scale is None else scale
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 100)
    Q = torch.randn(starts[-1], h, d, generator=gen, device="cuda").to(getattr(torch, DTYPES[dtype]))
    kw = dict(q_ptr=torch.tensor(starts, dtype=torch.int32, device="cuda"), max_q=max([1] + new) if max_q is None else max_q, window=window, sinks=sinks,
              max_len=max_len, **c.exps())
    LSE = attn.attn_paged_fwd(Q, *c.args(), c_scale, **kw)[1]
    if starts[-1] > 2:
        LSE[1, 0] = -math.inf  # a query that adds nothing
    slots = c.table.shape[1] * page if max_len is None else max_len
    weight = torch.rand(len(lens), kvh, slots + 3, generator=gen, device="cuda") if old else None
    if old:
        for b, l in enumerate(lens):
            weight[b, :, max(0, l - new[b]):] = math.nan  # not read
    was = weight.clone() if old else None
    out = weight if in_place else torch.full((len(lens), kvh, slots + 7), 9.0, device="cuda")[:, :, 2:]
    kept = out.clone()
    got = attn.attn_cache_weigh(Q, LSE, *c.args(), c_scale, weight=weight, decay=0.75, out=out, **kw)
    assert got is out
    worst = 0.0
    for b, l in enumerate(lens):
        assert torch.equal(out[b, :, l:].nan_to_num(5.0), kept[b, :, l:].nan_to_num(5.0))
        first = l - new[b]
        rows = slice(starts[b], starts[b] + min(new[b], kw["max_q"]))
        for z in range(kvh):
            want, bound = torch.zeros(l, dtype=torch.float64, device="cuda"), torch.zeros(l, dtype=torch.float64, device="cuda")
            for y in range(z * (h // kvh), (z + 1) * (h // kvh)):
                w, e = keep_ref.weigh(Q[rows, y].double(), c.keys[b][:, z], LSE[rows, y].double(), first, c_scale, window, sinks)
                want, bound = want + w, bound + e
            bound += h // kvh * F * want
            if old and first > 0:
                want[:first] += 0.75 * was[b, z, :first].double()
                bound[:first] += 2 * F * want[:first]
            worst = max(worst, check("sequence %d key head %d" % (b, z), out[b, z, :l], want, bound))
    print("share of the bound %.2f" % worst, flush=True)
    return c, Q, LSE, kw, out


WEIGH = [
    # dtype, kind, lens, new tokens, heads, kv heads, d, page, window, sinks
    ("bf16", "plain", [1], [1], 1, 1, 64, 16, 0, 0),
    ("bf16", "fp8", [5, 1, 0], [1, 1, 0], 4, 2, 128, 16, 0, 0),
    ("bf16", "plain", [17, 600, 64, 333], [1, 1, 1, 1], 8, 2, 64, 16, 0, 0),
    ("bf16", "fp8", [130, 900], [1, 1], 40, 1, 128, 64, 0, 0),
    ("bf16", "fp8", [9000, 30, 700], [1, 0, 1], 8, 2, 128, 16, 0, 0),                  # a sequence without new tokens
    ("bf16", "plain", [4100, 2000, 100], [1, 1, 1], 8, 2, 128, 16, 100, 4),
    ("bf16", "fp8", [700, 431], [300, 431], 6, 2, 64, 16, 0, 0),
    ("bf16", "plain", [1300], [1300], 4, 1, 128, 16, 0, 0),                            # a whole prompt
    ("bf16", "plain", [5000, 257], [33, 257], 8, 2, 128, 16, 0, 0),
    ("bf16", "plain", [1500, 64, 900, 3], [37, 64, 1, 3], 8, 2, 128, 16, 130, 5),
    ("bf16", "fp8", [1500, 64, 900, 3], [700, 64, 1, 3], 6, 2, 128, 64, 130, 65),
    ("bf16", "fp8", [300, 200], [100, 200], 4, 2, 256, 256, 50, 3),
    ("bf16", "plain", [300, 1111], [100, 200], 8, 2, 256, 16, 0, 0),
    ("bf16", "plain", [90, 40], [5, 2], 260, 2, 64, 16, 0, 0),                         # groups of more heads than a tile has rows
    ("bf16", "fp8", [300, 40], [33, 40], 34, 2, 128, 16, 20, 2),                       # tiles of 7 tokens of 17 heads
    ("bf16", "plain", [700, 128, 129], [32, 32, 16], 8, 2, 256, 16, 0, 0),             # a tile that is full
    ("bf16", "plain", [400], [90], 15, 3, 96, 16, 60, 3),
    ("bf16", "plain", [400, 90], [1, 70], 6, 3, 200, 16, 0, 0),
    ("bf16", "fp8", [2000, 50], [1, 7], 4, 2, 72, 16, 0, 0),
    ("f32", "plain", [1, 40, 2100], [1, 13, 2], 6, 3, 40, 8, 0, 0),
    ("f32", "plain", [77, 500], [77, 1], 2, 1, 33, 16, 20, 2),
    ("f32", "plain", [77, 300], [77, 1], 4, 1, 250, 16, 0, 0),
    ("f32", "fp8", [130, 500], [1, 60], 4, 1, 128, 4096, 0, 0),
]


@pytest.mark.parametrize("case", WEIGH)
def test_weights(case):
    print("case weigh", *case, flush=True)
    _weigh_case(*case)
    _weigh_case(*case, old=False)
    _weigh_case(*case, in_place=True)


@pytest.mark.parametrize("seed", range(16))
def test_weights_of_random_sizes(seed):
    rng = random.Random(seed)
    for _ in range(3):
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        kind, kvh = rng.choice(["plain", "fp8"]), rng.choice([1, 2, 3, 5])
        h, b = kvh * rng.choice([1, 2, 3, 4, 8, 17]), rng.choice([1, 2, 3, 7])
        most = rng.choice([1, 1, 3, 20, 200, 900])
        new = [rng.randint(0, most) for _ in range(b)]
        lens = [max(0, q - rng.choice([0, 0, 0, 2])) + rng.choice([0, rng.randint(0, 60), rng.randint(0, 2500)]) for q in new]
        d = rng.choice([64, 128, 256, 8 * rng.randint(1, 32)]) if dtype == "bf16" or kind == "fp8" else rng.randint(1, 256)
        window = rng.choice([0, 0, rng.randint(1, 64), rng.randint(1, 1000)])
        case = (dtype, kind, lens, new, h, kvh, d, 8 << rng.randint(0, 5), window, rng.choice([0, 1, 4, 70]))
        print("case weigh", seed, *case, flush=True)
        _weigh_case(*case, seed=seed, layout=rng.choice(["phnd", "pnhd"]), old=rng.random() < 0.5, scale=rng.choice([None, None, -0.1, 0.0]))


@pytest.mark.parametrize("kind,d", [("fp8", 128), ("plain", 40)])
def test_weights_of_more_than_64_sequences(kind, d):
    print("case weigh many sequences", kind, d, flush=True)
    lens = [(37 * i) % 700 for i in range(90)]
    _weigh_case("bf16", kind, lens, [min(l, 1) for l in lens], 4, 2, d, 16)
    _weigh_case("bf16", kind, lens, [min(l, (0, 20, 3)[i % 3]) for i, l in enumerate(lens)], 4, 2, d, 16)
    _weigh_case("bf16", kind, lens, [min(l, (0, 200, 3)[i % 3]) for i, l in enumerate(lens)], 4, 2, d, 16)


def test_a_tight_bound_on_the_lengths_and_a_cut_number_of_new_tokens():
    print("case weigh bounds", flush=True)
    _weigh_case("bf16", "plain", [300, 77, 1000], [30, 7, 100], 4, 2, 128, 16, max_len=1000)
    _weigh_case("bf16", "fp8", [300, 77, 1000], [30, 7, 100], 4, 2, 128, 16, max_q=20)


@pytest.mark.parametrize("kind,d", [("plain", 64), ("fp8", 128), ("plain", 96), ("fp8", 72)])
@pytest.mark.parametrize("new", [1, 50])
def test_weights_of_pages_behind_the_window(kind, d, new):
    """Tokens that nobody sees keep decay times their weight; their pages may be gone."""
    import torch
    from paper_2410_09397_amd import attn
    print("case weigh pages gone", kind, d, new, flush=True)
    page, lens = 16, [900, 300, 5000, 120]
    c, Q, LSE, kw, out = _weigh_case("bf16", kind, lens, [new] * 4, 4, 2, d, page, 100, 4, old=False)
    for b, l in enumerate(lens):
        for x in range(1, max(0, l - new - 100 + 1) // page):
            gone = int(c.table[b, x])
            c.table[b, x] = [-1, 10 ** 9, -(10 ** 9)][x % 3]
            for pages, exps in ((c.K, c.K_exp), (c.V, c.V_exp)):
                if exps is None:
                    pages[gone] = math.nan
                else:
                    pages.view(torch.uint8)[gone] = 0x7f
                    exps[gone] = 255
    again = attn.attn_cache_weigh(Q, LSE, *c.args(), d ** -0.5, out=torch.full_like(out, 9.0), **kw)
    assert torch.equal(again, out)


@pytest.mark.parametrize("dtype,kind,d,new,h", [("bf16", "plain", 64, 3, 4), ("bf16", "fp8", 128, 20, 4), ("bf16", "plain", 128, 150, 4), ("bf16", "plain", 64, 3, 260),
                                                ("f32", "plain", 40, 3, 4), ("f32", "plain", 64, 50, 4), ("bf16", "fp8", 72, 20, 4)])
def test_queries_without_an_lse_add_nothing(dtype, kind, d, new, h):
    """LSE = -inf: a query that adds nothing, also where its Q holds NaN; the others' weights are as without it."""
    import torch
    from paper_2410_09397_amd import attn
    print("case weigh left out", dtype, kind, d, new, h, flush=True)
    c = Cache(dtype, kind, [300], 2, d, 16)
    Q = torch.randn(new, h, d, device="cuda").to(getattr(torch, DTYPES[dtype]))
    kw = dict(max_q=new, **c.exps())
    _, LSE = attn.attn_paged_fwd(Q, *c.args(), d ** -0.5, **kw)
    LSE[::2] = -float("inf")
    want = attn.attn_cache_weigh(Q, LSE, *c.args(), d ** -0.5, **kw)
    Q[::2] = float("nan")
    got = attn.attn_cache_weigh(Q, LSE, *c.args(), d ** -0.5, **kw)
    assert bool(got.isfinite().all()) and torch.equal(got, want)
    # (a row's weights add up to e^(error of its LSE); their own exponents are of sums of 40, rounded by 2^-24 each in two steps)
    assert abs(float(got.double().sum()) - (new // 2) * h) <= (new // 2) * h * (1.01 * LSE_TOL[dtype] * max(1.0, float(LSE[1::2].abs().max())) + 1e-5)


def test_weights_of_one_query_are_its_softmax():
    import torch
    from paper_2410_09397_amd import attn
    print("case weigh sums", flush=True)
    c = Cache("bf16", "fp8", [3000, 40], 2, 128, 16)
    Q = torch.randn(2, 8, 128, device="cuda").to(torch.bfloat16)
    LSE = attn.attn_paged_fwd(Q, *c.args(), 0.1, **c.exps())[1]
    w = attn.attn_cache_weigh(Q, LSE, *c.args(), 0.1, **c.exps())
    assert float((w.double().sum(-1) - 4.0).abs().max()) <= 4.0 * 1e-4  # (LSE: LSE_TOL of helpers for 32-bit sums)


# ------------------------------------------------------------------------------------------------------------ eviction
def _weights(style, b, kvh, slots, gen):
    import torch
    w = torch.exp(1.5 * torch.randn(b, kvh, slots, generator=gen, device="cuda"))
    if style == "ties":
        w = torch.randint(0, 3, w.shape, generator=gen, device="cuda").float()
        w[..., ::7] = -0.0
    elif style == "odd":
        pick = torch.randint(0, 9, w.shape, generator=gen, device="cuda")
        for x, v in ((0, math.nan), (1, math.inf), (2, -math.inf), (3, -1.5), (4, 1e-42)):
            w = torch.where(pick == x, torch.full_like(w, v), w)
    elif style == "same":
        w = torch.full_like(w, 0.25)
    return w


def _evict_case(dtype, kind, lens, kvh, d, page, budget, first=0, recent=0, style="normal", positions=True, kept=None, in_place=True, layout="phnd", seed=0,
                max_len=None):
    import torch
    from paper_2410_09397_amd import attn
    c = Cache(dtype, kind, lens, kvh, d, page, seed=seed, layout=layout)
    if kind == "fp8":
        for e in (c.K_exp, c.V_exp):
            e.copy_(torch.randint(100, 140, e.shape, device="cuda"))
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    slots, B = c.table.shape[1] * page if max_len is None else max_len, len(lens)
    weight = _weights(style, B, kvh, slots, gen)
    pos = torch.randint(0, 5000, (B, kvh, slots), generator=gen, device="cuda", dtype=torch.int32) if positions else None
    on_gpu = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    seen = [5000 + l for l in lens] if positions else list(lens)
    kept = ([min(l, budget) for l in lens] if kept is None else kept) if positions else [0] * B
    was_w, was_p = weight.clone(), pos.clone() if positions else None
    out = None
    if not in_place:
        n = min(budget, slots)
        out = (torch.full((B, kvh, n + 5), 7.0, device="cuda"), torch.full((B, kvh, n + 5), -7, dtype=torch.int32, device="cuda"), on_gpu([9] * B))
    arrays = [x for x in (c.K, c.V, c.K_exp, c.V_exp) if x is not None]
    before, after = ([_raw(x).clone() for x in arrays] for _ in range(2))
    table = c.table.cpu()
    w, p, new_lens = attn.attn_cache_evict(weight, *c.args(), budget, first=first, recent=recent, pos=pos, kept=on_gpu(kept) if positions else None,
                                           seen=on_gpu(seen) if positions else None, max_len=max_len, out=out, **c.exps())
    assert new_lens.tolist() == [min(l, budget) for l in lens]
    if in_place:
        assert w is weight and p is pos
    want_w, want_p = (was_w.clone(), was_p.clone() if positions else None) if in_place else (torch.full_like(w, 7.0), torch.full_like(p, -7))
    host_w, host_p = was_w.cpu(), was_p.cpu() if positions else None
    for b, l in enumerate(lens):
        for h in range(kvh):
            at = [int(host_p[b, h, s]) if positions and s < kept[b] else seen[b] - l + s for s in range(l)]
            source = keep_ref.evict(host_w[b, h, :l].tolist(), at, l, budget, first, recent, seen[b])
            n = len(source)
            want_w[b, h, :n] = host_w[b, h, source].cuda() if n else want_w[b, h, :0]
            if want_p is not None:
                want_p[b, h, :n] = torch.tensor([at[s] for s in source], dtype=torch.int32, device="cuda")
            moved = [(s, t) for t, s in enumerate(source) if s != t]
            if moved:
                s, t = (torch.tensor(x) for x in zip(*moved))
                rows = lambda y: (table[b, y // page].long().cuda(), h, (y % page).cuda())
                for target, old in zip(after, before):
                    target[rows(t)] = old[rows(s)]
    for a, target in zip(arrays, after):
        assert torch.equal(_raw(a), target)
    raw = lambda x: x.view(torch.int32)
    assert torch.equal(raw(w), raw(want_w))
    if want_p is not None:
        assert torch.equal(p, want_p)
    return c, w, p, new_lens


EVICT = [
    # dtype, kind, lens, kv heads, d, page, budget, first, recent, weights
    ("bf16", "plain", [1], 1, 64, 16, 1, 0, 0, "normal"),
    ("bf16", "plain", [2, 1, 0], 2, 64, 16, 1, 0, 1, "normal"),
    ("bf16", "fp8", [100, 33, 0, 300], 3, 128, 16, 32, 4, 8, "normal"),
    ("bf16", "plain", [1100, 1024, 1025, 5000], 2, 128, 16, 1024, 4, 100, "normal"),
    ("bf16", "fp8", [2100, 700], 2, 256, 64, 600, 0, 0, "ties"),
    ("bf16", "plain", [2100, 700], 2, 40, 64, 600, 1, 30, "odd"),
    ("bf16", "fp8", [2100, 700], 2, 72, 8, 1, 0, 0, "odd"),
    ("bf16", "fp8", [513, 200], 2, 64, 8, 199, 100, 99, "same"),
    ("f32", "plain", [777, 100], 3, 33, 16, 90, 2, 10, "ties"),
    ("f32", "plain", [70000], 2, 16, 128, 30000, 4, 1000, "normal"),
    ("f32", "plain", [20000, 17000], 1, 16, 128, 16500, 4, 16000, "ties"),
    ("f32", "fp8", [900], 2, 104, 4096, 333, 0, 5, "normal"),
    ("f32", "plain", [300], 2, 255, 16, 290, 0, 5, "odd"),
    ("bf16", "plain", [1025] * 70, 2, 64, 16, 1024, 4, 16, "normal"),
    ("bf16", "plain", [64, 65, 66, 63, 128], 2, 64, 16, 64, 64, 0, "normal"),   # nothing but protected tokens stays
]


@pytest.mark.parametrize("case", EVICT)
def test_eviction(case):
    print("case evict", *case, flush=True)
    _evict_case(*case)
    _evict_case(*case, positions=False, in_place=False)
    _evict_case(*case, kept=[0] * len(case[2]), in_place=False, layout="pnhd")


@pytest.mark.parametrize("seed", range(12))
def test_eviction_of_random_sizes(seed):
    rng = random.Random(seed)
    for _ in range(3):
        dtype, kind, kvh = rng.choice(["bf16", "f32"]), rng.choice(["plain", "fp8"]), rng.choice([1, 2, 3])
        lens = [rng.randint(0, rng.choice([20, 300, 4000])) for _ in range(rng.choice([1, 2, 5]))]
        budget = rng.randint(1, max(2, max(lens) + 5))
        first = rng.randint(0, budget) if rng.random() < 0.5 else 0
        recent = rng.randint(0, budget - first) if rng.random() < 0.5 else 0
        d = 8 * rng.randint(1, 32) if dtype == "bf16" or kind == "fp8" else rng.randint(1, 256)
        kept = [rng.randint(0, l) for l in lens]
        case = (dtype, kind, lens, kvh, d, 8 << rng.randint(0, 5), budget, first, recent, rng.choice(["normal", "ties", "odd", "same"]))
        print("case evict", seed, *case, flush=True)
        _evict_case(*case, positions=rng.random() < 0.7, kept=kept, in_place=rng.random() < 0.5, layout=rng.choice(["phnd", "pnhd"]), seed=seed,
                    max_len=rng.choice([None, max(lens + [1])]))


def test_tokens_whose_pages_are_gone_do_not_move():
    import torch
    from paper_2410_09397_amd import attn
    print("case evict pages gone", flush=True)
    c = Cache("bf16", "plain", [64], 1, 64, 16)
    weight = torch.arange(64, device="cuda").float()[None, None].contiguous()  # the last 32 stay: slots 32 .. 63 move to 0 .. 31
    table = c.table.cpu()
    c.table[0, 1], c.table[0, 2] = -1, 10 ** 9  # slots 16 .. 31 cannot be written, 32 .. 47 not be read
    before = c.K.clone(), c.V.clone()
    w, _, n = attn.attn_cache_evict(weight, *c.args(), 32)
    assert n.tolist() == [32] and w[0, 0, :32].tolist() == list(range(32, 64))
    assert torch.equal(_raw(c.K), _raw(before[0])) and torch.equal(_raw(c.V), _raw(before[1]))
    c.table.copy_(table)
    c.table[0, 1] = -1  # 32 .. 47 move to 0 .. 15, 48 .. 63 nowhere
    attn.attn_cache_evict(torch.arange(64, device="cuda").float()[None, None].contiguous(), *c.args(), 32)
    before[0][table[0, 0]], before[1][table[0, 0]] = before[0][table[0, 2]].clone(), before[1][table[0, 2]].clone()
    assert torch.equal(_raw(c.K), _raw(before[0])) and torch.equal(_raw(c.V), _raw(before[1]))


def test_offsets_beyond_32_bits():
    import torch
    from paper_2410_09397_amd import attn
    kvh, page, n, d = 8, 64, 300, 128
    num = (1 << 32) // (kvh * page * d) + 100
    for kind in ("plain", "fp8"):
        print("case evict large cache", kind, flush=True)
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
        for new in (1, 40):
            Q = torch.randn(new, 16, d, device="cuda").to(torch.bfloat16)
            LSE = attn.attn_paged_fwd(Q, *small.args(), 0.1, **small.exps())[1]
            far = attn.attn_cache_weigh(Q, LSE, K, V, table, small.lens, 0.1, **exps)
            near = attn.attn_cache_weigh(Q, LSE, *small.args(), 0.1, **small.exps())
            assert torch.equal(far, near)
        attn.attn_cache_evict(far, K, V, table, small.lens, 100, recent=20, **exps)
        attn.attn_cache_evict(near, *small.args(), 100, recent=20, **small.exps())
        assert torch.equal(far, near)
        for x, y in ((K, small.K), (V, small.V)):
            assert torch.equal(_raw(x)[-used:], _raw(y))
        del K, V, far, exps


def test_calls_without_work():
    import torch
    from paper_2410_09397_amd import attn
    c = Cache("bf16", "plain", [5, 9], 2, 64, 16)
    Q, LSE = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(0, 4, device="cuda")
    w = torch.ones(2, 2, 16, device="cuda")
    attn.attn_cache_weigh(Q, LSE, *c.args(), 1.0, weight=w, decay=0.5)  # no new token: decay alone
    assert w[0, :, :5].eq(0.5).all() and w[0, :, 5:].eq(1.0).all() and w[1, :, :9].eq(0.5).all() and w[1, :, 9:].eq(1.0).all()
    none = torch.empty(2, 0, 16, 64, dtype=torch.bfloat16, device="cuda")
    out = attn.attn_cache_evict(torch.empty(2, 0, 16, device="cuda"), none, none, c.table, c.lens, 7)
    assert out[2].tolist() == [5, 7]
