"""Trees, weights and eviction as a server uses them, together with the rest of the paged cache: step after step against 64 bits, captured in a graph, and on
a stream of their own."""
import math
import random

import pytest

from tests import keep_ref
from tests.window_bounds import check

pytestmark = pytest.mark.gpu


def _ints(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("kind,d", [("plain", 64), ("fp8", 128), ("fp8", 72)])
def test_drafting_and_eviction_step_by_step(kind, d):
    """Prompts are written, attended to, weighed and cut down; then every step drafts a tree, attends, keeps a branch, weighs the tokens of it by their rows,
    and evicts.  After each call the cache is set against lists of tokens that are kept here."""
    import torch
    from paper_2410_09397_amd import attn
    print("case run", kind, d, flush=True)
    rng, B, h, kvh, page, budget, first, recent, scale = random.Random(d), 3, 6, 2, 16, 60, 3, 10, d ** -0.5
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    K_pages, V_pages, K_exp, V_exp = attn.attn_cache_pages(60, kvh, page, d, torch.bfloat16 if kind == "plain" else torch.float8_e4m3fn)
    exps = dict(K_exp=K_exp, V_exp=V_exp)
    table = torch.randperm(60)[:48].view(B, 16).to(device="cuda", dtype=torch.int32)
    at = (K_pages, V_pages, table)
    weight, pos = torch.zeros(B, kvh, 256, device="cuda"), torch.zeros(B, kvh, 256, dtype=torch.int32, device="cuda")
    lens, seen, kept = [0] * B, [0] * B, _ints([0] * B)
    new_rows = lambda heads, n: torch.randn(n, heads, d, generator=gen, device="cuda").to(torch.bfloat16)

    def cached(b, n):
        k, v = attn.attn_cache_read(K_pages, V_pages, table[b:b + 1], _ints([n]), torch.bfloat16, n, **exps)
        return k.double(), v.double()

    def attended(O, LSE, Q, rows, b, n, bits):
        k, v = cached(b, n)
        seen_by = keep_ref.tree_seen(bits, n, bits.shape[0], 0, 0).cuda()
        for y in range(h):
            o, lse, bound = keep_ref.attend(Q[rows, y].double(), k[:, y // (h // kvh)], v[:, y // (h // kvh)], seen_by, scale, "bf16")
            check("O", O[rows, y], o, bound)
            assert float((LSE[rows, y].double() - lse).abs().max()) <= 2e-3

    def evict():
        old_w, old_p, was = weight.cpu(), pos.cpu(), [cached(b, lens[b]) for b in range(B)]
        covered = kept.tolist()
        new = attn.attn_cache_evict(weight, *at, _ints(lens), budget, first=first, recent=recent, pos=pos, kept=kept, seen=_ints(seen), max_len=256, **exps)[2]
        for b in range(B):
            k, v = cached(b, int(new[b]))
            for z in range(kvh):
                where = [int(old_p[b, z, s]) if s < covered[b] else seen[b] - lens[b] + s for s in range(lens[b])]
                source = keep_ref.evict(old_w[b, z, :lens[b]].tolist(), where, lens[b], budget, first, recent, seen[b])
                assert torch.equal(k[:, z], was[b][0][source, z]) and torch.equal(v[:, z], was[b][1][source, z])
                assert pos[b, z, :len(source)].tolist() == [where[s] for s in source]
                assert set(range(first)) | set(range(seen[b] - recent, seen[b])) <= set(pos[b, z, :len(source)].tolist())
                assert torch.equal(weight[b, z, :len(source)].cpu(), old_w[b, z, source])
        kept.copy_(new)
        return new.tolist()

    # prompts, weighed by all of their tokens
    new = [100, 70, 61]
    lens, seen, ptr = list(new), list(new), _ints([0, 100, 170, 231])
    Q, K, V = new_rows(h, 231), new_rows(kvh, 231), new_rows(kvh, 231)
    where = dict(q_ptr=ptr, max_q=100, **exps)
    attn.attn_cache_write(K, V, *at, _ints(lens), **where)
    LSE = attn.attn_paged_fwd(Q, *at, _ints(lens), scale, **where)[1]
    attn.attn_cache_weigh(Q, LSE, *at, _ints(lens), scale, weight=weight, max_len=256, **where)
    assert all(abs(float(weight[b, z, :lens[b]].sum()) - 3 * new[b]) <= 0.01 * new[b] for b in range(B) for z in range(kvh))
    lens = evict()
    for step in range(6):
        new = [rng.randint(1, 40) for _ in range(B)]
        starts = [sum(new[:b]) for b in range(B + 1)]
        parents = [[rng.randint(-1, t - 1) for t in range(q)] for q in new]
        bits = [keep_ref.ancestors(p, len(p)) for p in parents]
        context, lens = list(lens), [l + q for l, q in zip(lens, new)]
        Q, K, V = new_rows(h, starts[-1]), new_rows(kvh, starts[-1]), new_rows(kvh, starts[-1])
        where = dict(q_ptr=_ints(starts), max_q=max(new), **exps)
        attn.attn_cache_write(K, V, *at, _ints(lens), **where)
        mask = attn.attn_tree_mask(_ints([x for p in parents for x in p]), max(new), q_ptr=where["q_ptr"])
        O, LSE = attn.attn_tree_fwd(Q, mask, *at, _ints(lens), scale, max_len=max(lens), **where)
        for b in range(B):
            attended(O, LSE, Q, slice(starts[b], starts[b + 1]), b, lens[b], bits[b])
        leaf = [rng.randint(-1, q - 1) for q in new]
        drafted = [cached(b, lens[b]) for b in range(B)]
        left = attn.attn_tree_commit(mask, _ints(leaf), *at, _ints(lens), **where).tolist()
        paths = [[u for u in range(q) if l >= 0 and bits[b][l, u]] for b, (q, l) in enumerate(zip(new, leaf))]
        assert left == [c + len(p) for c, p in zip(context, paths)]
        for b in range(B):
            order = list(range(context[b])) + [context[b] + u for u in paths[b]]
            k, v = cached(b, left[b])
            assert torch.equal(k, drafted[b][0][order]) and torch.equal(v, drafted[b][1][order])
        lens, seen = left, [s + len(p) for s, p in zip(seen, paths)]
        # the rows of the branch that stayed, which see one another as new tokens in their order do
        rows = torch.tensor([starts[b] + u for b in range(B) for u in paths[b]], dtype=torch.long, device="cuda")
        count = [len(p) for p in paths]
        stay = dict(q_ptr=_ints([sum(count[:b]) for b in range(B + 1)]), max_q=max(count + [1]), **exps)
        before = weight.clone()
        attn.attn_cache_weigh(Q[rows], LSE[rows], *at, _ints(lens), scale, weight=weight, decay=0.5, max_len=256, **stay)
        for b in range(B):
            for z in range(kvh):
                add = weight[b, z, :lens[b]].double()
                add[:context[b]] -= 0.5 * before[b, z, :context[b]].double()
                assert abs(float(add.sum()) - 3 * count[b]) <= 1e-3 * (1 + count[b])
        lens = evict()


def test_a_step_in_a_graph():
    """Drafting, committing, weighing and evicting captured once, replayed with other inputs, with eager work in between: the bits of eager calls."""
    import torch
    from paper_2410_09397_amd import attn
    print("case graph", flush=True)
    B, h, kvh, d, page, n = 4, 8, 2, 128, 16, 24
    scale, budget = d ** -0.5, 500
    gen = torch.Generator(device="cuda")
    gen.manual_seed(8)
    fixed = attn.attn_cache_pages(B * 40, kvh, page, d, torch.float8_e4m3fn)
    table = torch.randperm(B * 40).view(B, 40).to(device="cuda", dtype=torch.int32)
    Q = torch.empty(B * n, h, d, dtype=torch.bfloat16, device="cuda")
    K, V = (torch.empty(B * n, kvh, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    parents, leaf, lens = (torch.zeros(x, dtype=torch.int32, device="cuda") for x in (B * n, B, B))
    weight, was = torch.zeros(B, kvh, 640, device="cuda"), torch.zeros(B, kvh, 640, device="cuda")

    def step(pages, weight):
        at, exps = (pages[0], pages[1], table), dict(K_exp=pages[2], V_exp=pages[3])
        attn.attn_cache_write(K, V, *at, lens, **exps)
        mask = attn.attn_tree_mask(parents, n)
        O, LSE = attn.attn_tree_fwd(Q, mask, *at, lens, scale, **exps)
        left = attn.attn_tree_commit(mask, leaf, *at, lens, **exps)
        attn.attn_cache_weigh(Q[n - 1::n].contiguous(), LSE[n - 1::n].contiguous(), *at, left, scale, weight=weight, **exps)
        _, _, new = attn.attn_cache_evict(weight, *at, left, budget, recent=20, **exps)
        return mask, O, LSE, left, new

    def inputs(seed):
        rng = random.Random(seed)
        for x in (Q, K, V):
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        parents.copy_(_ints([rng.randint(-1, t - 1) for _ in range(B) for t in range(n)]))
        leaf.copy_(_ints([rng.randint(-1, n - 1) for _ in range(B)]))
        lens.copy_(_ints([rng.randint(n, 640) for _ in range(B)]))
        was.copy_(torch.rand(was.shape, generator=gen, device="cuda"))
        for x in fixed[:2]:
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda").to(torch.float8_e4m3fn))

    raw = lambda x: x.view(torch.uint8) if x.dtype is torch.float8_e4m3fn else x
    inputs(0)
    pages = [x.clone() for x in fixed]
    step(pages, weight)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        out = step(pages, weight)
    for seed in range(1, 6):
        inputs(seed)
        eager, eager_weight = [x.clone() for x in fixed], was.clone()
        want = step(eager, eager_weight)
        for x, y in zip(pages, fixed):
            raw(x).copy_(raw(y))
        weight.copy_(was)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip([*out, weight], [*want, eager_weight]):
            assert torch.equal(x, y), seed
        for x, y in zip(pages, eager):
            assert torch.equal(raw(x), raw(y)), seed


def test_results_come_from_the_pool_of_the_stream():
    import torch
    from paper_2410_09397_amd import attn
    from tests.test_gpu_window_streams import _freed
    B, n, page = 4, 64, 16
    K, V = (torch.randn(B * 512, 4, 128, device="cuda").to(torch.bfloat16) for _ in range(2))
    Q = torch.randn(B * n, 8, 128, device="cuda").to(torch.bfloat16)
    pages = attn.attn_cache_pages(B * 32, 4, page, 128, torch.bfloat16)[:2]
    table, lens = torch.arange(B * 32, dtype=torch.int32, device="cuda").view(B, -1), _ints([512] * B)
    attn.attn_cache_write(K, V, *pages, table, lens)
    parents = _ints(([-1] + list(range(n - 1))) * B)
    leaf = _ints([n - 1] * B)

    def all_of(stream):
        mask = attn.attn_tree_mask(parents, n, stream=stream)
        O, LSE = attn.attn_tree_fwd(Q, mask, *pages, table, lens, 0.1, stream=stream)
        weight = attn.attn_cache_weigh(Q, LSE, *pages, table, lens, 0.1, stream=stream)
        left = attn.attn_tree_commit(mask, leaf, *pages, table, lens, stream=stream)
        return mask, O, LSE, weight, left
    want = all_of(None)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    free = _freed(*want)
    got = all_of(side)
    side.synchronize()
    for x, y in zip(got, want):
        assert x.data_ptr() not in free and torch.equal(x, y)


def test_eviction_keeps_the_attention_of_what_stays():
    """A query over an evicted cache: the softmax over the tokens that stayed, whatever their order in the slots."""
    import torch
    from paper_2410_09397_amd import attn
    from tests.test_gpu_paged import Cache
    print("case evict and attend", flush=True)
    c = Cache("bf16", "plain", [400], 1, 64, 16)
    Q = torch.randn(1, 4, 64, device="cuda").to(torch.bfloat16)
    O, LSE = attn.attn_paged_fwd(Q, *c.args(), 1.0)
    w = attn.attn_cache_weigh(Q, LSE, *c.args(), 1.0)
    total = w[0, 0, :400].clone()
    _, _, n = attn.attn_cache_evict(w, *c.args(), 100)
    stay = total.topk(100)[1].sort()[0]
    o, l = attn.attn_paged_fwd(Q, c.K, c.V, c.table, n, 1.0)
    k, v = c.keys[0][stay, 0], c.values[0][stay, 0]
    for y in range(4):
        want, lse, bound = keep_ref.attend(Q[:, y].double(), k, v, torch.ones(1, 100, dtype=torch.bool, device="cuda"), 1.0, "bf16")
        check("head %d" % y, o[:, y], want, bound)
    assert float(total.sum()) == pytest.approx(4.0, abs=4e-4) and math.isfinite(float(l.abs().max()))
