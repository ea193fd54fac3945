"""Trees of drafted tokens and eviction by attention weight from their definitions in 64 bits, with plain loops over sequences and heads; and how
far each value may be off (see tests/window_bounds.py for the terms)."""
import math

import torch

from tests.window_bounds import F, U, _weight_error


def ancestors(parents, count):
    """[count, count]: token t sees u: itself, and those that lead to it."""
    seen = torch.zeros(count, count, dtype=torch.bool)
    for t in range(count):
        u = t
        while u >= 0:
            seen[t, u] = True
            up = int(parents[u])
            u = up if 0 <= up < u else -1
    return seen


def pack(bits, words):
    """Rows of bits as int32 words."""
    out = torch.zeros(bits.shape[0], words, dtype=torch.int64)
    for t, u in bits.nonzero().tolist():
        out[t, u // 32] |= 1 << (u % 32)
    return torch.where(out >= 1 << 31, out - (1 << 32), out).to(torch.int32)


def tree_seen(bits, length, count, window, sinks):
    """[count, length]: which slots the queries of a sequence see.  bits: [count, count]; drafted token u is in slot length - count + u, if there is one."""
    seen = torch.zeros(count, length, dtype=torch.bool)
    first = length - count
    for t in range(count):
        keys = list(range(max(0, first))) + [first + u for u in range(count) if bits[t, u] and first + u >= 0]
        if window:
            keys = [k for r, k in enumerate(keys) if len(keys) - 1 - r < window or r < sinks]
        seen[t, keys] = True
    return seen


def attend(q, k, v, seen, c, dtype):
    """O, LSE of one head in 64 bits, and the bound of every value of O."""
    s = (c * (q @ k.t())).masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(s, 1) if k.shape[0] else torch.full((q.shape[0],), -math.inf, dtype=q.dtype, device=q.device)
    f = torch.where(lse[:, None] == -math.inf, torch.zeros_like(s), torch.exp(s - lse[:, None]))
    o = f @ v
    if k.shape[0] == 0:
        return o, lse, torch.zeros_like(o)
    size, e = f @ v.abs(), _weight_error(q, k, lse, c)
    return o, lse, U[dtype] * (o.abs() + size) + 2 * ((f * e) @ v.abs()) + (k.shape[0] + 4) * F * (size + o.abs())


def weigh(q, k, lse, first, c, window, sinks):
    """Weights that the queries of one head (positions first ..) add to its keys, and the bound of each: a term is off by the factor
    2^-24 ((d + 4) a + 4 |lse| + 16) with a = c sum |q| |k| (its score, that times log2 e, the difference and exp2), a sum of N of them by N 2^-24."""
    i, j = first + torch.arange(q.shape[0], device=q.device)[:, None], torch.arange(k.shape[0], device=q.device)[None]
    seen = (j <= i) & (i >= 0)
    if window:
        seen &= (i - j < window) | (j < sinks)
    seen &= (lse > -math.inf)[:, None]
    safe = torch.where(lse > -math.inf, lse, torch.zeros_like(lse))[:, None]
    f = torch.where(seen, torch.exp(c * (q @ k.t()) - safe), torch.zeros((), dtype=q.dtype, device=q.device))
    a = abs(c) * (q.abs() @ k.abs().t())
    e = F * ((q.shape[1] + 4) * a + 4 * safe.abs() + 16 + q.shape[0])
    return f.sum(0), (f * e).sum(0)


def evict(weight, pos, length, budget, first, recent, seen):
    """What happens to the tokens of one key head (lists of `length` weights and positions): the slot each of the slots 0 .. n - 1 is filled from."""
    n = min(length, budget)
    if length <= budget:
        return list(range(n))
    safe = [p < first or p >= seen - recent for p in pos]

    def heavy(w):  # NaN below everything
        return (0, 0.0) if w != w else (1, w)
    order = sorted(range(length), key=lambda s: (not safe[s], tuple(-x for x in heavy(weight[s])) if not safe[s] else (0, 0.0), s))
    stay = set(order[:n])
    free = [s for s in range(n) if s not in stay]
    come = [s for s in range(n, length) if s in stay]
    source = list(range(n))
    for to, at in zip(free, come):
        source[to] = at
    return source
