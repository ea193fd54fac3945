"""Windowed attention and the paged cache from their definitions in 64 bits, with plain loops over sequences and heads."""
import math

import torch


def visible(i, j, window, sinks):
    """Whether the query at position i sees key j (tensors of positions that broadcast)."""
    seen = (j <= i) & (i >= 0)
    return seen & ((i - j < window) | (j < sinks)) if window else seen


def attend(q, k, v, first, scale, window, sinks):
    """O, LSE and the weights of queries at positions first, first + 1, ... over keys 0, 1, ...; rows that see nothing: 0, -inf, 0."""
    i = first + torch.arange(q.shape[0], device=q.device)[:, None]
    j = torch.arange(k.shape[0], device=q.device)[None, :]
    s = (scale * (q @ k.t())).masked_fill(~visible(i, j, window, sinks), -math.inf)
    lse = torch.logsumexp(s, 1) if k.shape[0] else torch.full((q.shape[0],), -math.inf, dtype=q.dtype, device=q.device)
    f = torch.where(lse[:, None] == -math.inf, torch.zeros_like(s), torch.exp(s - lse[:, None]))
    return f @ v, lse, f


def window_attention(Q, K, V, dO, scale, window, sinks, lens=None, given=None):
    """O, LSE, dQ, dK, dV in 64 bits; the gradients from the O and LSE that the backward is `given` (its rounded inputs), if any."""
    b, h, n, d = Q.shape
    group = h // K.shape[1]
    Q, K, V, dO = (t.double() for t in (Q, K, V, dO))
    O, dQ, dK, dV = (torch.zeros_like(t) for t in (Q, Q, K, K))
    LSE = torch.full((b, h, n), -math.inf, dtype=torch.float64, device=Q.device)
    for x in range(b):
        r = slice(0, n if lens is None else min(max(int(lens[x]), 0), n))
        for y in range(h):
            z = y // group
            q, g, k, v = Q[x, y, r], dO[x, y, r], K[x, z, r], V[x, z, r]
            O[x, y, r], LSE[x, y, r], f = attend(q, k, v, 0, scale, window, sinks)
            o = O[x, y, r]
            if given is not None:
                o = given[0][x, y, r].double()
                f = f * torch.exp(LSE[x, y, r] - given[1][x, y, r].double())[:, None]
            p = f * (g @ v.t() - (g * o).sum(1, keepdim=True))
            dQ[x, y, r] = scale * (p @ k)
            dK[x, z, r] += scale * (p.t() @ q)
            dV[x, z, r] += f.t() @ g
    return O, LSE, dQ, dK, dV


def paged_attention(Q, keys, values, starts, lens, scale, window, sinks):
    """O, LSE of ragged queries; keys, values: per sequence [len, kv_heads, d] in 64 bits; starts: host row offsets."""
    total, h, d = Q.shape
    O = torch.zeros(total, h, d, dtype=torch.float64, device=Q.device)
    LSE = torch.zeros(total, h, dtype=torch.float64, device=Q.device)
    for b, (k, v) in enumerate(zip(keys, values)):
        r = slice(starts[b], starts[b + 1])
        for y in range(h):
            z = y // (h // k.shape[1])
            O[r, y], LSE[r, y], _ = attend(Q[r, y].double(), k[:, z], v[:, z], lens[b] - (starts[b + 1] - starts[b]), scale, window, sinks)
    return O, LSE


def quantise(x):
    """Codes (as the values they are) and exponent bytes of the rows of a CPU tensor, value by value in Python's own arithmetic where a
    row is not ordinary, by frexp and torch's rounding on the CPU elsewhere."""
    x = x.float()
    finite = torch.isfinite(x)
    top = torch.where(finite, x.abs(), torch.zeros_like(x)).amax(-1).double()
    m, e = torch.frexp(top)
    e = torch.where(top == 0, torch.zeros_like(e), (e - 9 + (m > 0.875).int()).clamp(min=-126))
    y = x.double() * torch.pow(torch.tensor(2.0, dtype=torch.float64), -e.double())[..., None]
    codes = torch.where(finite, y.float(), torch.full_like(x, math.nan)).to(torch.float8_e4m3fn)
    return codes, (e + 127).to(torch.uint8)


def values(codes, exps):
    return codes.double() if exps is None else codes.float().double() * torch.pow(torch.tensor(2.0, dtype=torch.float64, device=codes.device), exps.double() - 127)[..., None]
