"""How far each single value of windowed attention may be from its definition in 64 bits: gates relative to the largest value of a tensor say little
about rows that average over many keys, whose values are small.

One rounding to bf16 moves a value by at most 2^-8 of itself (u below).  The bf16 kernels round the weights P and dS and the result:
    |O - o| <= u |o| + u sum_j P_ij |v_j|                |dQ - dq| <= u |dq| + u c sum_j |dS_ij| |k_j|
    |dV - dv| <= u |dv| + u sum_i P_ij |do_i|            |dK - dk| <= u |dk| + u c sum_i |dS_ij| |q_i|
and everything else is fp32 arithmetic.  A score is a sum of d products that is off by at most (d + 1) 2^-24 a, a = c sum |q| |k|, and LSE in 32 bits by 2^-24 |LSE| (and a
few units of exp2 and log2): so every weight may be off by the factor e = 2^-24 ((d + 1) a + |LSE| + 16), dP by 2^-24 (d + 1) sum |do| |v|, delta by
2^-24 (d + 1) sum |do| |o|, and a sum of N terms by N 2^-24 of their magnitudes."""
import torch

from tests.window_ref import attend

U = {"bf16": 2.0 ** -8, "f32": 0.0}
F = 2.0 ** -24


def _weight_error(q, k, lse, c):
    a = abs(c) * (q.abs() @ k.abs().t())
    lse = torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)
    return F * ((q.shape[1] + 1) * a + a.amax(1, keepdim=True) + lse.abs()[:, None] + 16)


def forward(q, k, v, first, c, window, sinks, dtype):
    """O of one head in 64 bits and the bound of every value; queries at positions first, first + 1, ..."""
    o, lse, f = attend(q, k, v, first, c, window, sinks)
    if k.shape[0] == 0:
        return o, torch.zeros_like(o)
    size = f @ v.abs()
    e = _weight_error(q, k, lse, c)
    # (a sum of weights that are each off by e is off as far, and so is what it divides)
    return o, U[dtype] * (o.abs() + size) + 2 * ((f * e) @ v.abs()) + (k.shape[0] + 4) * F * (size + o.abs())


def backward(q, k, v, g, o, lse, first, c, window, sinks, dtype):
    """dQ, dK, dV of one query head from the O and LSE that the backward is given, and the bounds without the rounding of a sum over heads."""
    _, exact, f = attend(q, k, v, first, c, window, sinks)
    f = f * torch.exp(exact - torch.where(torch.isinf(lse), exact, lse))[:, None].nan_to_num(0.0)
    e, n = _weight_error(q, k, lse, c), max(q.shape[0], k.shape[0])
    dp, delta = g @ v.t(), (g * o).sum(1, keepdim=True)
    ds = f * (dp - delta)
    off = f * F * (q.shape[1] + 1) * (g.abs() @ v.abs().t() + (g * o).abs().sum(1, keepdim=True)) + ds.abs() * e
    u = U[dtype] + (n + 4) * F
    dq, dk, dv = c * (ds @ k), c * (ds.t() @ q), f.t() @ g
    return ((dq, dk, dv), (U[dtype] * dq.abs() + abs(c) * ((u * ds.abs() + off) @ k.abs()), abs(c) * ((u * ds.abs() + off).t() @ q.abs()),
                           (u * f + f * e).t() @ g.abs()))


def check(name, got, want, bound):
    """Every value within its bound; infinities and NaN fail."""
    err = (got.double() - want).abs()
    bad = ~(err <= bound)
    if bool(bad.any()):
        at = tuple(int(x) for x in bad.nonzero()[0])
        raise AssertionError("%s: %d of %d values beyond their bounds, first at %s: %g for %g, bound %g"
                             % (name, int(bad.sum()), bad.numel(), at, float(got[at]), float(want[at]), float(bound[at])))
    return float((err / bound.clamp(min=1e-300)).max()) if err.numel() else 0.0


def check_step(inputs, got, c, window, sinks, lens, dtype):
    """All of attn_win_fwd's and attn_win_bwd's results; returns the largest share of a bound that is used."""
    Q, K, V, dO = (t.double() for t in inputs)
    O, LSE, dQ, dK, dV = got
    b, h, n, _ = Q.shape
    group, most = h // K.shape[1], 0.0
    for x in range(b):
        length = n if lens is None else min(max(int(lens[x]), 0), n)
        r = slice(0, length)
        for t in (O[x, :, length:], dQ[x, :, length:], dK[x, :, length:], dV[x, :, length:]):
            assert not bool(t.any()), "padding"
        if length == 0:
            continue
        for z in range(K.shape[1]):
            want, bound = [torch.zeros_like(K[x, z, r]) for _ in range(2)], [torch.zeros_like(K[x, z, r]) for _ in range(2)]
            for y in range(z * group, (z + 1) * group):
                where = "sequence %d head %d " % (x, y)
                most = max(most, check(where + "O", O[x, y, r], *forward(Q[x, y, r], K[x, z, r], V[x, z, r], 0, c, window, sinks, dtype)))
                grads, limits = backward(Q[x, y, r], K[x, z, r], V[x, z, r], dO[x, y, r], O[x, y, r].double(), LSE[x, y, r].double(), 0, c, window, sinks, dtype)
                most = max(most, check(where + "dQ", dQ[x, y, r], grads[0], limits[0]))
                for i in range(2):
                    want[i] += grads[1 + i]
                    bound[i] += limits[1 + i]
            for i, (what, t) in enumerate((("dK", dK), ("dV", dV))):
                limit = (1 + group * F) * bound[i] + U[dtype] * want[i].abs()
                most = max(most, check("sequence %d key head %d %s" % (x, z, what), t[x, z, r], want[i], limit))
    return most


def check_pages(Q, O, keys, values, starts, lens, c, window, sinks, dtype):
    most = 0.0
    for b, (k, v) in enumerate(zip(keys, values)):
        r = slice(starts[b], starts[b + 1])
        for y in range(Q.shape[1]):
            z = y // (Q.shape[1] // k.shape[1])
            want = forward(Q[r, y].double(), k[:, z], v[:, z], lens[b] - (starts[b + 1] - starts[b]), c, window, sinks, dtype)
            most = max(most, check("sequence %d head %d O" % (b, y), O[r, y], *want))
    return most
