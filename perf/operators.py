"""Windowed attention and the paged key/value cache, as cases to be timed.

A case is a dict of plain values.  `op` says which operator a pass goes through:
  "train"  attn_win_fwd, then attn_win_bwd: a training step of attention with a sliding window, a few first keys that
           stay visible, heads that share keys and values, and sequences of different lengths in a batch
  "write"  attn_cache_write: the keys and values of new tokens into the pages of a cache, quantised on the way
  "read"   attn_cache_read: the last tokens of every sequence back out of the pages, in order and dequantised
  "paged"  attn_paged_fwd: the attention of new tokens (one or a chunk per sequence) over the paged cache

Visible keys.  A query at position i sees key j iff j <= i and (window == 0 or i - j < window or j < sinks), both inside
their sequence.  In a paged cache the new tokens of a sequence are its last ones.

Quantised pages ("fp8") hold e4m3 codes and, per token and head, one byte e: a stored code c stands for c 2^(e - 127), where
2^(e - 127) is the smallest power of two that brings the row's largest magnitude to 448 or less (e = 127 for a row of zeros).

The lengths of the sequences in a batch go by the case alone; the seed gives their order, the order of the pages, and all values.
Q, K, V and dO are normal with unit variance, as in the benchmark's workloads (scores of unit variance after the 1/sqrt(d)
scale); keys that go into a cache have channels of different spread, as projections do.
"""
import math

import torch

own = False

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4.0, "bf16": 2.0, "fp8": 1.0}


# ------------------------------------------------------------------------------------------------------------- cases
def _train(name, dtype, batch, heads, kv_heads, n, d, window=0, sinks=0, ragged=False):
    return _named(name, dict(op="train", dtype=dtype, batch=batch, heads=heads, kv_heads=kv_heads, n=n, d=d, window=window,
                             sinks=sinks, ragged=ragged))


def _cache(op, name, dtype, cache, batch, heads, kv_heads, d, page, len_lo, len_hi, q_lo, q_hi, window=0, sinks=0):
    return _named(name, dict(op=op, dtype=dtype, cache=cache, batch=batch, heads=heads, kv_heads=kv_heads, d=d, page=page,
                             len_lo=len_lo, len_hi=len_hi, q_lo=q_lo, q_hi=q_hi, window=window, sinks=sinks))


def _named(name, case):
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # a small model that trains in full precision, at an odd length and head dimension
        _train("train_f32_n777_d80_w128", "f32", 2, 6, 2, 777, 80, window=128),
        # an ordinary training step on padded sequences of different lengths
        _train("train_n2048_d64_w256_ragged", "bf16", 2, 16, 4, 2048, 64, window=256, sinks=4, ragged=True),
        # long-context training, the largest of the cases
        _train("train_n8192_d128_w1024", "bf16", 1, 32, 8, 8192, 128, window=1024, sinks=4),
        # serving, one new token for each of many requests goes into a quantised cache: latency
        _cache("write", "write_fp8_64x1", "bf16", "fp8", 64, 32, 8, 128, 16, 32, 2048, 1, 1),
        # the prompts of a batch go into a quantised cache
        _cache("write", "write_fp8_prompts", "bf16", "fp8", 8, 32, 8, 128, 16, 500, 4096, 500, 4096),
        # one short request leaves an unquantised cache (to another machine, to the host)
        _cache("read", "read_bf16_333", "bf16", "bf16", 1, 16, 4, 64, 16, 333, 333, 333, 333),
        # a batch of sequences read back for another pass over them
        _cache("read", "read_fp8_prompts", "bf16", "fp8", 8, 32, 8, 128, 64, 500, 4096, 500, 4096),
        # serving, the next token of a few short requests: latency
        _cache("paged", "decode_4_d64", "bf16", "bf16", 4, 16, 4, 64, 16, 20, 600, 1, 1),
        # the next token of many requests of all lengths, quantised cache
        _cache("paged", "decode_64_d128_fp8", "bf16", "fp8", 64, 32, 8, 128, 16, 100, 8192, 1, 1),
        # the next token of one very long request
        _cache("paged", "decode_1_len65536", "bf16", "bf16", 1, 32, 8, 128, 64, 65536, 65536, 1, 1),
        # a long prompt that is taken in chunks: 2048 new tokens behind 8192 cached ones
        _cache("paged", "chunk_2048_of_10240_fp8", "bf16", "fp8", 1, 32, 8, 128, 16, 10240, 10240, 2048, 2048),
        # a batch of requests that decode beside ones that take in a piece of their prompts, windowed
        _cache("paged", "mixed_16_w1024", "bf16", "bf16", 16, 32, 8, 128, 16, 300, 6000, 1, 256, window=1024, sinks=4),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        kind = rng.choice(["train", "train", "train", "train_f32", "train_odd_d", "write", "write", "read", "read", "decode", "decode",
                           "decode", "chunk", "chunk"])
        kv_heads = rng.choice([1, 2, 3, 4, 8])
        heads = kv_heads * rng.choice([1, 1, 2, 3, 4, 8])
        if kind.startswith("train"):
            batch, n, d, dtype = _log_int(rng, 1, 4), _log_int(rng, 33, 8192), rng.choice([64, 128, 128, 256]), "bf16"
            if kind == "train_f32":
                n, d, dtype = _log_int(rng, 33, 1500), rng.randint(16, 128), "f32"
            elif kind == "train_odd_d":
                n, d = _log_int(rng, 33, 2048), 8 * rng.choice([4, 5, 6, 7, 9, 10, 11, 12, 13, 14, 15, 17, 20, 24])
            window = _log_int(rng, 16, n) if rng.random() < 0.75 and n > 16 else 0
            sinks = rng.choice([0, 0, 1, 4, 16, 70]) if window else 0
            most = 2.7e11 if kind == "train" else 4e9
            if float(batch * heads) * n * n * d <= most and float(batch * heads) * n * n <= 2.1e9:
                return _train("", dtype, batch, heads, kv_heads, n, d, window, sinks, batch > 1 and rng.random() < 0.4)
            continue
        page, cache, dtype = rng.choice([16, 16, 32, 64, 128]), rng.choice(["fp8", "fp8", "bf16"]), "bf16"
        d = rng.choice([64, 128, 128, 256])
        if kind in ("write", "read"):
            if rng.random() < 0.2:
                d = 8 * rng.choice([4, 5, 10, 12, 20])
            batch = _log_int(rng, 1, 64)
            q_hi = _log_int(rng, 1, 4096)
            q_lo = _log_int(rng, 1, q_hi)
            len_hi = q_hi + rng.choice([0, 0, 17, 1000])
            len_lo = _log_int(rng, q_lo, len_hi)
            if batch * q_hi * kv_heads * d <= 8 * 4096 * 8 * 128:
                return _cache(kind, "", dtype, cache, batch, heads, kv_heads, d, page, len_lo, len_hi, q_lo, q_hi)
            continue
        if kind == "decode":
            batch, len_hi, q_lo, q_hi = _log_int(rng, 1, 128), _log_int(rng, 16, 65536), 1, 1
        else:
            batch, q_hi = _log_int(rng, 1, 16), _log_int(rng, 2, 2048)
            q_lo, len_hi = rng.choice([1, q_hi, max(1, q_hi // 2)]), q_hi + _log_int(rng, 1, 8192)
        len_lo = _log_int(rng, q_lo, len_hi)
        window = _log_int(rng, 16, len_hi) if rng.random() < 0.4 else 0
        sinks = rng.choice([0, 1, 4, 70]) if window else 0
        if float(batch) * len_hi * kv_heads * d <= 64 * 8192 * 8 * 128 and float(batch) * q_hi * len_hi * heads * d <= 8.6e10:
            return _cache("paged", "", dtype, cache, batch, heads, kv_heads, d, page, len_lo, len_hi, q_lo, q_hi, window, sinks)


def _spread(lo, hi, count):
    """`count` lengths between lo and hi, spread evenly over the logarithm; the first is hi."""
    return [max(lo, min(hi, int(round(hi * (lo / hi) ** (i / max(1, count - 1)))))) for i in range(count)]


def _lengths(case):
    """Host lists by the case alone: the length of every sequence, and (in a cache) the number of its new tokens."""
    if case["op"] == "train":
        n = case["n"]
        return (_spread(max(1, n // 3), n, case["batch"]) if case["ragged"] else [n] * case["batch"]), None
    lens = _spread(case["len_lo"], case["len_hi"], case["batch"])
    new = _spread(case["q_lo"], case["q_hi"], case["batch"])
    return lens, [min(a, b) for a, b in zip(lens, new)]


# ------------------------------------------------------------------------------------------------------------ inputs
class State:
    pass


def _power(e):
    """2^e in 32 bits, for whole numbers e from -126 to 127."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _quantise(x):
    """Codes and exponent bytes of the rows of x."""
    x = x.float()
    m, e = torch.frexp(x.abs().amax(-1))
    e = torch.where(m == 0, torch.zeros_like(e), (e - 9 + (m > 0.875).int()).clamp(-126, 120))
    return (x * _power(-e)[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def prepare(case, seed):
    s = State()
    s.case = dict(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    host = torch.Generator()
    host.manual_seed(int(seed))
    dtype = _DTYPE[case["dtype"]]
    B, H, Hk, d = case["batch"], case["heads"], case["kv_heads"], case["d"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    s.scale = d ** -0.5
    lens, new = _lengths(case)
    order = torch.randperm(B, generator=host).tolist()
    lens = [lens[i] for i in order]
    if case["op"] == "train":
        n = case["n"]
        s.Q, s.dO = (normal(B, H, n, d).to(dtype) for _ in range(2))
        s.K, s.V = (normal(B, Hk, n, d).to(dtype) for _ in range(2))
        s.lens = torch.tensor(lens, dtype=torch.int32, device="cuda") if case["ragged"] else None
        return s
    new = [new[i] for i in order]
    page = case["page"]
    s.max_len, s.max_q, s.total = max(lens), max(new), sum(new)
    s.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s.q_ptr = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(device="cuda", dtype=torch.int32)
    # every sequence's pages lie anywhere; entries past a sequence's last page are -1
    used = [-(-l // page) for l in lens]
    table = torch.full((B, max(used)), -1, dtype=torch.int32)
    owner = torch.arange(max(used))[None, :] < torch.tensor(used)[:, None]
    num = sum(used) + 3
    table[owner] = torch.randperm(num, generator=host)[:sum(used)].to(torch.int32)
    s.table = table.cuda()
    s.K_exp = s.V_exp = None
    channel = torch.exp(0.5 * normal(Hk, 1, d))
    channel = channel / channel.square().mean(-1, keepdim=True).sqrt()
    if case["op"] == "write":
        s.K = (normal(s.total, Hk, d) * channel.squeeze(1)).to(dtype)
        s.V = normal(s.total, Hk, d).to(dtype)
        kind = torch.float8_e4m3fn if case["cache"] == "fp8" else _DTYPE[case["cache"]]
        s.K_pages, s.V_pages = (torch.zeros(num, Hk, page, d, dtype=torch.float32, device="cuda").to(kind) for _ in range(2))
        if case["cache"] == "fp8":
            s.K_exp, s.V_exp = (torch.full((num, Hk, page), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
        return s
    K, V = (normal(num, Hk, page, d) * channel).to(dtype), normal(num, Hk, page, d).to(dtype)
    if case["cache"] == "fp8":
        (s.K_pages, s.K_exp), (s.V_pages, s.V_exp) = _quantise(K), _quantise(V)
    else:
        s.K_pages, s.V_pages = (x.to(_DTYPE[case["cache"]]) for x in (K, V))
    if case["op"] == "paged":
        s.Q = normal(s.total, H, d).to(dtype)
    return s


# ------------------------------------------------------------------------------------------------------- plain forms
def _sees(i, j, window, sinks):
    seen = (j <= i) & (i >= 0)
    if window:
        seen = seen & ((i - j < window) | (j < sinks))
    return seen


def _plain_train(s):
    c = s.case
    B, H, Hk, n, d = c["batch"], c["heads"], c["kv_heads"], c["n"], c["d"]
    G = H // Hk
    at = torch.arange(n, device="cuda")
    seen = _sees(at[:, None], at[None, :], c["window"], c["sinks"])[None, None, None]
    if s.lens is not None:
        inside = at[None] < s.lens[:, None]
        seen = seen & inside[:, None, None, None, :] & inside[:, None, None, :, None]
    # [batch, kv head, head of the group, n, d]
    Q, dO = (x.float().view(B, Hk, G, n, d) for x in (s.Q, s.dO))
    K, V = (x.float().view(B, Hk, 1, n, d) for x in (s.K, s.V))
    S = torch.matmul(Q, K.transpose(-1, -2)).mul_(s.scale).masked_fill_(~seen, -math.inf)
    m = S.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    P = S.sub_(m).exp_()
    l = P.sum(-1, keepdim=True)
    lse = (l.log() + m).squeeze(-1)
    P = P.div_(torch.where(l == 0, torch.ones_like(l), l))
    O = torch.matmul(P, V)
    dP = torch.matmul(dO, V.transpose(-1, -2))
    dV = torch.matmul(P.transpose(-1, -2), dO).sum(2)
    dS = dP.sub_((dO * O).sum(-1, keepdim=True)).mul_(P)
    del P
    dQ = torch.matmul(dS, K) * s.scale
    dK = torch.matmul(dS.transpose(-1, -2), Q).sum(2) * s.scale
    dt = s.Q.dtype
    return (O.view(B, H, n, d).to(dt), lse.view(B, H, n), dQ.view(B, H, n, d).to(dt), dK.to(dt), dV.to(dt))


def _token_places(s):
    """Sequence and position of every new token, and which page and row it lies in."""
    row = torch.arange(s.total, device="cuda")
    seq = torch.searchsorted(s.q_ptr[1:].contiguous(), row.to(torch.int32), right=True)
    pos = s.lens[seq] - (s.q_ptr[seq + 1] - row)
    page = s.case["page"]
    return seq, row - s.q_ptr[seq], pos, s.table[seq, torch.div(pos, page, rounding_mode="floor")].long(), pos % page


def _plain_write(s):
    _, _, _, page, slot = _token_places(s)
    if s.K_exp is None:
        s.K_pages[page, :, slot] = s.K.to(s.K_pages.dtype)
        s.V_pages[page, :, slot] = s.V.to(s.V_pages.dtype)
        return s.K_pages, s.V_pages
    (K, K_exp), (V, V_exp) = _quantise(s.K), _quantise(s.V)
    s.K_pages.view(torch.uint8)[page, :, slot] = K.view(torch.uint8)
    s.V_pages.view(torch.uint8)[page, :, slot] = V.view(torch.uint8)
    s.K_exp[page, :, slot] = K_exp
    s.V_exp[page, :, slot] = V_exp
    return s.K_pages, s.V_pages, s.K_exp, s.V_exp


def _values(pages, exps):
    x = pages.float()
    return x if exps is None else x * _power(exps.int() - 127)[..., None]


def _plain_read(s):
    _, _, _, page, slot = _token_places(s)
    dtype = _DTYPE[s.case["dtype"]]
    if s.K_exp is None:
        return s.K_pages[page, :, slot].to(dtype), s.V_pages[page, :, slot].to(dtype)
    K, V = (x.view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn) for x in (s.K_pages, s.V_pages))
    return _values(K, s.K_exp[page, :, slot]).to(dtype), _values(V, s.V_exp[page, :, slot]).to(dtype)


def _plain_paged(s):
    c = s.case
    B, H, Hk, d = c["batch"], c["heads"], c["kv_heads"], c["d"]
    G, nq = H // Hk, s.max_q
    seq, t, _, _, _ = _token_places(s)

    def gathered(pages, exps):  # [batch, kv head, key, d]
        page = s.table.clamp(min=0).long()
        if exps is None:
            x = pages[page].float()
        else:
            x = _values(pages.view(torch.uint8)[page].view(torch.float8_e4m3fn), exps[page])
        return x.permute(0, 2, 1, 3, 4).reshape(B, Hk, -1, d)

    K, V = gathered(s.K_pages, s.K_exp), gathered(s.V_pages, s.V_exp)
    Q = torch.zeros(B, nq, H, d, device="cuda")
    Q[seq, t] = s.Q.float()
    Q = Q.view(B, nq, Hk, G, d).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * nq, d)
    count = s.q_ptr[1:] - s.q_ptr[:-1]
    i = (s.lens - count)[:, None] + torch.arange(nq, device="cuda")[None]  # position of every query
    seen = _sees(i[:, :, None], torch.arange(K.shape[2], device="cuda")[None, None, :], c["window"], c["sinks"])
    seen = seen & (i < s.lens[:, None])[:, :, None]
    S = torch.matmul(Q, K.transpose(-1, -2)).mul_(s.scale).view(B, Hk, G, nq, -1)
    S = S.masked_fill_(~seen[:, None, None], -math.inf)
    m = S.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    P = S.sub_(m).exp_()
    l = P.sum(-1, keepdim=True)
    O = torch.matmul(P.view(B, Hk, G * nq, -1), V).view(B, Hk, G, nq, d) / torch.where(l == 0, torch.ones_like(l), l)
    lse = (l.log() + m).squeeze(-1)
    O = O.permute(0, 3, 1, 2, 4).reshape(B, nq, H, d)[seq, t]
    return O.to(s.Q.dtype), lse.permute(0, 3, 1, 2).reshape(B, nq, H)[seq, t]


# ------------------------------------------------------------------------------------------------------------ a pass
def _own(s):
    from paper_2410_09397_amd import attn
    c = s.case
    if c["op"] == "train":
        O, LSE = attn.attn_win_fwd(s.Q, s.K, s.V, s.scale, window=c["window"], sinks=c["sinks"], lens=s.lens)
        return (O, LSE) + tuple(attn.attn_win_bwd(s.Q, s.K, s.V, O, s.dO, LSE, s.scale, window=c["window"], sinks=c["sinks"],
                                                  lens=s.lens))
    if c["op"] == "write":
        attn.attn_cache_write(s.K, s.V, s.K_pages, s.V_pages, s.table, s.lens, q_ptr=s.q_ptr, max_q=s.max_q, K_exp=s.K_exp,
                              V_exp=s.V_exp)
        return (s.K_pages, s.V_pages) if s.K_exp is None else (s.K_pages, s.V_pages, s.K_exp, s.V_exp)
    if c["op"] == "read":
        return attn.attn_cache_read(s.K_pages, s.V_pages, s.table, s.lens, _DTYPE[c["dtype"]], s.total, q_ptr=s.q_ptr,
                                    max_q=s.max_q, K_exp=s.K_exp, V_exp=s.V_exp)
    return attn.attn_paged_fwd(s.Q, s.K_pages, s.V_pages, s.table, s.lens, s.scale, q_ptr=s.q_ptr, max_q=s.max_q,
                               max_len=s.max_len, window=c["window"], sinks=c["sinks"], K_exp=s.K_exp, V_exp=s.V_exp)


def run(s):
    if own:
        return _own(s)
    return {"train": _plain_train, "write": _plain_write, "read": _plain_read, "paged": _plain_paged}[s.case["op"]](s)


# -------------------------------------------------------------------------------------------------- the definition
def _exact_rows(Q, K, V, first, scale, window, sinks):
    """Softmax attention in 64 bits of queries at positions first, first + 1, ... over keys 0, 1, ...: O, LSE and the weights."""
    i = first + torch.arange(Q.shape[0], device=Q.device)
    j = torch.arange(K.shape[0], device=Q.device)
    gap = i[:, None] - j[None, :]
    hidden = gap < 0
    if window > 0:
        hidden |= (gap >= window) & (j[None, :] >= sinks)
    score = scale * (Q @ K.t())
    score[hidden] = -math.inf
    lse = torch.logsumexp(score, 1)
    f = torch.exp(score - lse[:, None])
    return f @ V, lse, f


_E4M3 = sorted({(m / 8 if e == 0 else 1 + m / 8) * 2.0 ** (max(e, 1) - 7) for e in range(16) for m in range(8) if (e, m) != (15, 7)})


def _two_to(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_codes(x):
    """What the codes and the exponents of rows stand for: the nearest value of the format, a tie to the even code."""
    top = x.abs().amax(-1)
    e = torch.where(top > 0, torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0)), torch.zeros_like(top))
    e = torch.where((top > 0) & (top <= 448.0 * _two_to(e - 1)), e - 1, e)
    e = torch.where(top > 448.0 * _two_to(e), e + 1, e).clamp(-126, 120)
    y = x / _two_to(e)[..., None]
    values = torch.tensor(_E4M3, dtype=torch.float64, device=x.device)
    up = torch.searchsorted(values, y.abs().contiguous()).clamp(max=len(_E4M3) - 1)
    low = (up - 1).clamp(min=0)
    a, b = y.abs() - values[low], values[up] - y.abs()
    pick = torch.where((b < a) | ((a == b) & (up % 2 == 0)), up, low)
    return torch.copysign(values[pick], y), e


def exact(case, seed):
    s = prepare(case, seed)
    B, H, Hk, d = case["batch"], case["heads"], case["kv_heads"], case["d"]
    G, window, sinks = H // Hk, case.get("window", 0), case.get("sinks", 0)
    if case["op"] == "train":
        n = case["n"]
        lens = [n] * B if s.lens is None else s.lens.tolist()
        new = lambda heads: torch.zeros(B, heads, n, d, dtype=torch.float64, device="cuda")
        O, dQ, dK, dV = new(H), new(H), new(Hk), new(Hk)
        lse = torch.full((B, H, n), -math.inf, dtype=torch.float64, device="cuda")
        for b in range(B):
            r = slice(0, lens[b])
            for h in range(H):
                q, g = s.Q[b, h, r].double(), s.dO[b, h, r].double()
                k, v = s.K[b, h // G, r].double(), s.V[b, h // G, r].double()
                o, lse[b, h, r], f = _exact_rows(q, k, v, 0, s.scale, window, sinks)
                p = f * (g @ v.t() - (g * o).sum(1, keepdim=True))
                O[b, h, r], dQ[b, h, r] = o, s.scale * (p @ k)
                dK[b, h // G, r] += s.scale * (p.t() @ q)
                dV[b, h // G, r] += f.t() @ g
        return O, lse, dQ, dK, dV
    page, lens, ptr, table = case["page"], s.lens.tolist(), s.q_ptr.tolist(), s.table.long()

    def rows(pages, exps, b, first, last):  # positions first .. last - 1 of sequence b: [token, kv head, d]
        at = torch.arange(first, last, device="cuda")
        x = pages.float()[table[b, at // page], :, at % page].double()
        return x if exps is None else x * _two_to(exps[table[b, at // page], :, at % page].long() - 127)[..., None]

    if case["op"] == "write":
        K, V = s.K_pages.double(), s.V_pages.double()
        (k, _), (v, _) = ((s.K.double(), 0), (s.V.double(), 0)) if s.K_exp is None else (_exact_codes(s.K.double()), _exact_codes(s.V.double()))
        for b in range(B):
            at = torch.arange(lens[b] - (ptr[b + 1] - ptr[b]), lens[b], device="cuda")
            K[table[b, at // page], :, at % page] = k[ptr[b]:ptr[b + 1]]
            V[table[b, at // page], :, at % page] = v[ptr[b]:ptr[b + 1]]
        return (K, V) if s.K_exp is None else (K, V, None, None)
    if case["op"] == "read":
        span = [(b, lens[b] - (ptr[b + 1] - ptr[b]), lens[b]) for b in range(B)]
        return tuple(torch.cat([rows(x, e, *at) for at in span]) for x, e in ((s.K_pages, s.K_exp), (s.V_pages, s.V_exp)))
    O = torch.zeros(s.total, H, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s.total, H, dtype=torch.float64, device="cuda")
    pages = [(x if e is None else x.double() * _two_to(e.long() - 127)[..., None]) for x, e in ((s.K_pages, s.K_exp), (s.V_pages, s.V_exp))]
    for b in range(B):
        r = slice(ptr[b], ptr[b + 1])
        at = torch.arange(lens[b], device="cuda")
        k, v = (x[table[b, at // page], :, at % page].double() for x in pages)
        first = lens[b] - (ptr[b + 1] - ptr[b])
        for h in range(H):
            O[r, h], lse[r, h], _ = _exact_rows(s.Q[r, h].double(), k[:, h // G], v[:, h // G], first, s.scale, window, sinks)
    return O, lse


# ------------------------------------------------------------------------------------------------------------- floors
def _visible(first, count, window, sinks):
    """Visible pairs of queries at positions first .. first + count - 1, and the number of keys that any of them sees."""
    pairs = 0
    for i in range(first, first + count):
        pairs += i + 1 if not window else min(i + 1, window) + max(0, min(sinks, i + 1 - window))
    last = first + count - 1
    start = max(0, first - window + 1) if window else 0
    return pairs, last + 1 - start + min(sinks, start)


def work(case):
    """Each input read once and each output written once (of a cache: the rows that some query sees), and the products of the
    visible pairs: two forward, five backward."""
    H, Hk, d, es = case["heads"], case["kv_heads"], case["d"], _SIZE[case["dtype"]]
    lens, new = _lengths(case)
    if case["op"] == "train":
        tokens, padded = float(sum(lens)), float(case["batch"] * case["n"])
        pairs = sum(_visible(0, l, case["window"], case["sinks"])[0] for l in lens)
        read, written = (2 * H + 2 * Hk) * d * es, (2 * H + 2 * Hk) * d * es + 4.0 * H
        return {"bytes": tokens * read + padded * written, "flops": 14.0 * pairs * H * d}
    row = 2.0 * Hk * (d * _SIZE[case["cache"]] + (1.0 if case["cache"] == "fp8" else 0.0))  # K and V of a cached token
    if case["op"] in ("write", "read"):
        # two operations for every value that is quantised (magnitude, scaling) or read back (scaling)
        return {"bytes": float(sum(new)) * (row + 2.0 * Hk * d * es), "flops": 4.0 * sum(new) * Hk * d}
    seen = [_visible(l - q, q, case["window"], case["sinks"]) for l, q in zip(lens, new)]
    return {"bytes": row * sum(k for _, k in seen) + float(sum(new)) * H * (2.0 * d * es + 4.0), "flops": 4.0 * sum(p for p, _ in seen) * H * d}
