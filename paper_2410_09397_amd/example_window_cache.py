"""Windowed attention in training, then served from a paged cache: `python -m paper_2410_09397_amd.example_window_cache`.

One attention layer with shared key heads is trained for some steps to give back the value of the token three places earlier, then
serves sequences that it has not seen: prompts enter a paged, quantised cache in chunks, further tokens one at a time, all sequences of a
batch together, and what comes out is set against one windowed forward over the whole sequences.
"""
import torch

from paper_2410_09397_amd import attn


class WindowAttention(torch.autograd.Function):
    """O = windowed attention of Q, K, V [batch, heads or kv_heads, n, d], differentiable."""

    @staticmethod
    def forward(ctx, Q, K, V, scale, window, sinks):
        O, LSE = attn.attn_win_fwd(Q, K, V, scale, window=window, sinks=sinks)
        ctx.save_for_backward(Q, K, V, O, LSE)
        ctx.rest = scale, window, sinks
        return O

    @staticmethod
    def backward(ctx, dO):
        Q, K, V, O, LSE = ctx.saved_tensors
        scale, window, sinks = ctx.rest
        dO = torch.empty_like(O).copy_(dO)  # (the gradients' layout is O's)
        return (*attn.attn_win_bwd(Q, K, V, O, dO, LSE, scale, window=window, sinks=sinks), None, None, None)


class Layer:
    def __init__(self, width, heads, kv_heads, d, window, sinks, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.heads, self.kv_heads, self.d, self.window, self.sinks, self.scale = heads, kv_heads, d, window, sinks, d ** -0.5
        new = lambda rows, cols: (torch.randn(rows, cols, generator=gen, device="cuda") * rows ** -0.5).requires_grad_()
        self.weights = [new(width, heads * d), new(width, kv_heads * d), new(width, kv_heads * d), new(heads * d, width)]

    def project(self, x):
        """Q, K, V [..., tokens, heads, d] of x [..., tokens, width]."""
        return [(x @ w).unflatten(-1, (-1, self.d)).to(torch.bfloat16) for w in self.weights[:3]]

    def train_forward(self, x):
        Q, K, V = (t.transpose(1, 2).contiguous() for t in self.project(x))
        O = WindowAttention.apply(Q, K, V, self.scale, self.window, self.sinks)
        return O.transpose(1, 2).flatten(2).float() @ self.weights[3]


def train(layer, steps, batch, n, width, lr=0.01, seed=1):
    """Losses of Adam steps on the task of giving back what stood three places earlier, with the place marked in the input."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    place = torch.randn(n + 3, width // 2, generator=gen, device="cuda")
    opt = torch.optim.Adam(layer.weights, lr=lr)
    losses = []
    for _ in range(steps):
        content = torch.randn(batch, n, width // 2, generator=gen, device="cuda")
        x = torch.cat([content, place[3:].expand(batch, -1, -1)], -1)
        want = torch.cat([torch.zeros_like(content[:, :3]), content[:, :-3]], 1)
        loss = (layer.train_forward(x)[..., :width // 2] - want).square().mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(float(loss.detach()))
    return losses


@torch.no_grad()
def serve(layer, x, prompts, chunk, page_size=16, quantised=True):
    """Attention outputs [tokens, heads * d] of every sequence of x (a list of [tokens, width]): the first prompts[b] tokens of sequence b in
    chunks, the others one at a time, all sequences together."""
    batch, lens = len(x), [0] * len(x)
    pages = [-(-t.shape[0] // page_size) for t in x]
    dtype = torch.float8_e4m3fn if quantised else torch.bfloat16
    K_pages, V_pages, K_exp, V_exp = attn.attn_cache_pages(sum(pages), layer.kv_heads, page_size, layer.d, dtype)
    table = torch.full((batch, max(pages)), -1, dtype=torch.int32)
    free = torch.randperm(sum(pages)).tolist()
    out = [[] for _ in x]
    while any(l < t.shape[0] for l, t in zip(lens, x)):
        new = [min(chunk, p - l) if l < p else min(1, t.shape[0] - l) for l, p, t in zip(lens, prompts, x)]
        rows = torch.cat([t[l:l + q] for t, l, q in zip(x, lens, new)])
        for b, q in enumerate(new):  # a page for the first token that needs it
            for i in range(-(-lens[b] // page_size), -(-(lens[b] + q) // page_size)):
                table[b, i] = free.pop()
            lens[b] += q
        on_gpu = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
        Q, K, V = layer.project(rows)
        where = dict(q_ptr=on_gpu([sum(new[:b]) for b in range(batch + 1)]), max_q=max(new), K_exp=K_exp, V_exp=V_exp)
        at = (K_pages, V_pages, table.cuda(), on_gpu(lens))
        attn.attn_cache_write(K, V, *at, **where)
        O, _ = attn.attn_paged_fwd(Q, *at, layer.scale, max_len=max(lens), window=layer.window, sinks=layer.sinks, **where)
        for b, o in enumerate(O.flatten(1).split(new)):
            out[b].append(o)
    # what the cache holds of the last sequence, back out of it
    n = lens[-1]
    K, V = attn.attn_cache_read(K_pages, V_pages, table[-1:].cuda(), on_gpu([n]), torch.bfloat16, n, K_exp=K_exp, V_exp=V_exp)
    return [torch.cat(o) for o in out], (K, V)


@torch.no_grad()
def whole(layer, x):
    """The same outputs of one sequence by one windowed forward."""
    Q, K, V = (t.transpose(0, 1)[None].contiguous() for t in layer.project(x))
    O, _ = attn.attn_win_fwd(Q, K, V, layer.scale, window=layer.window, sinks=layer.sinks)
    return O[0].transpose(0, 1).flatten(1), (K, V)


def main(steps=60, n=256, width=64, quantised=True):
    layer = Layer(width, heads=4, kv_heads=2, d=64, window=32, sinks=2)
    losses = train(layer, steps, batch=8, n=n, width=width)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    x = [torch.randn(t, width, generator=gen, device="cuda") for t in (n, n // 2 + 7, 5)]
    served, (K, V) = serve(layer, x, prompts=[n - 6, n // 2, 1], chunk=50, quantised=quantised)
    far = []
    for got, t in zip(served, x):
        want, (wK, _) = whole(layer, t)
        far.append(float((got.float() - want.float()).abs().max() / want.float().abs().max()))
    cache = float((K.float() - wK[0].transpose(0, 1).float()).abs().max() / wK.float().abs().max())
    print("loss %.3f -> %.3f" % (losses[0], losses[-1]))
    print("served against one forward, max error of each sequence:", " ".join("%.4f" % f for f in far))
    print("keys of the last sequence as the cache holds them: %.4f" % cache)
    return losses, far, cache


if __name__ == "__main__":
    main()
