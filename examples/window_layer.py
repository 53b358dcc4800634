"""One attention layer with positions, norms and a window, trained on packed prompts and then served from the ring that its window needs.

  train   q, k and v as views of one projection; rotate_heads norms and rotates q and k, prompt_attention with a window and first tokens
          that stay visible, torch's autograd through both
  serve   the prompts' keys and values, projected and rotated at once, into a WindowCache, then a token at a time: rotated by the cache's
          own count, through WindowCache.step, captured once and replayed

    python -m examples.window_layer [--prompts 1024,700,333,1] [--window 252] [--sinks 4] [--tokens 64]
"""
import argparse

import torch

from paper_2407_02328_amd import Rotary, WindowCache, prompt_attention, rotate_heads

DEV = "cuda:0"


class Layer:
    """x [tokens, hidden] -> attention -> [tokens, hidden]; weights in bf16, norms in fp32."""

    def __init__(self, hidden=1024, heads=16, kv_heads=4, head_dim=64, window=252, sinks=4, seed=0):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.heads, self.kv_heads, self.head_dim, self.window, self.sinks = heads, kv_heads, head_dim, window, sinks
        self.rotary = Rotary(head_dim)
        self.w_qkv = (torch.randn((hidden, (heads + 2 * kv_heads) * head_dim), generator=g, device=DEV) * hidden ** -0.5).bfloat16()
        self.w_out = (torch.randn((heads * head_dim, hidden), generator=g, device=DEV) * (heads * head_dim) ** -0.5).bfloat16()
        self.q_norm, self.k_norm = torch.ones(head_dim, device=DEV), torch.ones(head_dim, device=DEV)

    def parameters(self):
        return [self.w_qkv, self.w_out, self.q_norm, self.k_norm]

    def project(self, x, positions):
        """q, k, v [tokens, heads, head_dim] of tokens at `positions` (int32 [tokens])."""
        qkv = (x @ self.w_qkv).unflatten(-1, (-1, self.head_dim))
        q, k, v = qkv[:, :self.heads], qkv[:, self.heads:-self.kv_heads], qkv[:, -self.kv_heads:]
        q, k = rotate_heads(q, k, positions, self.rotary, q_weight=self.q_norm, k_weight=self.k_norm)
        return q, k, v

    def attend(self, q, k, v, start):
        return prompt_attention(q, k, v, q_start=start, k_start=start, rest=torch.is_grad_enabled(), window=self.window, sinks=self.sinks)[0]

    def __call__(self, x, start, positions):
        return self.attend(*self.project(x, positions), start).flatten(1) @ self.w_out


def packed(lengths):
    """Starts of sequences (int32 [batch + 1]) and positions of their tokens."""
    start = torch.tensor([0] + torch.tensor(lengths).cumsum(0).tolist(), dtype=torch.int32, device=DEV)
    return start, torch.cat([torch.arange(n, dtype=torch.int32, device=DEV) for n in lengths])


def train(layer: Layer, x, target, start, positions, steps: int, rate: float):
    """Steps down the gradient of the mean square distance to target by all weights; the losses."""
    losses = []
    for _ in range(steps):
        for w in layer.parameters():
            w.requires_grad_(True).grad = None
        loss = (layer(x, start, positions).float() - target).square().mean()
        loss.backward()
        losses.append(float(loss.detach()))
        with torch.no_grad():
            for w in layer.parameters():
                w.sub_((rate * w.grad.float()).to(w.dtype))
    for w in layer.parameters():
        w.requires_grad_(False).grad = None
    return losses


@torch.no_grad()
def serve(layer: Layer, x, start, positions, following):
    """The prompts into a ring, then `following` [tokens, batch, hidden] through it; the cache, and the attention's output per token
    [tokens, batch, heads, head_dim].  (What the prompts' own tokens answer, layer.attend of the same rows, is not asked for here.)"""
    _, k, v = layer.project(x, positions)
    batch = following.shape[1]
    cache = WindowCache(batch=batch, heads=layer.heads, kv_heads=layer.kv_heads, head_dim=layer.head_dim, window=layer.window, sinks=layer.sinks,
                        dtype=x.dtype)
    token = following[0].clone()

    def step():
        q, k, v = layer.project(token, cache.positions)
        return cache.step(q, k, v.contiguous())

    # the first launches load the kernels, which a capture must not
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        answer = step()
    cache.fill(k, v, k_start=start)
    outs = []
    for x_n in following:
        token.copy_(x_n)
        graph.replay()
        outs.append(answer.clone())
    return cache, torch.stack(outs)


@torch.no_grad()
def all_at_once(layer: Layer, x, start, following):
    """What serve() answers, with every sequence as one prompt."""
    bounds, t = start.tolist(), following.shape[0]
    outs = []
    for b, (s, e) in enumerate(zip(bounds, bounds[1:])):
        whole, positions = packed([e - s + t])
        outs.append(layer.attend(*layer.project(torch.cat([x[s:e], following[:, b]]), positions), whole)[e - s:])
    return torch.stack(outs, 1)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--prompts", default="1024,700,333,1", help="lengths of the packed prompts")
    ap.add_argument("--window", type=int, default=252, help="keys up to its own that a query sees")
    ap.add_argument("--sinks", type=int, default=4, help="first tokens that stay visible")
    ap.add_argument("--tokens", type=int, default=64, help="tokens to serve behind the prompts")
    ap.add_argument("--steps", type=int, default=20, help="training steps")
    args = ap.parse_args()
    lengths = [int(n) for n in args.prompts.split(",")]
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    layer = Layer(window=args.window, sinks=args.sinks)
    start, positions = packed(lengths)
    x = torch.randn((sum(lengths), 1024), generator=g, device=DEV).bfloat16()
    losses = train(layer, x, x.float().roll(1, 0), start, positions, args.steps, 100.0)
    print(f"training: mean square {losses[0]:.4f} -> {losses[-1]:.4f} in {args.steps} steps")
    following = torch.randn((args.tokens, len(lengths), 1024), generator=g, device=DEV).bfloat16()
    cache, outs = serve(layer, x, start, positions, following)
    want = all_at_once(layer, x, start, following).float()
    rows = 2 * layer.kv_heads * layer.head_dim * 2 * (sum(lengths) + args.tokens * len(lengths))
    print(f"serving: {args.tokens} tokens behind {len(lengths)} prompts, cache {cache.cache.nbytes / 1024:.0f} KB (all rows: {rows / 1024:.0f} KB), "
          f"output off by {float((outs.float() - want).norm() / want.norm()):.4f} of its norm from the prompts' pass")


if __name__ == "__main__":
    main()
