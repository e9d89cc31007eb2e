"""A stack of decoder layers with 8-bit weights, norms and experts, over a 4-bit cache, as a fixed sequence of library calls.

Every layer is, for new tokens of every sequence, in their running sum x:

* a norm of x with the last layer's result added to it, in 8 bits (`f8_norm`), and queries, keys and values of it (`f8_dot`);
* the keys and values go into the layer's paged cache (`mx4_cache_append`), over which the queries attend (`mx4_attend`);
* a projection back (`f8_quantize`, `f8_dot`), which the next norm adds to x;
* experts: every token's choices sorted by expert (`expert_sort`), two products with ReLU between them for the rows of each expert
  (`f8_expert_dot`), and the rows joined with their weights (`expert_join`).

Which experts a token has, and their weights, is what a caller's `route` says of the norm's numbers.  This module only sequences calls and owns
the weights and caches; it does no arithmetic.  No positions.
"""

from __future__ import annotations

from typing import Callable, Dict, List, Tuple

import torch

from . import binding as gs

DENSE, EXPERTS, NORMS = ("q", "k", "v", "o"), ("up", "down"), ("norm_attention", "norm_experts")

# (layer, the second norm's tokens in F8) -> experts (tokens, choices), int32, and weights of them in float32
Route = Callable[[int, gs.F8], Tuple[torch.Tensor, torch.Tensor]]


def weight_shapes(width: int, heads: int, kv_heads: int, head_dim: int, hidden: int, experts: int) -> Dict[str, tuple]:
    """A layer's weights: rows are outputs, columns inputs; norms have a weight for each number."""
    return {"q": (heads * head_dim, width), "k": (kv_heads * head_dim, width), "v": (kv_heads * head_dim, width), "o": (width, heads * head_dim),
            "up": (experts, hidden, width), "down": (experts, width, hidden), "norm_attention": (width,), "norm_experts": (width,)}


class Decoder8Stack:
    def __init__(self, layers: List[Dict[str, torch.Tensor]], heads: int, kv_heads: int, head_dim: int, n_pages: int, page_size: int, route: Route,
                 eps: float = 1e-6, window: int = 0, sinks: int = 0, device="cuda:0"):
        self.dev = torch.device(device)
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.route, self.eps, self.window, self.sinks = route, eps, window, sinks
        self.layers = []
        for w in layers:
            held = {name: gs.f8_quantize(w[name].to(self.dev), block_rows=128) for name in DENSE + EXPERTS}
            held.update({name: w[name].to(self.dev) for name in NORMS})
            self.layers.append(held)
        self.caches = [gs.mx4_cache(n_pages, kv_heads, page_size, head_dim, self.dev) for _ in layers]

    def step(self, x: torch.Tensor, table: torch.Tensor, first: torch.Tensor, lengths: torch.Tensor) -> torch.Tensor:
        """Tokens x (batch, T, width), bfloat16, at positions first[b] .. lengths[b] - 1 = first[b] + T - 1 -> the stack's outputs."""
        batch, tokens, width = x.shape
        bf16 = torch.bfloat16
        rows, added = x.view(batch * tokens, width), None
        for i, (w, cache) in enumerate(zip(self.layers, self.caches)):
            y, rows = gs.f8_norm(rows, w["norm_attention"], residual=added, eps=self.eps)
            q = gs.f8_dot(y, w["q"], out_dtype=bf16).view(batch, tokens, self.heads, self.head_dim)
            k = gs.f8_dot(y, w["k"], out_dtype=bf16).view(batch, tokens, self.kv_heads, self.head_dim)
            v = gs.f8_dot(y, w["v"], out_dtype=bf16).view(batch, tokens, self.kv_heads, self.head_dim)
            gs.mx4_cache_append(cache, table, first, k, v)
            a = gs.mx4_attend(q, cache, table, lengths, scale=self.head_dim ** -0.5, window=self.window, sinks=self.sinks)
            a = gs.f8_dot(gs.f8_quantize(a.view(batch * tokens, self.heads * self.head_dim)), w["o"], out_dtype=bf16)
            y, rows = gs.f8_norm(rows, w["norm_experts"], residual=a, eps=self.eps)
            experts, weights = self.route(i, y)
            n_experts, hidden = w["up"].shape[:2]
            s = gs.expert_sort(experts, n_experts)
            # (rows of dropped choices, which no call below looks at, need not be zeros as in new results)
            up, down = (torch.empty(s.tokens.shape[0], n, dtype=bf16, device=x.device) for n in (hidden, width))
            h = gs.f8_expert_dot(y, w["up"], s.offsets, tokens=s.tokens, act=gs.GS_ACT_RELU, out=up)
            h = gs.f8_expert_dot(gs.f8_quantize(h), w["down"], s.offsets, out=down)
            added = gs.expert_join(h, s.places, weights)
        if added is not None:
            rows = gs.pair_reduce(rows, added)
        return rows.view(batch, tokens, width)
