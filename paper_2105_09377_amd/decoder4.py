"""A stack of decoder layers whose weights and cache are held in 4 bits, as a fixed sequence of library calls.

Every layer is, for new tokens x of every sequence:

* queries, keys and values: `compute dotProd (cartProd x w)` with MX4 weights (`mx4_weight_dot`);
* the keys and values go into the layer's paged cache (`mx4_cache_append`), over which the queries attend (`mx4_attend`);
* a projection back, added to x (`pair_reduce`), then two products with ReLU between them, added likewise.

Prompts may run these two products on 4-bit activations (`quantize_rows`: from that many tokens on): `mx4_quantize` and `mx4_dot`,
which the matrix units multiply at the rate of 4-bit numbers.  This module only sequences calls and owns the weights and caches; it does no
arithmetic.  No norms and no positions: the stack exercises the operators that the library has, at the shapes of such layers.
"""

from __future__ import annotations

from typing import Dict, List, Optional

import torch

from . import binding as gs

NAMES = ("q", "k", "v", "o", "up", "down")


def weight_shapes(width: int, heads: int, kv_heads: int, head_dim: int, hidden: int) -> Dict[str, tuple]:
    """Rows of a layer's weights: outputs, inputs."""
    return {"q": (heads * head_dim, width), "k": (kv_heads * head_dim, width), "v": (kv_heads * head_dim, width),
            "o": (width, heads * head_dim), "up": (hidden, width), "down": (width, hidden)}


class Decoder4Stack:
    def __init__(self, layers: List[Dict[str, torch.Tensor]], heads: int, kv_heads: int, head_dim: int, n_pages: int, page_size: int,
                 window: int = 0, sinks: int = 0, quantize_rows: Optional[int] = None, device="cuda:0"):
        self.dev = torch.device(device)
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.window, self.sinks, self.quantize_rows = window, sinks, quantize_rows
        self.layers = [{name: gs.mx4_quantize(w[name].to(self.dev)) for name in NAMES} for w in layers]
        self.caches = [gs.mx4_cache(n_pages, kv_heads, page_size, head_dim, self.dev) for _ in layers]

    def step(self, x: torch.Tensor, table: torch.Tensor, first: torch.Tensor, lengths: torch.Tensor) -> torch.Tensor:
        """Tokens x (batch, T, width), bfloat16, at positions first[b] .. lengths[b] - 1 = first[b] + T - 1 -> the stack's outputs."""
        batch, tokens, width = x.shape
        bf16 = torch.bfloat16
        rows = x.view(batch * tokens, width)
        small = self.quantize_rows is not None and rows.shape[0] >= self.quantize_rows
        for w, cache in zip(self.layers, self.caches):
            q = gs.mx4_weight_dot(rows, w["q"], out_dtype=bf16).view(batch, tokens, self.heads, self.head_dim)
            k = gs.mx4_weight_dot(rows, w["k"], out_dtype=bf16).view(batch, tokens, self.kv_heads, self.head_dim)
            v = gs.mx4_weight_dot(rows, w["v"], out_dtype=bf16).view(batch, tokens, self.kv_heads, self.head_dim)
            gs.mx4_cache_append(cache, table, first, k, v)
            a = gs.mx4_attend(q, cache, table, lengths, scale=self.head_dim ** -0.5, window=self.window, sinks=self.sinks)
            a = gs.mx4_weight_dot(a.view(rows.shape[0], self.heads * self.head_dim), w["o"], out_dtype=bf16)
            rows = gs.pair_reduce(rows, a)
            if small:
                h = gs.mx4_dot(gs.mx4_quantize(rows), w["up"], out_dtype=bf16, act=gs.GS_ACT_RELU)
                h = gs.mx4_dot(gs.mx4_quantize(h), w["down"], out_dtype=bf16)
            else:
                h = gs.mx4_weight_dot(rows, w["up"], out_dtype=bf16, act=gs.GS_ACT_RELU)
                h = gs.mx4_weight_dot(h, w["down"], out_dtype=bf16)
            rows = gs.pair_reduce(rows, h)
        return rows.view(batch, tokens, width)
