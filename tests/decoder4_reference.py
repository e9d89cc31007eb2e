"""The stack of 4-bit decoder layers from its definition in float64, with weights that make each part count: scores of some units, so that few
tokens have most of the weight, and branches of the size of what they are added to.  Results of calls are rounded to bfloat16, as the
stack's are.  Mistakes that a stack could make can be planted, and the rest of the kernels' rounding added."""

import functools

import numpy as np
import torch

from helpers import to_oracle
from oracle import mx4
from paper_2105_09377_amd import decoder4, synth

WIDTH, HEADS, KV, DIM, HIDDEN = 320, 8, 2, 64, 700
TOKENS, PIECES = 70, (6, 1, 1, 40, 21, 1)
# by layer: what the second one is given has grown
GAINS = ({"q": 1.5, "k": 1.5, "v": 1.5, "o": 1.5, "up": 1.5, "down": 1.0}, {"q": 0.6, "k": 0.6, "v": 1.5, "o": 1.5, "up": 1.0, "down": 0.7})
MISTAKES = ("no attention", "no window", "no sinks", "sinks one too few", "window one too long", "a token does not see itself", "queries of zero",
            "keys and values of bfloat16", "no quantising", "quantising all the same", "one cache for both layers", "earlier pieces forgotten",
            "heads in another order", "no second product")


def layers(n):
    shapes = decoder4.weight_shapes(WIDTH, HEADS, KV, DIM, HIDDEN)
    return [{name: synth.normal_bf16(shape, GAINS[i][name] * shape[1] ** -0.5, 9500 + 10 * i + j) for j, (name, shape) in enumerate(shapes.items())}
            for i in range(n)]


def tokens(batch):
    return synth.normal_bf16((batch, TOKENS, WIDTH), 1.0, 9600)


def bf(x):
    return to_oracle(torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16))


def small(x):
    flat = x.reshape(-1, x.shape[-1])
    return mx4.dequantize(*mx4.quantize(flat), x.shape[-1]).reshape(x.shape)


@functools.lru_cache(maxsize=None)
def stored(n):
    """The layers' weights as they are held: quantised and read back."""
    return [{name: small(to_oracle(v)) for name, v in w.items()} for w in layers(n)]


def stack(n_layers, x, window, sinks, quantize, mistake=None, as_kernels=False):
    """All tokens x (T, width) of one sequence at once.  as_kernels: sums in fp32 and weights of the attention in bfloat16."""
    n = x.shape[0]

    def product(a, b):
        return (a.astype(np.float32) @ b.astype(np.float32).T).astype(np.float64) if as_kernels else a @ b.T

    if mistake == "no quantising":
        quantize = False
    if mistake == "quantising all the same":
        quantize = True
    i, t = np.arange(n)[:, None], np.arange(n)[None]
    wide = window + (mistake == "window one too long")
    few = 0 if mistake == "no sinks" else sinks - (mistake == "sinks one too few")
    seen = t <= i
    if window and mistake != "no window":
        seen = seen & ((i - t < wide) | (t < few))
    if mistake == "a token does not see itself":
        seen = seen & ((t < i) | (i == 0))
    if mistake == "earlier pieces forgotten":
        piece = np.repeat(np.arange(len(PIECES)), PIECES)
        seen = seen & (piece[:, None] == piece[None])
    first = None
    for w in stored(n_layers):
        q, k, v = (bf(product(x, w[name])).reshape(n, -1, DIM) for name in "qkv")
        if mistake == "queries of zero":
            q = 0 * q
        if mistake != "keys and values of bfloat16":
            k, v = small(k), small(v)
        if mistake == "one cache for both layers":
            first = first or (k, v)
            k, v = first
        order = np.repeat(np.arange(KV), HEADS // KV)
        if mistake == "heads in another order":
            order = np.tile(np.arange(KV), HEADS // KV)
        k, v = k[:, order], v[:, order]
        s = np.where(seen, np.einsum("ihd,thd->hit", q, k) * DIM ** -0.5, -np.inf)
        p = np.exp(s - s.max(-1, keepdims=True))
        if as_kernels:
            p = bf(p * 0.7)                  # (rounded at another place than at powers of two)
        a = bf(np.einsum("hit,thd->ihd", p / p.sum(-1, keepdims=True), v).reshape(n, -1))
        if mistake != "no attention":
            x = bf(x + bf(product(a, w["o"])))
        h = bf(np.maximum(product(small(x) if quantize else x, w["up"]), 0))
        if mistake != "no second product":
            x = bf(x + bf(product(small(h) if quantize else h, w["down"])))
    return x


def off(got, want, x):
    """The 2-norm of the difference, in that of what the stack adds to its input."""
    return np.linalg.norm(got - want) / np.linalg.norm(want - x)


# layers, window, sinks, quantised activations
STACKS = ((1, 0, 0, False), (1, 20, 3, False), (1, 0, 0, True), (1, 20, 3, True), (2, 0, 0, False), (2, 20, 3, False))


def allowed(x, n, window, sinks, quantize):
    """What the kernels' own rounding does here, half as much again: their sums and weights' rounding differ from the ones added here element by
    element, but not in the norm over all of a sequence's 22400 numbers.  Most of it is codes of quantised numbers that fall on the other side."""
    return 1.5 * off(stack(n, x, window, sinks, quantize, as_kernels=True), stack(n, x, window, sinks, quantize), x)
