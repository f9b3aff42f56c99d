"""A network block with attention: what a decoder layer that attends to an encoder's states does."""
from __future__ import annotations

import numpy as np

from .model import Builder, Workload, rope_frequencies


def decoder_block(seed: int = 0, batch: int = 2, heads: int = 4, kv_heads: int = 2, d: int = 8, tokens: int = 6, states: int = 9,
                  width: int = 24, state_width: int = 20, lengths=None) -> Workload:
    """Tokens [batch, width, 1, tokens] attend to states [batch, state_width, 1, states] (1 x 1 projections, norm and rotation of
    the heads of queries and keys, heads that share keys, key counts), a residual sum, then to each other (rotated pairs
    interleaved, a part of the head; no mask: every token reads every other). Inputs: the tokens, the states, positions of both, the states that count for each image
    (``lengths``; default: all but two of the first image's, none of the others')."""
    rng = np.random.default_rng(seed)
    b = Builder("decoder_block")
    x = b.input(batch, width, 1, tokens)
    memory, at, at_memory, counts = b.input(batch, state_width, 1, states), b.input(1, 1, 1, tokens), b.input(batch, 1, 1, states), b.input(batch, 1, 1, 1)
    x = b.conv1x1(x, heads * d)
    f = rope_frequencies(d)
    q = b.head_rope(x, at, heads, f)
    k = b.head_rope(b.conv1x1(memory, kv_heads * d), at_memory, kv_heads, f)
    y = b.attention(q, k, b.conv1x1(memory, kv_heads * d), heads, kv_heads, counts)
    y = b.add_n([b.conv1x1(y, heads * d), x])
    s = b.head_rope(b.conv1x1(y, heads * d), at, heads, f[:2], norm=False, interleaved=True)
    b.attention(s, s, b.conv1x1(y, heads * d), heads)
    b.draw_weights(rng, "he", "random")
    w = b.finish(rng)
    counted = [states - 2] + [0] * (batch - 1) if lengths is None else lengths
    w.inputs = {memory: rng.standard_normal((batch, state_width, 1, states)).astype(np.float32),
                at: np.arange(tokens, dtype=np.float32).reshape(1, 1, 1, -1) + 100,
                at_memory: rng.integers(0, 50, (batch, 1, 1, states)).astype(np.float32),
                counts: np.array(counted, np.float32).reshape(batch, 1, 1, 1)}
    return w
