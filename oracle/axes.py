"""TEST INFRASTRUCTURE: plain numpy oracle of position ids with axes and of the rotary embedding by them.

Positions are counted along each unpacked sequence (x, y^k) token by token; the embedding is the fp64
rotation of pairs (i, i + D/2).  Pinned by tests/test_oracle_axes_pins.py.  Shares no code with the CUDA library.
"""
from __future__ import annotations

import numpy as np

from .policy import sequences


def _count(tokens, number, spans, pos):
    """Numbers `tokens` from `number` on; returns the number behind them."""
    i = 0
    while i < len(tokens):
        t = tokens[i]
        if t in spans:
            f, h, w = spans[t]
            for k in range(f * h * w):
                pos[:, t + k] = number + k // (h * w), number + k // w % h, number + k % w
            number += max(f, h, w)
            i += f * h * w
        else:
            pos[:, t] = number
            number += 1
            i += 1
    return number


def position_ids(rows, span_start, span_grid):
    spans = {int(s): tuple(int(x) for x in g) for s, g in zip(span_start, span_grid)}
    groups = sequences(rows)
    pos = np.zeros((3, groups[-1][1][-1][-1] + 1), np.int64)
    for prompt, resp in groups:
        behind = _count(prompt, 0, spans, pos)
        for y in resp:
            _count(y, behind, spans, pos)
    return pos


def rope(x, pos, axis_of_freq, base, inverse=False):
    """x [T, H, D], pos [axes, T]: the rotated tensor in fp64."""
    x = np.asarray(x, np.float64)
    half = x.shape[-1] // 2
    angle = np.stack([np.asarray(pos, np.float64)[axis_of_freq[i]] * base ** (-2.0 * i / x.shape[-1])
                      for i in range(half)], 1)[:, None]
    if inverse:
        angle = -angle
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * np.cos(angle) - b * np.sin(angle), b * np.cos(angle) + a * np.sin(angle)], -1)
