"""CPU oracle for the logit processing calls and the token counts (plain numpy, double precision, written from the
definitions in the C header).

TEST INFRASTRUCTURE.  Only tests may import this module; the product never does.

Section 4 leaves the sampling method to the user; what the calls compute is stated in the header: penalties for used
tokens with the drafted ones among them, biases, masks, a temperature, and then top-k, top-p and min-p on the values as they
are stored.  ``process_row`` and ``cut_row`` take one row; nothing here works on bits, keys or histograms.
"""

from __future__ import annotations

import math

import numpy as np


def bit(words: np.ndarray, t: int) -> bool:
    return bool(int(words[t // 32]) >> (t % 32) & 1)


def context(parent, row: int):
    """The drafted tokens' places before target row `row`: all in front of it, or on a tree its node and that one's ancestors."""
    if parent is None:
        return list(range(row))
    out, j = [], row - 1
    while j >= 0:
        out.append(j)
        p = int(parent[j])
        j = p if -1 <= p < j else -1
    return out


def context_row(parent, side: str, r: int) -> int:
    if side == "target" or parent is None:
        return r
    p = int(parent[r])
    return (p if -1 <= p < r else -1) + 1


def process_row(x, counts=None, seen=None, drafted=(), repetition=None, frequency=None, presence=None, biases=(), allowed=None,
                temperature=None):
    """(values, size) of one row in double precision, before they are stored: `size` is the largest magnitude a value went
    through, for the rounding errors of a single-precision evaluation.  drafted: the tokens before the row, biases:
    (token, value) pairs of which the last for a token counts."""
    x = np.array(x, dtype=np.float64)
    V = x.size
    size = np.abs(x)
    if repetition is not None or frequency is not None or presence is not None:
        n = np.zeros(V) if counts is None else counts.astype(np.float64).copy()
        used = np.zeros(V, dtype=bool) if seen is None else np.array([bit(seen, t) for t in range(V)])
        for t in drafted:
            if 0 <= t < V:
                n[t] += 1
                used[t] = True
        with np.errstate(invalid="ignore", over="ignore"):
            if repetition is not None:
                r = float(np.float32(repetition))
                x[used] = np.where(x[used] > 0, x[used] / r, x[used] * r)
                size = np.maximum(size, np.abs(x))
            if frequency is not None:
                f = float(np.float32(frequency))
                x = x - f * n
                size = size + np.abs(f * n)
            if presence is not None:
                x = x - float(np.float32(presence)) * (n > 0)
                size = size + abs(float(np.float32(presence)))
    last = {}
    for t, v in biases:
        if 0 <= t < V:
            last[int(t)] = float(np.float32(v))
    for t, v in last.items():
        x[t] += v
        size[t] += abs(v)
    if temperature is not None and temperature > 0:
        with np.errstate(invalid="ignore"):
            x = x / float(np.float32(temperature))
            size = size / float(np.float32(temperature))
    if allowed is not None:
        for t in range(V):
            if not bit(allowed, t):
                x[t] = -np.inf
    return x, size


def kept(y, top_k=None, top_p=None, min_p=None):
    """Which tokens of a row of stored values are kept: a truth value each."""
    y = np.asarray(y, dtype=np.float64)
    V = y.size
    if np.isnan(y).any() or np.isposinf(y).any() or not np.isfinite(y).any():
        return np.ones(V, dtype=bool)
    order = np.argsort(-y, kind="stable")
    if top_k is not None and 0 < top_k < V:
        order = order[:top_k]
    first = y[order[0]]
    with np.errstate(under="ignore"):
        w = np.exp(y[order] - first)
    keep = np.ones(order.size, dtype=bool)
    if top_p is not None and np.float32(top_p) < 1:
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        keep &= before < float(np.float32(top_p)) * float(w.sum())
        keep[0] = True
    if min_p is not None and np.float32(min_p) > 0:
        keep &= y[order] - first >= math.log(min(float(np.float32(min_p)), 1.0))
    out = np.zeros(V, dtype=bool)
    out[order[keep]] = True
    return out


def build(prompts, outputs, V: int):
    """(counts, seen) of lists of prompt and generated tokens, a list a sequence."""
    B, W = len(prompts), (V + 31) // 32
    counts, seen = np.zeros((B, V), dtype=np.int32), np.zeros((B, W), dtype=np.uint32)
    for b in range(B):
        for t in outputs[b]:
            if 0 <= t < V:
                counts[b, t] += 1
        for t in [*prompts[b], *outputs[b]]:
            if 0 <= t < V:
                seen[b, t // 32] |= np.uint32(1 << (t % 32))
    return counts, seen


def append(counts, seen, tokens):
    """The state after the given tokens, a list a sequence."""
    counts, seen = counts.copy(), seen.copy()
    V = counts.shape[1]
    for b, more in enumerate(tokens):
        for t in more:
            if 0 <= t < V:
                counts[b, t] += 1
                seen[b, t // 32] |= np.uint32(1 << (t % 32))
    return counts, seen
