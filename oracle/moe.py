"""CPU oracle of the norms around a block and of a mixture of experts -- TEST INFRASTRUCTURE.

Plain numpy in 64 bits, written from the definitions of include/kmq.h; it shares no code with the GPU library.
bf16 values are held as uint16 bit patterns, as everywhere in the tests.
"""
from __future__ import annotations

import numpy as np

from oracle.kv import bf16_value

BLOCK = 64


def _f32(x):
    return float(np.float32(x))


def block_norm(x, residual=None, gate=None, post_gain=None, pre_gain=None, scale=1.0, residual_scale=1.0, eps=0.0, post_norm=False, gate_sigmoid=False):
    """(out, normed) in 64 bits, not rounded; x, residual, gate: rows of patterns, gate also one row for all."""
    with np.errstate(all="ignore"):
        unit = lambda v, g: v / np.sqrt((v * v).mean(-1, keepdims=True) + _f32(eps)) * (1.0 if g is None else bf16_value(g))  # noqa: E731
        n = bf16_value(x)
        if post_norm:
            n = unit(n, post_gain)
        if gate is not None:
            g = bf16_value(gate)
            n = n * (1 / (1 + np.exp(-g)) if gate_sigmoid else g)
        s = _f32(scale) * n
        if residual is not None:
            s = s + _f32(residual_scale) * bf16_value(residual)
        return s, unit(s, pre_gain)


def route(x, weights, top_k, sigmoid=False, bias=None, groups=1, top_groups=1, normalise=True, scale=1.0):
    """(ids, gates in 64 bits) of every row."""
    experts, size = weights.shape[0], weights.shape[0] // groups
    with np.errstate(all="ignore"):
        logits = bf16_value(x) @ bf16_value(weights).T
        if sigmoid:
            s = 1 / (1 + np.exp(-logits))
        else:
            e = np.exp(logits - logits.max(-1, keepdims=True))
            s = e / e.sum(-1, keepdims=True)
        c = s if bias is None else s + np.asarray(bias, dtype=np.float32).astype(np.float64)
    number = np.where(np.isnan(c), -np.inf, c)
    ids, gates = np.zeros((len(x), top_k), dtype=np.int32), np.zeros((len(x), top_k))
    for row in range(len(x)):
        two = np.sort(number[row].reshape(groups, size), axis=1)[:, -2:].sum(1)
        best = sorted(range(groups), key=lambda g: (-two[g], g))[:top_groups]
        order = sorted((e for e in range(experts) if e // size in best), key=lambda e: (bool(np.isnan(c[row, e])), -number[row, e], e))[:top_k]
        w = s[row, order]
        if normalise:
            w = np.zeros(top_k) if w.sum() == 0 else w / w.sum()
        ids[row], gates[row] = order, w * _f32(scale)
    return ids, gates


def matrix(idx, codebook, scales):
    """Indices (N, K), codebook patterns and scale patterns (N, K / 64) -> the matrix in 64 bits."""
    return bf16_value(codebook)[idx] * np.repeat(bf16_value(scales), BLOCK, axis=1)


def experts(x, ids, gates, matrices, residual=None):
    """matrices[e] = (gate, up, down) in 64 bits.  Returns y, and what bounds its error: a list over the pairs that count of
    (token, weight, products and their absolute sums) -- see tolerance.moe_bound."""
    v = bf16_value(x)
    pairs = []
    y = np.zeros((len(x), matrices[next(iter(matrices))][2].shape[0])) if residual is None else bf16_value(residual).copy()
    with np.errstate(all="ignore"):
        for token in range(len(x)):
            for e in sorted(set(int(i) for i in ids[token])):
                if e not in matrices:
                    continue
                w = float(sum(np.float64(g) for i, g in zip(ids[token], gates[token]) if i == e))
                G, U, D = matrices[e]
                g, u = G @ v[token], U @ v[token]
                h = g / (1 + np.exp(-g)) * u
                y[token] += w * (D @ h)
                pairs.append(dict(token=token, expert=e, weight=w, g=g, u=u, h=h, g_size=np.abs(G) @ np.abs(v[token]), u_size=np.abs(U) @ np.abs(v[token])))
    return y, pairs
