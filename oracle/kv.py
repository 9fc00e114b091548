"""CPU oracle of the operators between the QKV product and the output product -- TEST INFRASTRUCTURE.

Plain numpy in 64 bits, written from the definitions of include/kmq.h; it shares no code with the GPU library.
bf16 values are held as uint16 bit patterns, as everywhere in the tests.
"""
from __future__ import annotations

import numpy as np

BLOCK = 64


def bf16_value(p):
    return (np.asarray(p, dtype=np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def round_bf16(x):
    """float64 -> float32 -> bf16 patterns, each to nearest even; a NaN stays one."""
    with np.errstate(over="ignore", invalid="ignore"):
        f = np.asarray(x, dtype=np.float64).astype(np.float32)
    u = f.view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(f), np.uint16(0x7FC0), r)


def turn(x, positions=None, inv_freq=None, rotary_dim=0, interleaved=False, rmsnorm=False, gain=None, eps=0.0):
    """Heads x (rows, heads, D; bf16 patterns) normalised and rotated, in 64 bits (not rounded)."""
    v = bf16_value(x)
    if rmsnorm:
        v = v / np.sqrt((v * v).mean(-1, keepdims=True) + float(np.float32(eps)))
        if gain is not None:
            v = v * bf16_value(gain)
    if rotary_dim:
        i = np.arange(rotary_dim // 2)
        left, right = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary_dim // 2)
        a = np.asarray(positions, dtype=np.float64)[:, None] * np.asarray(inv_freq, dtype=np.float32).astype(np.float64)[None]
        c, s = np.cos(a)[:, None], np.sin(a)[:, None]
        l, r = v[..., left].copy(), v[..., right].copy()
        v[..., left], v[..., right] = l * c - r * s, r * c + l * s
    return v


def boundaries(codebook):
    c = bf16_value(codebook).astype(np.float32)
    return ((c[:-1] + c[1:]) * np.float32(0.5)).astype(np.float64)


def quantize(x, codebook):
    """Rows of bf16 patterns (..., D) -> indices (..., D) and scale patterns (..., D / 64)."""
    x = np.asarray(x, dtype=np.uint16)
    blocks = x.reshape(*x.shape[:-1], -1, BLOCK)
    scale = (blocks & 0x7FFF).max(-1)
    unit = np.where(scale == 0, 1.0, bf16_value(scale))[..., None]
    v = bf16_value(blocks)
    idx = np.zeros(blocks.shape, dtype=np.int64)
    with np.errstate(invalid="ignore"):
        for b in boundaries(codebook):
            idx += v > b * unit
    return idx.reshape(x.shape), scale.astype(np.uint16)


def values(idx, scale, codebook):
    """The values that indices and scales stand for, in 64 bits."""
    v = bf16_value(codebook)[idx].reshape(*idx.shape[:-1], -1, BLOCK)
    return (v * bf16_value(scale)[..., None]).reshape(idx.shape)


class Pages:
    """Pages of a cache as bytes, addressed element by element as include/kmq.h specifies them."""

    def __init__(self, num_pages, page_size, kv_heads, head_dim, fill=None):
        self.num_pages, self.page_size, self.kv_heads, self.D = num_pages, page_size, kv_heads, head_dim
        self.page_bytes = kv_heads * (page_size // 16) * 17 * head_dim
        self.bytes = np.zeros(num_pages * self.page_bytes, dtype=np.uint8) if fill is None else np.array(fill, dtype=np.uint8)
        assert self.bytes.size == num_pages * self.page_bytes

    def places(self, page, token):
        """Byte addresses (heads, D) of a token's K and V nibbles with their shifts, and of the scales (heads, 2, D / 64)."""
        D = self.D
        tile = ((page * self.kv_heads + np.arange(self.kv_heads)) * (self.page_size // 16) + token // 16)[:, None] * 17 * D
        t, d = token % 16, np.arange(D)
        k = tile + ((d // 16 % 4) * 16 + t) * (D // 8) + (d // 64) * 8 + (d % 16) // 2
        v = tile + 8 * D + ((t // 4) * 16 + d % 16) * (D // 8) + (d // 32) * 4 + t % 4
        b = np.arange(D // BLOCK)
        s = np.stack([tile + 16 * D + ((t // 4 * 2 + kv) * (D // BLOCK) + b) * 8 + (t % 4) * 2 for kv in (0, 1)], 1)
        return k, 4 * (d % 2), v, 4 * (d % 32 // 16), s

    def write(self, page, token, k, v, codebooks):
        """One token's K and V rows (kv_heads, D; bf16 patterns)."""
        ka, ks, va, vs, sa = self.places(page, token)
        for x, a, shift, kv in ((k, ka, ks, 0), (v, va, vs, 1)):
            idx, scale = quantize(x, codebooks[kv])
            for nibble in (0, 4):
                at = np.broadcast_to(shift == nibble, a.shape)
                keep = 0xF0 if nibble == 0 else 0x0F
                self.bytes[a[at]] = (self.bytes[a[at]] & keep) | (idx[at] << nibble).astype(np.uint8)
            self.bytes[sa[:, kv]] = scale & 0xFF
            self.bytes[sa[:, kv] + 1] = scale >> 8

    def read(self, page, token, codebooks):
        """One token's K and V rows in 64 bits."""
        ka, ks, va, vs, sa = self.places(page, token)
        out = []
        for a, shift, kv in ((ka, ks, 0), (va, vs, 1)):
            scale = self.bytes[sa[:, kv]].astype(np.uint16) | self.bytes[sa[:, kv] + 1].astype(np.uint16) << 8
            with np.errstate(invalid="ignore"):
                out.append(values((self.bytes[a] >> shift & 15).astype(np.int64), scale, codebooks[kv]))
        return out


def place(table_row, page_size, num_pages, pos):
    """(page, token) of a position, or None where it is not in the cache."""
    if pos < 0 or pos // page_size >= len(table_row):
        return None
    page = int(table_row[pos // page_size])
    return (page, pos % page_size) if 0 <= page < num_pages else None


def sequence(pages, table_row, length, codebooks):
    """K and V (tokens, heads, D) of a sequence's positions below `length`, and which of them are in the cache."""
    n = max(0, min(length, len(table_row) * pages.page_size))
    k, v = np.zeros((n, pages.kv_heads, pages.D)), np.zeros((n, pages.kv_heads, pages.D))
    there = np.zeros(n, dtype=bool)
    for p in range(n):
        at = place(table_row, pages.page_size, pages.num_pages, p)
        if at is not None:
            there[p] = True
            k[p], v[p] = pages.read(*at, codebooks)
    return k, v, there


def attention(q, k, v, there, length, scale, causal=True, window=0):
    """q (rows, heads, D; bf16 patterns): a sequence's last rows.  Returns out, lse, sum p |v| / sum p, and the largest
    |scale| * sum |q k| of each (row, head) over the tokens that it sees."""
    qv = bf16_value(q)
    n, heads, D = qv.shape
    group = heads // k.shape[1]
    out, lse = np.zeros((n, heads, D)), np.full((n, heads), -np.inf)
    spread, size = np.zeros((n, heads, D)), np.zeros((n, heads))
    j = np.arange(k.shape[0])
    for i in range(n):
        p = length - n + i
        seen = there & ((j <= p) if causal else True)
        if window:
            seen = seen & (j > p - window)
        if not seen.any():
            continue
        for h in range(heads):
            ks, vs = k[seen, h // group], v[seen, h // group]
            s = scale * (ks @ qv[i, h])
            m = s.max()
            w = np.exp(s - m)
            out[i, h] = w @ vs / w.sum()
            spread[i, h] = w @ np.abs(vs) / w.sum()
            lse[i, h] = m + np.log(w.sum())
            size[i, h] = (abs(scale) * (np.abs(ks) @ np.abs(qv[i, h]))).max()
    return out, lse, spread, size
