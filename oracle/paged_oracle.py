"""Float64 CPU definition of the cache in pages: the FP4 and E4M3 rows, writing and reading rows, attention over them.

TEST INFRASTRUCTURE ONLY, as dapq_oracle.  A pool is a dict of numpy arrays as they lie in memory: "k" and "v" are bf16
bits uint16 [layers][n_pages][heads][page_rows][128], or codes uint8 [...][64] (FP4) or [...][128] (E4M3) with "k_scales",
"v_scales" uint8 [...][4].  Every function changes copies.
"""
from __future__ import annotations

import numpy as np

from .dapq_oracle import bf16_bits_to_f64, f64_to_bf16_bits, rope_apply

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def fp4_quantise(x):
    """Float64 rows [..., 128] -> codes uint8 [..., 64], scale bytes uint8 [..., 4].

    Per group of 32 channels the least e in [-125, 125] with max |x| <= 7 * 2^e; each value the level nearest to x / 2^e,
    of two the one with the even code, at most 6.  Groups that are not finite: scale byte 255, codes 0."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(x.shape[:-1] + (4, 32))
    bad = ~np.isfinite(g).all(-1)
    g0 = np.where(bad[..., None], 0.0, g)
    largest = np.abs(g0).max(-1)
    e = np.full(largest.shape, -125)
    for candidate in range(-124, 126):
        e = np.where(largest > 7.0 * 2.0 ** (candidate - 1), candidate, e)
    y = np.abs(g0) / (2.0 ** e)[..., None]
    distance = np.abs(y[..., None] - LEVELS)
    nearest = distance == distance.min(-1, keepdims=True)
    prefer = np.array([1, 0, 1, 0, 1, 0, 1, 0])                 # of two nearest levels the even code
    code = np.argmax(nearest * (1 + prefer), -1) + np.where(np.signbit(g0), 8, 0)
    code = np.where(bad[..., None], 0, code).reshape(x.shape)
    codes = (code[..., 0::2] | (code[..., 1::2] << 4)).astype(np.uint8)
    return codes, np.where(bad, 255, e + 127).astype(np.uint8)


def fp4_values(codes, scales):
    """The values that codes and scale bytes stand for, float64 [..., 128]."""
    codes = np.asarray(codes)
    c = np.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[:-1] + (128,)).astype(np.int64)
    two = np.where(np.asarray(scales) == 255, np.nan, 2.0 ** (np.asarray(scales).astype(np.float64) - 127.0))
    return np.where(c >= 8, -1.0, 1.0) * LEVELS[c & 7] * np.repeat(two, 32, -1)


# Magnitudes of the E4M3 codes 0 .. 126: E = 0 counts as E = 1 without the leading 8.  127 is no number.
E4M3_LEVELS = np.array([(m if e == 0 else 8 + m) * 2.0 ** (max(e, 1) - 10) for e in range(16) for m in range(8)][:127])


def e4m3_quantise(x):
    """Float64 rows [..., 128] -> codes uint8 [..., 128], scale bytes uint8 [..., 4].

    Per group of 32 channels the least e in [-117, 119] with max |x| <= 464 * 2^e; each value the level nearest to x / 2^e, of
    two the one with the even code, at most 448.  Groups that are not finite: scale byte 255, codes 0."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(x.shape[:-1] + (4, 32))
    bad = ~np.isfinite(g).all(-1)
    g0 = np.where(bad[..., None], 0.0, g)
    largest = np.abs(g0).max(-1)
    e = np.full(largest.shape, -117)
    for candidate in range(-116, 120):
        e = np.where(largest > 464.0 * 2.0 ** (candidate - 1), candidate, e)
    y = np.abs(g0) / (2.0 ** e)[..., None]
    above = np.clip(np.searchsorted(E4M3_LEVELS, y), 1, 126)
    to_low, to_high = y - E4M3_LEVELS[above - 1], E4M3_LEVELS[above] - y
    code = np.where((to_high < to_low) | ((to_high == to_low) & (above % 2 == 0)), above, above - 1)  # of two nearest levels the even code
    code = code + np.where(np.signbit(g0), 128, 0)
    return np.where(bad[..., None], 0, code).reshape(x.shape).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def e4m3_values(codes, scales):
    """The values that codes and scale bytes stand for, float64 [..., 128]."""
    c = np.asarray(codes).astype(np.int64)
    two = np.where(np.asarray(scales) == 255, np.nan, 2.0 ** (np.asarray(scales).astype(np.float64) - 127.0))
    return np.where(c >= 128, -1.0, 1.0) * np.append(E4M3_LEVELS, np.nan)[c & 127] * np.repeat(two, 32, -1)


def code_values(codes, scales):
    """Of the format whose rows have as many bytes."""
    return (fp4_values if np.asarray(codes).shape[-1] == 64 else e4m3_values)(codes, scales)


def place(table, n_pages, page_rows, seq, i):
    """(page, slot) of row i of a sequence, or None if it is on no page."""
    if i < 0 or i >= table.shape[1] * page_rows:
        return None
    page = int(table[seq, i // page_rows])
    return (page, i % page_rows) if 0 <= page < n_pages else None


def put(pool, name, layer, head, where, bits):
    """One bf16 row (bits [128]) into the pool, in place."""
    page, slot = where
    if name + "_scales" in pool:
        quantise = fp4_quantise if pool[name].shape[-1] == 64 else e4m3_quantise
        codes, scales = quantise(bf16_bits_to_f64(bits))
        pool[name][layer, page, head, slot] = codes
        pool[name + "_scales"][layer, page, head, slot] = scales
    else:
        pool[name][layer, page, head, slot] = bits


def value(pool, name, layer, head, where):
    """One row of the pool, float64 [128]."""
    page, slot = where
    row = pool[name][layer, page, head, slot]
    return code_values(row, pool[name + "_scales"][layer, page, head, slot]) if name + "_scales" in pool else bf16_bits_to_f64(row)


def _shape(pool):
    layers, n_pages, heads, page_rows = pool["k"].shape[:4]
    return layers, n_pages, heads, page_rows


def copy(pool):
    return {n: a.copy() for n, a in pool.items()}


def gather(pool, table, k_bits, v_bits, cu_seqlens, idx, count):
    """k_bits, v_bits [layers][tokens][heads][128]; idx [layers][batch][heads][budget]; count [layers][batch][heads]."""
    pool = copy(pool)
    layers, n_pages, heads, page_rows = _shape(pool)
    for layer, seq, head in np.ndindex(count.shape):
        start, length = int(cu_seqlens[seq]), int(cu_seqlens[seq + 1] - cu_seqlens[seq])
        for i in range(min(int(count[layer, seq, head]), idx.shape[3])):
            j, where = int(idx[layer, seq, head, i]), place(table, n_pages, page_rows, seq, i)
            if where is not None and 0 <= j < length:
                put(pool, "k", layer, head, where, k_bits[layer, start + j, head])
                put(pool, "v", layer, head, where, v_bits[layer, start + j, head])
    return pool


def append(pool, table, lengths, cu_new, max_new, k_bits, v_bits, positions, theta, pairing="half"):
    """k_bits, v_bits [layers][total_new][heads][128] before the rotation."""
    pool = copy(pool)
    layers, n_pages, heads, page_rows = _shape(pool)
    for layer in range(layers):
        k = k_bits[layer] if positions is None else rope_apply(k_bits[layer], positions, theta, pairing)
        for seq in range(len(lengths)):
            for t in range(min(int(cu_new[seq + 1] - cu_new[seq]), max_new)):
                where = place(table, n_pages, page_rows, seq, int(lengths[seq]) + t)
                for head in range(heads):
                    if where is not None:
                        put(pool, "k", layer, head, where, k[cu_new[seq] + t, head])
                        put(pool, "v", layer, head, where, v_bits[layer, cu_new[seq] + t, head])
    return pool


def read(pool, table, lengths, max_rows, fill):
    """(k_out, v_out) bf16 bits [layers][batch][heads][max_rows][128]; rows that are not read hold `fill`."""
    layers, n_pages, heads, page_rows = _shape(pool)
    out = []
    for name in ("k", "v"):
        got = np.full((layers, len(lengths), heads, max_rows, 128), fill, dtype=np.uint16)
        for layer, seq, head in np.ndindex(got.shape[:3]):
            for i in range(min(int(lengths[seq]), max_rows)):
                where = place(table, n_pages, page_rows, seq, i)
                if where is not None:
                    got[layer, seq, head, i] = f64_to_bf16_bits(value(pool, name, layer, head, where))
        out.append(got)
    return tuple(out)


def attention(pool, table, lengths, cu_new, q, scale, softcap=0.0):
    """q float64 [layers][total_new][n_q_heads][128].  Returns (out, weighted, logit): the output in the same shape, the same
    sum over |v| in its place, and for every (layer, token, query head) the largest sum over |q_c k_c| * scale (finite k_c), of
    which a logit's rounding errors are a small part."""
    layers, n_pages, heads, page_rows = _shape(pool)
    group = q.shape[2] // heads
    out, weighted, size = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:3])
    for layer in range(layers):
        for seq in range(len(lengths)):
            new = int(cu_new[seq + 1] - cu_new[seq])
            rows = [i for i in range(int(lengths[seq]) + new) if place(table, n_pages, page_rows, seq, i) is not None]
            at = np.array(rows, dtype=np.int64)
            for head in range(heads):
                if not rows or not new:
                    continue
                pages, slots = table[seq, at // page_rows], at % page_rows
                k, v = (code_values(pool[n][layer, pages, head, slots], pool[n + "_scales"][layer, pages, head, slots])
                        if n + "_scales" in pool else bf16_bits_to_f64(pool[n][layer, pages, head, slots]) for n in ("k", "v"))
                for t in range(new):
                    r, seen = int(cu_new[seq]) + t, at <= int(lengths[seq]) + t
                    if not seen.any():
                        continue
                    for h in range(head * group, (head + 1) * group):
                        x = k[seen] @ q[layer, r, h] * scale
                        if softcap:
                            x = softcap * np.tanh(x / softcap)
                        with np.errstate(invalid="ignore"):
                            w = np.exp(x - x.max())
                            w = w / w.sum()
                            out[layer, r, h] = w @ v[seen]
                            weighted[layer, r, h] = w @ np.abs(v[seen])
                        size[layer, r, h] = (np.where(np.isfinite(k[seen]), np.abs(k[seen]), 0.0) @ np.abs(q[layer, r, h])).max() * scale
    return out, weighted, size
