"""Float64 CPU definition of the blocks of a cache in pages: bounds of their keys, the blocks that a token reads, attention over them.

TEST INFRASTRUCTURE ONLY, as dapq_oracle.  Pools are those of paged_oracle; bounds are int8 [layers][n_pages][heads][page_rows / block_rows][2][128]
(upper, lower), scales uint8 without the last two axes.  Every function changes copies.
"""
from __future__ import annotations

import numpy as np

from .dapq_oracle import bf16_bits_to_f64
from .paged_oracle import code_values, place


def rows_of(pool, name, layer, head, where):
    """Rows of the pool, float64 [n][128], at (page, slot) each."""
    pages, slots = (np.array(x, dtype=np.int64) for x in zip(*where))
    row = pool[name][layer, pages, head, slots]
    return code_values(row, pool[name + "_scales"][layer, pages, head, slots]) if name + "_scales" in pool else bf16_bits_to_f64(row)


def unit(largest):
    """The least e in [-50, 50] with largest <= 127 * 2^e (50 where there is none)."""
    for e in range(-50, 50):
        if largest <= 127.0 * 2.0 ** e:
            return e
    return 50


def block_bounds(keys):
    """Keys float64 [rows][128] -> (upper, lower int8 [128], scale byte)."""
    if not np.isfinite(keys).all():
        return np.zeros(128, np.int8), np.zeros(128, np.int8), 255
    e = unit(np.abs(keys).max())
    upper = np.clip(np.ceil(keys.max(0) / 2.0 ** e), -127, 127)
    lower = np.clip(np.floor(keys.min(0) / 2.0 ** e), -127, 127)
    return upper.astype(np.int8), lower.astype(np.int8), e + 127


def bounds(pool, table, block_rows, first, lengths, max_rows, old, old_scales):
    out, scales = old.copy(), old_scales.copy()
    layers, n_pages, heads, page_rows = pool["k"].shape[:4]
    for seq in range(len(lengths)):
        begin = max(0, int(first[seq])) if first is not None else 0
        end = min(int(lengths[seq]), begin + max_rows, table.shape[1] * page_rows)
        for b in range(begin // block_rows, end // block_rows):
            where = place(table, n_pages, page_rows, seq, b * block_rows)
            if where is None:
                continue
            for layer in range(layers):
                for head in range(heads):
                    keys = rows_of(pool, "k", layer, head, [(where[0], where[1] + i) for i in range(block_rows)])
                    at = (layer, where[0], head, where[1] // block_rows)
                    out[at][0], out[at][1], scales[at] = block_bounds(keys)
    return out, scales


def whole_query(q):
    """One query row float64 [128] -> whole numbers and their exponent."""
    if not np.isfinite(q).all():
        return np.zeros(128), -50
    f = unit(np.abs(q).max())
    return np.clip(np.rint(q / 2.0 ** f), -127, 127), f


def select(table, n_pages, page_rows, upper_lower, scales, block_rows, n_select, n_first, n_last, lengths, cu_new, max_new, q):
    """q float64 [layers][total_new][n_q_heads][128].  Returns a dict (layer, token, head) -> ascending blocks; tokens past max_new are not in it."""
    layers, heads = scales.shape[0], scales.shape[2]
    group = q.shape[2] // heads
    result = {}
    for layer in range(layers):
        for seq in range(len(lengths)):
            for t in range(min(int(cu_new[seq + 1] - cu_new[seq]), max_new)):
                r = int(cu_new[seq]) + t
                rows = max(0, min(int(lengths[seq]) + t + 1, table.shape[1] * page_rows))
                n = -(-rows // block_rows)
                places = [place(table, n_pages, page_rows, seq, b * block_rows) for b in range(n)]
                for head in range(heads):
                    whole = [whole_query(q[layer, r, h]) for h in range(head * group, (head + 1) * group)]
                    order = []
                    for b, where in enumerate(places):
                        if where is None:
                            continue
                        at = (layer, where[0], head, where[1] // block_rows)
                        if b < n_first or b >= n - n_last:
                            rank = (0, 0)
                        elif scales[at] == 255:
                            rank = (1, 0)
                        else:
                            ul = upper_lower[at].astype(np.float64)
                            e = int(scales[at]) - 127
                            rank = (2, -max(2.0 ** (f + e) * np.maximum(u * ul[0], u * ul[1]).sum() for u, f in whole))
                        order.append((rank, b))
                    result[layer, r, head] = sorted(b for _, b in sorted(order)[:n_select])
    return result


def sparse_attention(pool, table, lengths, cu_new, max_new, q, idx, count, block_rows, scale, softcap=0.0):
    """As paged_oracle.attention, over the rows of idx [layers][total_new][heads][n_select] (count [layers][total_new][heads])."""
    layers, n_pages, heads, page_rows = pool["k"].shape[:4]
    group, n_select = q.shape[2] // heads, idx.shape[3]
    out, weighted, size = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:3])
    for layer in range(layers):
        for seq in range(len(lengths)):
            for t in range(min(int(cu_new[seq + 1] - cu_new[seq]), max_new)):
                r = int(cu_new[seq]) + t
                for head in range(heads):
                    rows = []
                    for b in idx[layer, r, head, :max(0, min(int(count[layer, r, head]), n_select))].tolist():
                        rows += [i for i in range(b * block_rows, (b + 1) * block_rows) if 0 <= i <= int(lengths[seq]) + t] if 0 <= b < 1 << 26 else []
                    where = [place(table, n_pages, page_rows, seq, i) for i in rows]
                    where = [w for w in where if w is not None]
                    if not where:
                        continue
                    k, v = (rows_of(pool, name, layer, head, where) for name in ("k", "v"))
                    for h in range(head * group, (head + 1) * group):
                        with np.errstate(invalid="ignore"):
                            x = k @ q[layer, r, h] * scale
                            if softcap:
                                x = softcap * np.tanh(x / softcap)
                            w = np.exp(x - x.max())
                            w = w / w.sum()
                            out[layer, r, h] = w @ v
                            weighted[layer, r, h] = w @ np.abs(v)
                        size[layer, r, h] = (np.where(np.isfinite(k), np.abs(k), 0.0) @ np.abs(q[layer, r, h])).max() * scale
    return out, weighted, size
