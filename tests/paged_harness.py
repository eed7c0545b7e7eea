"""Shared helpers of the tests of the cache in pages: a pool with its table on the host and on the device."""
from __future__ import annotations

import numpy as np
import torch

import paper_2603_11564_amd as D
from oracle import dapq_oracle as O
from oracle import paged_oracle as PO

THETA = 500000.0
SCALE = 128 ** -0.5
JUNK = 0x7fc1                                       # a bf16 NaN: what nobody wrote


def normal_bits(rng, *shape):
    return O.f64_to_bf16_bits(rng.standard_normal(shape))


class Cache:
    """A pool of pages in random order.  rows: what each sequence has pages for.  Everything is NaN to begin with."""

    def __init__(self, rng, fmt, layers, heads, page_rows, rows, spare=2, extra_entries=1):
        self.fmt, self.layers, self.heads, self.page_rows, self.batch = fmt, layers, heads, page_rows, len(rows)
        need = [(n + page_rows - 1) // page_rows for n in rows]
        self.max_pages, self.n_pages = max(need) + extra_entries, sum(need) + spare
        order = rng.permutation(self.n_pages)
        self.table = np.full((self.batch, self.max_pages), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        shape = (layers, self.n_pages, heads, page_rows)
        if fmt == "fp4":
            self.pool = {"k": np.full(shape + (64,), 0x77, np.uint8), "v": np.full(shape + (64,), 0x77, np.uint8),
                         "k_scales": np.full(shape + (4,), 255, np.uint8), "v_scales": np.full(shape + (4,), 255, np.uint8)}
        elif fmt == "e4m3":
            self.pool = {"k": np.full(shape + (128,), 0x7f, np.uint8), "v": np.full(shape + (128,), 0x7f, np.uint8),
                         "k_scales": np.full(shape + (4,), 255, np.uint8), "v_scales": np.full(shape + (4,), 255, np.uint8)}
        else:
            self.pool = {"k": np.full(shape + (128,), JUNK, np.uint16), "v": np.full(shape + (128,), JUNK, np.uint16)}

    def fill(self, rng, lengths, gain=1.0):
        """Random rows 0 .. lengths[seq] - 1 on the host's pool."""
        for seq, n in enumerate(lengths):
            for i in range(n):
                where = PO.place(self.table, self.n_pages, self.page_rows, seq, i)
                if where is None:
                    continue
                page, slot = where
                for name, g in (("k", gain), ("v", 1.0)):
                    x = rng.standard_normal((self.layers, self.heads, 128)) * g
                    if self.fmt != "bf16":
                        quantise = PO.fp4_quantise if self.fmt == "fp4" else PO.e4m3_quantise
                        self.pool[name][:, page, :, slot], self.pool[name + "_scales"][:, page, :, slot] = quantise(x)
                    else:
                        self.pool[name][:, page, :, slot] = O.f64_to_bf16_bits(x)
        return self

    def to_device(self):
        """The pool on the GPU and its descriptor."""
        def dev(a):
            return torch.from_numpy(np.ascontiguousarray(a).view(np.int16 if a.dtype == np.uint16 else a.dtype)).cuda()
        self.dev = {n: dev(a) for n, a in self.pool.items()}
        self.dev_table = dev(self.table)
        self.pages = D.make_pages(n_layers=self.layers, batch=self.batch, n_kv_heads=self.heads, page_rows=self.page_rows,
                                  n_pages=self.n_pages, max_pages=self.max_pages, format=self.fmt, k=self.dev["k"], v=self.dev["v"],
                                  k_scales=self.dev.get("k_scales"), v_scales=self.dev.get("v_scales"), table=self.dev_table)
        return self

    def from_device(self):
        return {n: t.cpu().numpy().view(self.pool[n].dtype) for n, t in self.dev.items()}


def dev_bits(bits):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(torch.bfloat16)


def dev_int(values):
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


def starts(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(np.int32)


def strided(bits, pad_row=0, pad_head=0):
    """bits [layers][rows][heads][128] on the device with gaps of junk between heads and rows, and its strides."""
    layers, rows, heads, d = bits.shape
    head, row = d + pad_head, heads * (d + pad_head) + pad_row
    buf = np.full((layers, max(rows, 1), row), JUNK, dtype=np.uint16)
    for h in range(heads):
        buf[:, :rows, h * head:h * head + d] = bits[:, :, h]
    return dev_bits(buf), (max(rows, 1) * row, row, head)


def make_step(lengths, new, ragged=True, heads=1, max_new=None, **kw):
    return D.make_step(n_q_heads=kw.pop("n_q_heads", heads), total_new=int(sum(new)), max_new=max(new) if max_new is None else max_new,
                       cu_new=dev_int(starts(new)) if ragged else None, lengths=dev_int(lengths), scale=kw.pop("scale", SCALE), **kw)


def same_pool(got, want):
    for name in want:
        diff = np.argwhere(got[name] != want[name])
        assert diff.size == 0, f"{name}: {len(diff)} elements differ, first at {diff[0]}: {got[name][tuple(diff[0])]:#x}, {want[name][tuple(diff[0])]:#x}"


def attend(cache, lengths, new, q_bits, scale=SCALE, softcap=0.0, ragged=True, pads=(0, 0), max_new=None):
    """dapq_paged_attention on the device; returns float64 [layers][tokens][n_q_heads][128]."""
    q, strides = strided(q_bits, *pads)
    step = make_step(lengths, new, ragged, n_q_heads=q_bits.shape[2], q_strides=strides, scale=scale, softcap=softcap, max_new=max_new)
    out = dev_bits(np.full(q_bits.shape, JUNK, dtype=np.uint16))
    n = D.paged_attention_workspace_bytes(cache.pages, step)
    work = torch.full((n,), 0xA5, dtype=torch.uint8, device="cuda")
    D.dapq_paged_attention(cache.pages, step, q, out, work)
    torch.cuda.synchronize()
    return out.float().cpu().numpy().astype(np.float64)


def attention_bound(out, weighted, size, rows_of_q):
    """How far a result may be from the exact `out`, element by element.

    A logit is a sum of 128 products in fp32, at worst 128 roundings of 2^-24 of `size` (the sum of the products' magnitudes);
    its scaling, cap and exponential lose a few 2^-23 of a magnitude that is below size + 1.  A weight is off by that
    much on both sides of the division: 2 * 128 * 2^-24 + 2^-20 of (size + 1).  Weights meet the values with 16 bits (2^-15 on both sides), beyond 32 query
    rows of a KV head with 8 (2^-8 against values, and the same in the sum).  Accumulating up to 2^14 rows in fp32 in blocks loses at
    most 2^-13 in all.  Each is a part of the sum over |v|; then half a step of bf16: 2^-8."""
    part = (2.0 ** -16 + 2.0 ** -20) * (size[..., None] + 1) + 2.0 ** -15 + 2.0 ** -13 + (2.0 ** -7 if rows_of_q > 32 else 0.0)
    e = part * weighted
    return e + 2.0 ** -8 * (np.abs(out) + e) + 2.0 ** -133
