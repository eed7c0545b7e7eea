"""The operators of decoding over a cache in pages that is held in 8 bits, and of steps that read only a part of it, as cases that can be timed: rows
written in 8 bits and read back, attention over them, the bounds of the keys of a block, the choice of blocks for every query by those bounds, and attention
over the chosen blocks.

  listed()            the cases that are reported
  draw(rng)           one more case of the same ranges
  prepare(case, seed) what a program holds before the call: page pools, tables, lengths, new rows, bounds, chosen blocks, workspace
  run(state)          one pass: the library's entry points (own) or the same mathematics in elementary torch operations
  work(case)          bytes and floating-point operations the pass cannot do without
  exact(case, seed)   the outputs from the definition in 64 bits

A page pool holds rows of 128 channels: as bf16, or as codes (FP4: e2m1, two to a byte; e4m3: one to a byte) with one power-of-two scale per 32
channels.  Cases that write codes end with reading all rows back, as the values that the codes stand for.  The bounds of a block are whole numbers from
-127 to 127 in units of a power of two, and so are the queries that meet them, so that scores are exact sums of whole numbers and every choice can be
told to the last block.
"""
import math
import random

import torch

own = False

HEAD_DIM = 128
THETA = 500000.0
SCALE = 1.0 / math.sqrt(HEAD_DIM)
FP4_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
ROW_BYTES = {"bf16": 256, "fp4": 68, "e4m3": 132}


def _append(name, batch, kv_heads, held, new, page_rows, layers=1):
    """new rows for each sequence of the batch behind those it holds, in 8 bits; held and new: (low, high), lengths drawn between."""
    return dict(name=name, kind="append", format="e4m3", layers=layers, batch=batch, kv_heads=kv_heads, held_low=held[0],
                held_high=held[1], new_low=new[0], new_high=new[1], page_rows=page_rows)


def _gather(name, layers, batch, kv_heads, keys, budget, layout, page_rows):
    """the retained rows of prompts of keys = (low, high) tokens into pages of 8 bits.  layout: "heads" = K as
    [layer][head][token][d], "tokens" = [layer][token][head][d]."""
    return dict(name=name, kind="gather", format="e4m3", layers=layers, batch=batch, kv_heads=kv_heads, held_low=keys[0],
                held_high=keys[1], budget=budget, layout=layout, page_rows=page_rows)


def _attention(name, batch, q_heads, kv_heads, held, new, softcap, page_rows):
    """attention of the new tokens of each sequence over what it held before, in 8 bits, and, causally, over themselves."""
    return dict(name=name, kind="attention", format="e4m3", layers=1, batch=batch, q_heads=q_heads, kv_heads=kv_heads,
                held_low=held[0], held_high=held[1], new_low=new[0], new_high=new[1], softcap=softcap, page_rows=page_rows)


def _bounds(name, fmt, layers, batch, kv_heads, held, new, page_rows, block_rows):
    """the bounds of the blocks that the new rows complete."""
    return dict(name=name, kind="bounds", format=fmt, layers=layers, batch=batch, kv_heads=kv_heads, held_low=held[0], held_high=held[1],
                new_low=new[0], new_high=new[1], page_rows=page_rows, block_rows=block_rows)


def _select(name, batch, q_heads, kv_heads, held, new, page_rows, block_rows, n_select, first=1, last=1):
    """n_select blocks for every new token and KV head, the first and the last ones among them."""
    return dict(name=name, kind="select", format="bf16", layers=1, batch=batch, q_heads=q_heads, kv_heads=kv_heads, held_low=held[0], held_high=held[1],
                new_low=new[0], new_high=new[1], page_rows=page_rows, block_rows=block_rows, n_select=n_select, first=first, last=last)


def _sparse(name, fmt, batch, q_heads, kv_heads, held, new, softcap, page_rows, block_rows, n_select):
    """attention of the new tokens over n_select blocks for every token and KV head."""
    return dict(name=name, kind="sparse", format=fmt, layers=1, batch=batch, q_heads=q_heads, kv_heads=kv_heads, held_low=held[0], held_high=held[1],
                new_low=new[0], new_high=new[1], softcap=softcap, page_rows=page_rows, block_rows=block_rows, n_select=n_select)


def listed():
    return [
        # a token of each of 64 short sequences into 8 bits, small pages
        _append("append_batch_e4m3", 64, 8, (16, 96), (1, 1), 16),
        # a packed ragged batch of all layers evicted into 8 bits
        _gather("gather_ragged_e4m3", 32, 8, 8, (4096, 16384), 512, "tokens", 32),
        # decoding one token of each of 64 sequences over what turns and answers have left, one layer
        _attention("attention_batch_e4m3", 64, 32, 8, (1000, 4000), (1, 1), 0.0, 64),
        # the next turns of 8 conversations behind what the eviction kept: as much arithmetic as a prompt
        _attention("attention_turn_e4m3", 8, 32, 8, (983, 983), (200, 2500), 0.0, 64),
        # behind one decoded token of 64 sequences, of which a few complete a block: the smallest call, all latency
        _bounds("bounds_step", "bf16", 1, 64, 8, (256, 1100), (1, 1), 64, 16),
        # behind a prompt that is kept whole, 8 layers at a time
        _bounds("bounds_prompt", "bf16", 8, 1, 8, (0, 0), (32768, 32768), 64, 64),
        # choosing 64 of 2048 blocks for one token in one layer
        _select("select_layer", 1, 32, 8, (32767, 32767), (1, 1), 64, 16, 64),
        # the same for a token of each of 64 sequences, larger blocks, more of them kept at both ends
        _select("select_batch", 64, 32, 8, (4096, 32768), (1, 1), 64, 32, 64, 2, 4),
        # four drafted tokens of each of 32 sequences, 8 query heads per KV head
        _select("select_verify", 32, 64, 8, (8192, 32768), (4, 4), 128, 16, 128),
        # decoding one token of one sequence over 2048 of 128k rows: a model calls this once per layer
        _sparse("sparse_layer", "bf16", 1, 64, 8, (131071, 131071), (1, 1), 0.0, 64, 16, 128),
        # a token of each of 64 sequences over 2048 rows in 8 bits
        _sparse("sparse_batch_e4m3", "e4m3", 64, 32, 8, (2048, 16384), (1, 1), 0.0, 64, 32, 64),
        # four drafted tokens of each of 32 sequences over 1024 rows each, 8 query heads per KV head
        _sparse("sparse_verify", "bf16", 32, 64, 8, (4096, 16384), (4, 4), 0.0, 64, 64, 16),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kv_heads = rng.choice((8, 8, 8, 4, 2, 1, 5))
    page_rows = rng.choice((16, 16, 32, 64, 128, 256))
    kind = rng.choice(("append", "gather", "attention", "bounds", "select", "select", "sparse", "sparse"))

    def between(high):
        return (high, high) if rng.random() < 0.5 else (max(1, high // rng.randint(2, 8)), high)

    while True:
        fmt = rng.choice(("bf16", "fp4", "e4m3"))
        layers = rng.choice((1, 1, 2, 8, 32))
        batch = _log_int(rng, 1, 64)
        group = rng.choice((4, 4, 8, 2, 1, 7, 16))
        block_rows = rng.choice([n for n in (16, 32, 64, 128) if n <= page_rows])
        n_select = _log_int(rng, 4, 256)
        draw_new = rng.random()
        if kind == "append":
            held = between(_log_int(rng, 1, 2048))
            new = (1, 1) if draw_new < 0.4 else between(_log_int(rng, 2, 2500))
            if layers * batch * new[1] * kv_heads <= 150000 and layers * batch * (held[1] + new[1]) * kv_heads <= 400000:
                case = _append(None, batch, kv_heads, held, new, page_rows, layers)
                break
        elif kind == "gather":
            keys = between(_log_int(rng, 64, 32768))
            budget = min(_log_int(rng, 16, 4096), keys[1])
            if layers * batch * kv_heads * keys[1] <= 8.4e6 and layers * batch * kv_heads * budget <= 260000:
                case = _gather(None, layers, batch, kv_heads, keys, budget, rng.choice(("heads", "tokens")), page_rows)
                break
        elif kind == "attention":
            held = between(_log_int(rng, 16, 131071))
            new = (1, 1) if draw_new < 0.5 else between(_log_int(rng, 2, 16)) if draw_new < 0.75 else between(_log_int(rng, 16, 2500))
            rows = held[1] + new[1]
            if batch * kv_heads * rows <= 1.6e6 and batch * kv_heads * group * new[1] * rows <= 1.6e9:
                case = _attention(None, batch, kv_heads * group, kv_heads, held, new, rng.choice((0.0, 0.0, 30.0, 50.0)), page_rows)
                break
        elif kind == "bounds":
            held = between(_log_int(rng, 1, 2048))
            new = (1, 1) if draw_new < 0.3 else between(_log_int(rng, 2, 32768))
            if layers * batch * kv_heads * (held[1] + new[1]) <= 2.0e6:
                case = _bounds(None, fmt, layers, batch, kv_heads, held, new, page_rows, block_rows)
                if any((h + n) // block_rows > h // block_rows for h, n in zip(*_rows(case))):
                    break
        elif kind == "select":
            held = between(_log_int(rng, 512, 131071))
            new = (1, 1) if draw_new < 0.6 else between(_log_int(rng, 2, 200))
            rows = held[1] + new[1]
            first, last = rng.choice((0, 1, 1, 2)), rng.choice((1, 1, 2, 3))
            n_select = max(n_select, first + last + 2)
            # (there is something to choose from)
            if batch * kv_heads * rows <= 1.2e7 and batch * kv_heads * group * new[1] * rows / block_rows <= 3.2e7 and held[1] >= 4 * n_select * block_rows:
                case = _select(None, batch, kv_heads * group, kv_heads, held, new, page_rows, block_rows, n_select, first, last)
                break
        else:
            held = between(_log_int(rng, 16, 131071))
            new = (1, 1) if draw_new < 0.6 else between(_log_int(rng, 2, 200))
            rows = held[1] + new[1]
            if batch * kv_heads * rows <= 2.0e6 and batch * kv_heads * new[1] * n_select * block_rows <= 1.04e6:
                case = _sparse(None, fmt, batch, kv_heads * group, kv_heads, held, new, rng.choice((0.0, 0.0, 0.0, 50.0)), page_rows, block_rows, n_select)
                break
    del case["name"]
    return case


# --- sizes of a case: part of the case, not of the seed, so that a case is the same amount of work ------------------------
def _drawn(case, what):
    low, high = case[what + "_low"], case[what + "_high"]
    if low == high:
        return [high] * case["batch"]
    r = random.Random(low * 1000003 + high + (7 if what == "new" else 0))
    return [r.randint(low, high) for _ in range(case["batch"])]


def _rows(case):
    """(rows held before, new rows) of each sequence; rows in the pages are their sum (gather: the retained ones)."""
    held = _drawn(case, "held")
    if case["kind"] == "gather":
        return [min(n, case["budget"]) for n in held], [0] * case["batch"]
    return held, _drawn(case, "new")


def _blocks(rows, block_rows):
    return (rows + block_rows - 1) // block_rows


def work(case):
    held, new = _rows(case)
    heads = case["layers"] * case["kv_heads"]
    row, value = ROW_BYTES[case["format"]], 2 * HEAD_DIM
    rows_all = heads * (sum(held) + sum(new))
    read_back = 2 * rows_all * (row + value)
    if case["kind"] == "append":
        n = heads * sum(new)
        return {"bytes": 2 * n * (value + row) + 4 * sum(new) + read_back, "flops": 3 * HEAD_DIM * n}
    if case["kind"] == "gather":
        return {"bytes": rows_all * (2 * (value + row) + 4) + read_back, "flops": 0}
    if case["kind"] == "attention":
        pairs = sum(n * h + n * (n + 1) // 2 for h, n in zip(held, new)) * case["q_heads"]
        return {"bytes": 2 * rows_all * row + 2 * sum(new) * case["q_heads"] * value, "flops": 4 * HEAD_DIM * pairs}
    size = case["block_rows"]
    if case["kind"] == "bounds":
        blocks = heads * sum((h + n) // size - h // size for h, n in zip(held, new))
        return {"bytes": blocks * (size * row + 2 * HEAD_DIM + 1), "flops": 2 * HEAD_DIM * size * blocks}
    tokens = [(h, n, t) for h, n in zip(held, new) for t in range(n)]
    if case["kind"] == "select":
        ends = case["first"] + case["last"]
        scored = sum(max(0, _blocks(h + n, size) - ends) for h, n in zip(held, new) if n > 0)         # their bounds once, for all tokens
        pairs = sum(max(0, _blocks(h + t + 1, size) - ends) for h, _, t in tokens)
        chosen = sum(min(case["n_select"], _blocks(h + t + 1, size)) for h, _, t in tokens)
        return {"bytes": heads * (scored * (2 * HEAD_DIM + 1) + 4 * (chosen + len(tokens))) + len(tokens) * case["q_heads"] * value,
                "flops": 2 * HEAD_DIM * pairs * case["q_heads"]}
    # rows that several tokens of a sequence choose are read once: as many as are different where choices are independent
    distinct, pairs = 0.0, 0
    for h, n in zip(held, new):
        others = 1.0
        for t in range(n):
            blocks = _blocks(h + t + 1, size)
            kept = min(case["n_select"], blocks)
            others *= 1.0 - kept / blocks
            pairs += min(kept * size, h + t + 1)
        if n > 0:
            distinct += min(h + n, _blocks(h + n, size) * (1.0 - others) * size)
    return {"bytes": int(2 * heads * distinct * row) + 2 * len(tokens) * case["q_heads"] * value + heads * pairs // size * 4,
            "flops": 4 * HEAD_DIM * pairs * case["q_heads"]}


# --- plain forms of the formats -------------------------------------------------------------------------------------------
def _bf16_once(x):
    """float64 -> bf16, rounded once (nearest even): over float32 rounded to odd, which leaves no false ties."""
    f = x.to(torch.float32)
    back = f.to(torch.float64)
    u = f.view(torch.int32)
    u = torch.where(back.abs() > x.abs(), u - 1, u)
    u = torch.where((back != x) & torch.isfinite(x), u | 1, u)
    return u.view(torch.float32).to(torch.bfloat16)


def _power_of_two(e):
    """2^e in float32, -126 <= e <= 127, from its bits."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantise(x, fmt):
    """bf16 [..., 128] -> codes uint8 [..., 64 or 128] and scale bytes uint8 [..., 4]."""
    g = x.to(torch.float32).unflatten(-1, (4, 32))
    largest = g.abs().amax(-1)
    bad = ~torch.isfinite(g).all(-1)
    # the least e with largest <= limit * 2^e, up to which the largest level is a nearest one: 7 of levels up to 6, 464 of levels up to 448
    limit, low, high, top = (0.875, -125, 125, 3) if fmt == "fp4" else (0.90625, -117, 119, 9)
    m, e = torch.frexp(torch.where(bad, 1.0, largest))           # largest = m * 2^e, 1/2 <= m < 1; limit * 2^top is 7 or 464
    e = torch.where(m > limit, e - top + 1, e - top)
    e = torch.where(largest == 0, low, e).clamp(low, high)
    # (in two steps: neither power is past what float32 holds)
    y = torch.where(bad.unsqueeze(-1), 0.0, g.abs()) * _power_of_two(-(e // 2)).unsqueeze(-1) * _power_of_two(e // 2 - e).unsqueeze(-1)
    scales = torch.where(bad, 255, e + 127).to(torch.uint8)
    if fmt == "fp4":
        step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
        y = torch.clamp(torch.round(y / step) * step, max=6.0)
        code = torch.bucketize(y, torch.tensor(FP4_LEVELS, device=x.device)).to(torch.uint8)
        code = code + torch.where((g < 0) & ~bad.unsqueeze(-1), 8, 0).to(torch.uint8)
        code = code.flatten(-2)
        return code[..., 0::2] | (code[..., 1::2] << 4), scales
    _, x2 = torch.frexp(y)
    step = _power_of_two(x2.clamp(min=-5) - 4)                   # four bits of a value from 2^-6 on, 2^-9 below
    y = torch.clamp(torch.round(y / step) * step, max=448.0)
    return torch.where(g < 0, -y, y).flatten(-2).to(torch.float8_e4m3fn).view(torch.uint8), scales


def _values(codes, scales, fmt):
    """float32 values [..., 128] of codes and scale bytes."""
    two = torch.where(scales == 255, float("nan"), _power_of_two(scales.to(torch.int32) - 127)).unsqueeze(-1)
    if fmt == "fp4":
        table = torch.tensor(FP4_LEVELS + tuple(-v for v in FP4_LEVELS), device=codes.device)
        x = table[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).to(torch.int32)]
    else:
        x = codes.view(torch.float8_e4m3fn).to(torch.float32)
    return (x.unflatten(-1, (4, 32)) * two).flatten(-2)


def _whole_bounds(x):
    """float32 keys [..., rows, 128] -> bounds int8 [..., 2, 128] (the upper ones first) and scale bytes uint8 [...]."""
    most, least = x.amax(-2), x.amin(-2)
    bad = ~torch.isfinite(x).flatten(-2).all(-1)
    most, least = (torch.where(bad.unsqueeze(-1), 0.0, b) for b in (most, least))
    e = _whole_exponent(torch.maximum(most, -least).amax(-1))
    unit = _power_of_two(-e).unsqueeze(-1)
    hi, lo = torch.ceil(most * unit).clamp(-127, 127), torch.floor(least * unit).clamp(-127, 127)
    return torch.stack((hi, lo), -2).to(torch.int8), torch.where(bad, 255, e + 127).to(torch.uint8)


def _whole_exponent(largest):
    """The least e in [-50, 50] with largest <= 127 * 2^e."""
    m, e = torch.frexp(largest)
    return torch.where(largest == 0, -50, torch.where(m > 127.0 / 128.0, e - 6, e - 7)).clamp(-50, 50)


def _bf16(gen, *shape):
    """N(0, 1) in bf16."""
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)


def _model_keys(gen, *shape):
    """Keys as a model leaves them: some channels are several times as large as the others in every row, and rows of a page are alike."""
    gain = torch.ones(HEAD_DIM, device="cuda")
    gain[::17] = 4.0
    alike = _bf16(gen, *shape[:-2], 1, HEAD_DIM)
    return (_bf16(gen, *shape) + alike) * gain.to(torch.bfloat16)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    held, new = _rows(case)
    kind, fmt = case["kind"], case["format"]
    layers, batch, heads, page_rows = case["layers"], case["batch"], case["kv_heads"], case["page_rows"]
    rows = [h + n for h, n in zip(held, new)]
    pages_of = [(n + page_rows - 1) // page_rows for n in rows]
    max_pages = max(pages_of)
    n_pages = sum(pages_of) + max(1, sum(pages_of) // 8)
    state = dict(case=case, held=held, new=new, rows=rows, n_pages=n_pages, max_pages=max_pages)
    # the pages of a sequence stand anywhere in the pool; entries behind its last page are -1
    order = torch.randperm(n_pages, generator=gen, device="cuda", dtype=torch.int32)
    table = torch.full((batch, max_pages), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(pages_of):
        table[b, :n] = order[at:at + n]
        at += n
    state["table"] = table
    state["lengths"] = _int32(held)                    # before the new rows
    pool = (layers, n_pages, heads, page_rows)
    step = max(1, (1 << 26) // (heads * page_rows * HEAD_DIM))
    if kind == "select":
        # of the keys only their bounds: selection reads nothing else.  (A pool of one row stands for the keys themselves.)
        size = case["block_rows"]
        state["bounds"] = torch.empty(pool[:3] + (page_rows // size, 2, HEAD_DIM), dtype=torch.int8, device="cuda")
        state["bound_scales"] = torch.empty(pool[:3] + (page_rows // size,), dtype=torch.uint8, device="cuda")
        for p in range(0, n_pages, step):
            x = _model_keys(gen, min(step, n_pages - p), heads, page_rows // size, size, HEAD_DIM)
            state["bounds"][0, p:p + step], state["bound_scales"][0, p:p + step] = _whole_bounds(x.to(torch.float32))
        state["k"] = state["v"] = torch.zeros(HEAD_DIM, dtype=torch.bfloat16, device="cuda")
        state["k_scales"] = state["v_scales"] = None
    else:
        for name, keys in (("k", True), ("v", False)):
            make = _model_keys if keys else _bf16
            if fmt == "bf16":
                state[name], state[name + "_scales"] = make(gen, *pool, HEAD_DIM), None
                continue
            codes = torch.zeros(pool + (HEAD_DIM // (2 if fmt == "fp4" else 1),), dtype=torch.uint8, device="cuda")
            scales = torch.full(pool + (4,), 127, dtype=torch.uint8, device="cuda")
            if kind != "gather":
                for layer in range(layers):
                    for p in range(0, n_pages, step):
                        x = make(gen, min(step, n_pages - p), heads, page_rows, HEAD_DIM)
                        codes[layer, p:p + step], scales[layer, p:p + step] = _quantise(x, fmt)
            state[name], state[name + "_scales"] = codes, scales
    if max(new):
        total = sum(new)
        ragged = case["new_low"] != case["new_high"]
        state["cu_new"] = _int32([sum(new[:b]) for b in range(batch + 1)]) if ragged else None
        state["total_new"], state["max_new"] = total, max(new)
    if kind == "append":
        state["k_new"] = _model_keys(gen, layers, total, heads, HEAD_DIM)
        state["v_new"] = _bf16(gen, layers, total, heads, HEAD_DIM)
        # the positions go on behind the prompt that was evicted, far behind the rows that were kept of it
        first = [33 * h for h in held]
        state["positions"] = _int32([f + t for f, n in zip(first, new) for t in range(n)])
    if kind in ("attention", "select", "sparse"):
        state["q"] = _bf16(gen, 1, total, case["q_heads"], HEAD_DIM) * 1.5
    if kind in ("attention", "sparse"):
        state["out"] = torch.empty_like(state["q"])
    if kind == "gather":
        keys = _drawn(case, "held")
        tokens = sum(keys)
        cu = [sum(keys[:b]) for b in range(batch + 1)]
        shape = (layers, heads, tokens, HEAD_DIM) if case["layout"] == "heads" else (layers, tokens, heads, HEAD_DIM)
        state["k_prompt"], state["v_prompt"] = _model_keys(gen, *shape), _bf16(gen, *shape)
        state["cu_seqlens"], state["cu"] = _int32(cu), cu
        idx = torch.zeros((layers, batch, heads, case["budget"]), dtype=torch.int32, device="cuda")
        for b, n in enumerate(held):
            noise = torch.rand((layers, heads, keys[b]), generator=gen, device="cuda")
            idx[:, b, :, :n] = noise.topk(n, -1).indices.sort(-1).values.to(torch.int32)
        state["idx"] = idx
        state["count"] = state["lengths"][None, :, None].expand(layers, batch, heads).contiguous()
    if kind in ("append", "gather"):
        shape = (layers, batch, heads, max(rows), HEAD_DIM)
        state["k_out"] = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
        state["v_out"] = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
        state["filled"] = _int32(rows)
    if kind == "bounds":
        size = case["block_rows"]
        state["bounds"] = torch.zeros(pool[:3] + (page_rows // size, 2, HEAD_DIM), dtype=torch.int8, device="cuda")
        state["bound_scales"] = torch.zeros(pool[:3] + (page_rows // size,), dtype=torch.uint8, device="cuda")
        state["filled"] = _int32(rows)
    if kind in ("select", "sparse"):
        state["idx"] = torch.full((1, total, heads, case["n_select"]), -1, dtype=torch.int32, device="cuda")
        state["count"] = torch.zeros((1, total, heads), dtype=torch.int32, device="cuda")
    if kind == "sparse":
        # blocks chosen anywhere, the first and the last one among them
        r = 0
        for b in range(batch):
            for t in range(new[b]):
                n = _blocks(held[b] + t + 1, case["block_rows"])
                noise = torch.rand((heads, n), generator=gen, device="cuda")
                noise[:, 0] = noise[:, -1] = 2.0
                kept = min(case["n_select"], n)
                state["idx"][0, r, :, :kept] = noise.topk(kept, -1).indices.sort(-1).values.to(torch.int32)
                state["count"][0, r] = kept
                r += 1
    if own:
        import paper_2603_11564_amd as D
        state["pages"] = D.make_pages(n_layers=layers, batch=batch, n_kv_heads=heads, page_rows=page_rows, n_pages=n_pages,
                                      max_pages=max_pages, format=fmt, k=state["k"], v=state["v"],
                                      k_scales=state["k_scales"], v_scales=state["v_scales"], table=table)
        if max(new):
            q_heads = case.get("q_heads", heads)
            kv = (total * heads * HEAD_DIM, heads * HEAD_DIM, HEAD_DIM)
            state["step"] = D.make_step(n_q_heads=q_heads, total_new=total, max_new=max(new), cu_new=state["cu_new"],
                                        lengths=state["lengths"], k_strides=kv, v_strides=kv,
                                        q_strides=(total * q_heads * HEAD_DIM, q_heads * HEAD_DIM, HEAD_DIM),
                                        scale=SCALE, softcap=case.get("softcap", 0.0))
        if "block_rows" in case:
            state["blocks"] = D.make_blocks(block_rows=case["block_rows"], n_select=case.get("n_select", 1), n_first=case.get("first", 0),
                                            n_last=case.get("last", 1), bounds=state.get("bounds"), scales=state.get("bound_scales"))
        if kind in ("attention", "select", "sparse"):
            if kind == "attention":
                n = D.paged_attention_workspace_bytes(state["pages"], state["step"])
            elif kind == "select":
                n = D.paged_select_workspace_bytes(state["pages"], state["blocks"], state["step"])
            else:
                n = D.paged_sparse_attention_workspace_bytes(state["pages"], state["blocks"], state["step"])
            state["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        if kind == "gather":
            tokens = state["cu"][-1]
            strides = (tokens * heads * HEAD_DIM, 0, tokens * HEAD_DIM, HEAD_DIM) if case["layout"] == "heads" else \
                (tokens * heads * HEAD_DIM, 0, HEAD_DIM, heads * HEAD_DIM)
            state["shape"] = D.make_shape(n_layers=layers, batch=batch, n_q_heads=heads, n_kv_heads=heads, n_pseudo=1,
                                          total_tokens=tokens, cu_seqlens=state["cu_seqlens"], k_strides=strides,
                                          v_strides=strides, scale=SCALE)
    return state


# --- one pass through the library ------------------------------------------------------------------------------------------
def _run_own(s):
    import paper_2603_11564_amd as D
    kind = s["case"]["kind"]
    if kind == "attention":
        D.dapq_paged_attention(s["pages"], s["step"], s["q"], s["out"], s["workspace"])
        return s["out"]
    if kind == "sparse":
        D.dapq_paged_sparse_attention(s["pages"], s["blocks"], s["step"], s["q"], s["idx"], s["count"], s["out"], s["workspace"])
        return s["out"]
    if kind == "select":
        D.dapq_paged_select(s["pages"], s["blocks"], s["step"], s["q"], s["idx"], s["count"], s["workspace"])
        return s["idx"], s["count"]
    if kind == "bounds":
        D.dapq_paged_bounds(s["pages"], s["blocks"], s["lengths"], s["filled"], max(s["new"]))
        return s["bounds"], s["bound_scales"]
    if kind == "append":
        D.dapq_paged_append(s["pages"], s["step"], s["k_new"], s["v_new"], s["positions"], THETA, 0)
    else:
        D.dapq_paged_gather(s["shape"], s["pages"], s["k_prompt"], s["v_prompt"], s["idx"], s["count"], s["case"]["budget"])
    D.dapq_paged_read(s["pages"], s["filled"], max(s["rows"]), s["k_out"], s["v_out"])
    return s["k_out"], s["v_out"]


# --- the same in elementary operations -------------------------------------------------------------------------------------
def _places(s, first, count):
    """Rows first[b] .. first[b] + count[b] - 1 of every sequence, one after the other: their pages and slots."""
    page_rows = s["case"]["page_rows"]
    total = sum(count)
    seq = torch.repeat_interleave(torch.arange(len(count), device="cuda"), torch.tensor(count, device="cuda"), output_size=total)
    start = torch.tensor([f - sum(count[:b]) for b, f in enumerate(first)], device="cuda")
    row = torch.arange(total, device="cuda") + start[seq]
    return seq, row, s["table"][seq, row // page_rows].long(), row % page_rows


def _held(s, name, *at):
    """float32 rows of the pool at an index of its axes [layer][page][head][slot]."""
    x = s[name][at]
    if s[name + "_scales"] is not None:
        return _values(x, s[name + "_scales"][at], s["case"]["format"])
    return x.to(torch.float32)


def _put(s, name, page, slot, x):
    """x: bf16 [layer][row][head][d] into the pool."""
    codes, scales = _quantise(x, s["case"]["format"])
    s[name][:, page, :, slot] = codes.transpose(0, 1)
    s[name + "_scales"][:, page, :, slot] = scales.transpose(0, 1)


def _read_plain(s):
    seq, row, page, slot = _places(s, [0] * len(s["rows"]), s["rows"])
    for name in ("k", "v"):
        s[name + "_out"][:, seq, :, row] = _held(s, name, slice(None), page, slice(None), slot).to(torch.bfloat16)
    return s["k_out"], s["v_out"]


def _rotated(x, positions):
    """x: bf16 [layer][row][head][d]; channel c is paired with c + 64.  Angles and products in 64 bits, rounded once."""
    half = HEAD_DIM // 2
    omega = THETA ** (-2.0 * torch.arange(half, device="cuda", dtype=torch.float64) / HEAD_DIM)
    angle = positions.to(torch.float64)[:, None, None] * omega
    a, b = x[..., :half].to(torch.float64), x[..., half:].to(torch.float64)
    return _bf16_once(torch.cat((a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()), -1))


def _padded(s):
    """The new tokens as [sequence][number]: their rows in q, which of them there are, and the rows that each sees."""
    new = torch.tensor(s["new"], device="cuda")
    token = torch.arange(s["max_new"], device="cuda")
    at = (new.cumsum(0) - new)[:, None] + token
    return at.clamp(max=s["total_new"] - 1), token < new[:, None], s["lengths"][:, None].long() + token + 1


def _capped_softmax(x, softcap, hidden):
    x = x * SCALE
    if softcap:
        x = torch.tanh(x / softcap) * softcap
    x = x.masked_fill(hidden, -math.inf)
    x = torch.exp(x - x.amax(-1, keepdim=True))
    return x / x.sum(-1, keepdim=True)


def _attention_plain(s):
    case = s["case"]
    batch, heads, page_rows = case["batch"], case["kv_heads"], case["page_rows"]
    group = case["q_heads"] // heads
    row = torch.arange(max(s["rows"]), device="cuda")
    page = s["table"][:, row // page_rows].long().clamp(min=0)      # [seq][row]
    k, v = (_held(s, name, 0, page, slice(None), (row % page_rows).expand(batch, -1)).transpose(1, 2) for name in ("k", "v"))
    at, real, visible = _padded(s)
    q = s["q"][0][at].to(torch.float32).unflatten(2, (heads, group)).permute(0, 2, 3, 1, 4).flatten(2, 3)  # [seq][head][group * token][d]
    hidden = (row >= visible[..., None])[:, None, None].expand(-1, heads, group, -1, -1).flatten(2, 3)
    x = torch.matmul(_capped_softmax(torch.matmul(q, k.transpose(-1, -2)), case["softcap"], hidden), v)
    x = x.unflatten(2, (group, s["max_new"])).permute(0, 3, 1, 2, 4).flatten(2, 3)  # [seq][token][q head][d]
    s["out"][0] = x[real].to(torch.bfloat16)
    return s["out"]


def _bounds_plain(s):
    case = s["case"]
    size, page_rows = case["block_rows"], case["page_rows"]
    first = [h // size for h in s["held"]]
    seq, block, _, _ = _places(s, first, [n // size - f for n, f in zip(s["rows"], first)])
    page, part = s["table"][seq, block * size // page_rows].long(), block % (page_rows // size)
    slot = part[:, None] * size + torch.arange(size, device="cuda")
    x = _held(s, "k", slice(None), page[:, None], slice(None), slot)  # [block][row][layer][head][d]
    whole, scales = _whole_bounds(x.permute(0, 2, 3, 1, 4))
    s["bounds"][:, page, :, part] = whole
    s["bound_scales"][:, page, :, part] = scales
    return s["bounds"], s["bound_scales"]


def _select_plain(s):
    case = s["case"]
    heads, size, page_rows = case["kv_heads"], case["block_rows"], case["page_rows"]
    group = case["q_heads"] // heads
    block = torch.arange(_blocks(max(s["rows"]), size), device="cuda")
    page = s["table"][:, block * size // page_rows].long()          # [seq][block]
    there, page, part = page >= 0, page.clamp(min=0), (block % (page_rows // size)).expand(len(s["rows"]), -1)
    whole = s["bounds"][0, page, :, part].to(torch.float32).transpose(1, 2)   # [seq][head][block][2][d]
    scale = s["bound_scales"][0, page, :, part].transpose(1, 2)               # [seq][head][block]
    at, real, visible = _padded(s)
    q = s["q"][0][at].to(torch.float32)                             # [seq][token][q head][d]
    bad = ~torch.isfinite(q).all(-1, keepdim=True)
    q = torch.where(bad, 0.0, q)
    f = _whole_exponent(q.abs().amax(-1))
    q = torch.round(q * _power_of_two(-f).unsqueeze(-1)).clamp(-127, 127)
    q = q.unflatten(2, (heads, group)).permute(0, 2, 3, 1, 4).flatten(2, 3)   # [seq][head][group * token][d]
    # sums of whole numbers below 2^24: exact in 32 bits
    x = torch.matmul(q.clamp(min=0), whole[..., 0, :].transpose(-1, -2)) + torch.matmul(q.clamp(max=0), whole[..., 1, :].transpose(-1, -2))
    x = x.unflatten(2, (group, -1)) * _power_of_two(f).unflatten(2, (heads, group)).permute(0, 2, 3, 1).unsqueeze(-1)
    x = x.amax(2) * _power_of_two(torch.where(scale == 255, 0, scale.to(torch.int32) - 127)).unsqueeze(2)  # [seq][head][token][block]
    blocks = ((visible + size - 1) // size)[:, None, :, None]
    ends = (block < case["first"]) | (block >= blocks - case["last"])
    x = torch.where((scale == 255).unsqueeze(2), torch.finfo(torch.float32).max, x)
    x = torch.where(ends, math.inf, x).masked_fill((block >= blocks) | ~there[:, None, None], -math.inf)
    best = torch.sort(x, dim=-1, descending=True, stable=True)      # (of equal ones the lowest block first)
    n = min(case["n_select"], x.shape[-1])
    none = x.shape[-1]
    chosen = torch.where(best.values[..., :n] > -math.inf, best.indices[..., :n], none).sort(-1).values
    chosen = torch.where(chosen == none, -1, chosen).to(torch.int32).transpose(1, 2)    # [seq][token][head][n]
    s["idx"][0, :, :, :n] = chosen[real]
    s["count"][0] = (chosen >= 0).sum(-1).to(torch.int32)[real]
    return s["idx"], s["count"]


def _sparse_plain(s):
    case = s["case"]
    heads, size, page_rows = case["kv_heads"], case["block_rows"], case["page_rows"]
    group, total = case["q_heads"] // heads, s["total_new"]
    seq = torch.repeat_interleave(torch.arange(case["batch"], device="cuda"), torch.tensor(s["new"], device="cuda"), output_size=total)
    _, real, visible = _padded(s)
    visible = visible[real]                                         # [token]
    slot = torch.arange(case["n_select"], device="cuda")
    real = slot < s["count"][0][..., None]                          # [token][head][slot]
    row = (torch.where(real, s["idx"][0], 0).long()[..., None] * size + torch.arange(size, device="cuda")).flatten(2)
    hidden = ~real.repeat_interleave(size, -1) | (row >= visible[:, None, None])
    page = s["table"][seq[:, None, None], (row // page_rows).clamp(max=s["max_pages"] - 1)].long().clamp(min=0)
    head = torch.arange(heads, device="cuda")[:, None]
    k, v = (_held(s, name, 0, page, head, row % page_rows) for name in ("k", "v"))   # [token][head][row][d]
    q = s["q"][0].to(torch.float32).unflatten(1, (heads, group))
    x = torch.matmul(_capped_softmax(torch.matmul(q, k.transpose(-1, -2)), case["softcap"], hidden.unsqueeze(2)), v)
    s["out"][0] = x.flatten(1, 2).to(torch.bfloat16)
    return s["out"]


def run(state):
    if own:
        return _run_own(state)
    s, kind = state, state["case"]["kind"]
    if kind in ("attention", "bounds", "select", "sparse"):
        return {"attention": _attention_plain, "bounds": _bounds_plain, "select": _select_plain, "sparse": _sparse_plain}[kind](s)
    if kind == "append":
        _, _, page, slot = _places(s, s["held"], s["new"])
        _put(s, "k", page, slot, _rotated(s["k_new"], s["positions"]))
        _put(s, "v", page, slot, s["v_new"])
    else:
        seq, row, page, slot = _places(s, [0] * len(s["rows"]), s["rows"])
        token = (s["idx"][:, seq, :, row] + torch.tensor(s["cu"], device="cuda")[seq][:, None, None]).long()  # [row][layer][head]
        layer = torch.arange(s["case"]["layers"], device="cuda")[:, None]
        head = torch.arange(s["case"]["kv_heads"], device="cuda")
        for name in ("k", "v"):
            x = s[name + "_prompt"]
            x = x[layer, head, token] if s["case"]["layout"] == "heads" else x[layer, token, head]
            _put(s, name, page, slot, x.transpose(0, 1))
    return _read_plain(s)


# --- from the definition, in 64 bits ---------------------------------------------------------------------------------------
def _levels(fmt):
    """The magnitudes that codes 0, 1, 2, ... stand for."""
    if fmt == "fp4":
        return torch.tensor(FP4_LEVELS, dtype=torch.float64, device="cuda")
    return torch.tensor([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127] + [math.nan],
                        dtype=torch.float64, device="cuda")


def _nearest_e4m3(x):
    """float64 [..., 32] groups -> what e4m3 keeps of them: the level whose distance is least, the even code of two."""
    largest = x.abs().amax(-1, keepdim=True)
    scale = torch.full_like(largest, 2.0 ** -117)
    for e in range(-116, 120):
        scale = torch.where(largest > 464.0 * 2.0 ** (e - 1), 2.0 ** e, scale)
    y = x.abs() / scale
    levels = _levels("e4m3")[:127]
    above = torch.searchsorted(levels, y.contiguous()).clamp(1, 126)
    low, high = levels[above - 1], levels[above]
    up = (y - low > high - y) | ((y - low == high - y) & (above % 2 == 0))
    return torch.where(up, high, low) * scale * torch.sign(x)


def _held_values(s, name, layer, b, n):
    """float64 [head][n][d]: the first n rows of sequence b in one layer."""
    page_rows, fmt = s["case"]["page_rows"], s["case"]["format"]
    pages = s["table"][b, :(n + page_rows - 1) // page_rows].long()
    def rows(x):
        return x[layer].index_select(0, pages).permute(1, 0, 2, 3).flatten(1, 2)[:, :n]
    x = rows(s[name])
    if fmt == "bf16":
        return x.double()
    codes, half = x.long(), 128
    if fmt == "fp4":
        codes, half = torch.empty(x.shape[:2] + (HEAD_DIM,), dtype=torch.long, device="cuda"), 8
        codes[..., 0::2], codes[..., 1::2] = (x & 15).long(), (x >> 4).long()
    powers = torch.tensor([2.0 ** (e - 127) for e in range(255)] + [math.nan], dtype=torch.float64, device="cuda")
    return _levels(fmt)[codes % half] * (1 - 2 * (codes // half)) * powers[rows(s[name + "_scales"]).long()].repeat_interleave(32, -1)


def _new_values(s, name, layer, b):
    """float64 [head][n][d]: the new rows of sequence b as the cache holds them."""
    at = sum(s["new"][:b])
    x = s[name + "_new"][layer, at:at + s["new"][b]].double()
    if name == "k":
        turn = torch.polar(torch.ones(64, dtype=torch.float64, device="cuda"),
                           s["positions"][at:at + s["new"][b], None, None].double()
                           * torch.exp(torch.arange(64, dtype=torch.float64, device="cuda") * (-math.log(THETA) / 64)))
        z = torch.complex(x[..., :64], x[..., 64:]) * turn
        x = torch.cat((z.real, z.imag), -1)
    apart = x.transpose(0, 1) * (2.0 ** 45 + 1.0)                    # the nearest number of 53 - 45 = 8 bits, as bf16 has
    return _nearest_e4m3((apart - (apart - x.transpose(0, 1))).unflatten(-1, (4, 32))).flatten(-2)


def _exact_softmax(x, softcap, hidden=None):
    x = x * SCALE
    x = softcap * torch.tanh(x / softcap) if softcap else x
    return torch.softmax(x if hidden is None else x.masked_fill(hidden, -math.inf), -1)


def _exact_whole_exponent(largest):
    e = torch.full_like(largest, -50.0)
    for candidate in range(-49, 51):
        e = torch.where(largest > 127.0 * 2.0 ** (candidate - 1), float(candidate), e)
    return e


def _exact_bounds(s):
    case = s["case"]
    size, page_rows = case["block_rows"], case["page_rows"]
    bounds, scales = s["bounds"].clone(), s["bound_scales"].clone()
    for layer in range(case["layers"]):
        for b in range(case["batch"]):
            first, last = s["held"][b] // size, s["rows"][b] // size
            if first == last:
                continue
            x = _held_values(s, "k", layer, b, last * size)[:, first * size:].unflatten(1, (last - first, size))
            most, least = x.max(2).values, x.min(2).values          # [head][block][d]
            e = _exact_whole_exponent(torch.maximum(most.abs(), least.abs()).max(-1).values)
            unit = torch.pow(2.0, e).unsqueeze(-1)
            block = torch.arange(first, last, device="cuda")
            page, part = s["table"][b].long()[block * size // page_rows], block % (page_rows // size)
            bounds[layer, page, :, part] = torch.stack((torch.ceil(most / unit), torch.floor(least / unit)), 2).transpose(0, 1).to(torch.int8)
            scales[layer, page, :, part] = (e + 127).T.to(torch.uint8)
    return bounds, scales


def _exact_select(s):
    case = s["case"]
    heads, size, page_rows = case["kv_heads"], case["block_rows"], case["page_rows"]
    idx, count = torch.full_like(s["idx"], -1), torch.zeros_like(s["count"])
    for b in range(case["batch"]):
        at = sum(s["new"][:b])
        block = torch.arange(_blocks(s["rows"][b], size), device="cuda")
        page, part = s["table"][b].long()[block * size // page_rows], block % (page_rows // size)
        whole, scale = s["bounds"][0, page, :, part].double(), s["bound_scales"][0, page, :, part].double()   # [block][head]...
        upper, lower = (whole[:, :, i] * torch.pow(2.0, scale - 127).unsqueeze(-1) for i in (0, 1))
        for t in range(s["new"][b]):
            q = s["q"][0, at + t].double()                          # [q head][d]
            unit = torch.pow(2.0, _exact_whole_exponent(q.abs().max(-1).values)).unsqueeze(-1)
            q = (torch.round(q / unit) * unit).unflatten(0, (heads, -1))
            n = _blocks(s["held"][b] + t + 1, size)
            # products of 16 bits, and their sums, are exact in 64
            score = torch.stack([torch.stack([(torch.maximum(q[h, i] * upper[:n, h], q[h, i] * lower[:n, h])).sum(-1)
                                              for i in range(q.shape[1])]).max(0).values for h in range(heads)])
            score[:, :case["first"]] = math.inf
            score[:, max(0, n - case["last"]):] = math.inf
            kept = min(case["n_select"], n)
            order = torch.argsort(score, dim=-1, descending=True, stable=True)
            idx[0, at + t, :, :kept] = order[:, :kept].sort(-1).values.to(torch.int32)
            count[0, at + t] = kept
    return idx, count


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    layers, batch, heads, size = case["layers"], case["batch"], case["kv_heads"], case.get("block_rows")
    if kind == "bounds":
        return _exact_bounds(s)
    if kind == "select":
        return _exact_select(s)
    if kind in ("attention", "sparse"):
        group = case["q_heads"] // heads
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        for b in range(batch):
            n, held = s["new"][b], s["held"][b]
            at = sum(s["new"][:b])
            k, v = _held_values(s, "k", 0, b, held + n), _held_values(s, "v", 0, b, held + n)
            if kind == "attention":
                hidden = torch.arange(held + n, device="cuda") > held + torch.arange(n, device="cuda")[:, None]
                for h in range(case["q_heads"]):
                    w = _exact_softmax(s["q"][0, at:at + n, h].double() @ k[h // group].T, case["softcap"], hidden)
                    out[0, at:at + n, h] = w @ v[h // group]
                continue
            for t in range(n):
                kept = int(s["count"][0, at + t, 0])
                row = (s["idx"][0, at + t, :, :kept].long()[..., None] * size + torch.arange(size, device="cuda")).flatten(1)
                row = row[:, :int((row[0] <= held + t).sum())]      # (only the last block, which all heads have, ends behind the token)
                rows = row[..., None].expand(-1, -1, HEAD_DIM)
                q = s["q"][0, at + t].double().unflatten(0, (heads, group))
                w = _exact_softmax(torch.matmul(q, k.gather(1, rows).transpose(1, 2).contiguous()), case["softcap"])
                out[0, at + t] = torch.matmul(w, v.gather(1, rows)).flatten(0, 1)
        return out
    result = []
    for name in ("k", "v"):
        got = torch.zeros(s[name + "_out"].shape, dtype=torch.float64, device="cuda")
        for layer in range(layers):
            for b in range(batch):
                if kind == "gather":
                    n = s["held"][b]
                    rows = s["idx"][layer, b, :, :n].long() + s["cu"][b]
                    x = s[name + "_prompt"][layer]
                    x = x if case["layout"] == "heads" else x.transpose(0, 1)
                    x = torch.stack([x[h].index_select(0, rows[h]) for h in range(heads)]).double()
                    x, first = _nearest_e4m3(x.unflatten(-1, (4, 32))).flatten(-2), 0
                else:
                    x, first = _new_values(s, name, layer, b), s["held"][b]
                    got[layer, b, :, :first] = _held_values(s, name, layer, b, first)
                got[layer, b, :, first:first + x.shape[1]] = x
        result.append(got)
    return tuple(result)
