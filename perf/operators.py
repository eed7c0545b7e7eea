"""The operators of decoding over a paged cache, as cases that can be timed: writing the rows that an eviction kept into
pages, appending the rows of new tokens with their rotation, reading rows back, and attention over the pages.

  listed()            the cases that are reported
  draw(rng)           one more case of the same ranges
  prepare(case, seed) what a program holds before the call: page pools, tables, lengths, new rows, workspace
  run(state)          one pass: the library's entry points (own) or the same mathematics in elementary torch operations
  work(case)          bytes and floating-point operations the pass cannot do without
  exact(case, seed)   the outputs from the definition in 64 bits

A page pool holds rows of 128 channels: as bf16, or as FP4 (e2m1 codes, two to a byte, one power-of-two scale per 32
channels).  Cases that write FP4 end with reading all rows back, as the values that the codes stand for.
"""
import math
import random

import torch

own = False

HEAD_DIM = 128
THETA = 500000.0
SCALE = 1.0 / math.sqrt(HEAD_DIM)
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _append(name, fmt, layers, batch, kv_heads, held, new, page_rows):
    """new rows for each sequence of the batch behind those it holds; held and new: (low, high), lengths drawn between."""
    return dict(name=name, kind="append", format=fmt, layers=layers, batch=batch, kv_heads=kv_heads, held_low=held[0],
                held_high=held[1], new_low=new[0], new_high=new[1], page_rows=page_rows)


def _gather(name, fmt, layers, batch, kv_heads, keys, budget, layout, page_rows):
    """the retained rows of prompts of keys = (low, high) tokens into pages.  layout: "heads" = K as
    [layer][head][token][d], "tokens" = [layer][token][head][d]."""
    return dict(name=name, kind="gather", format=fmt, layers=layers, batch=batch, kv_heads=kv_heads, held_low=keys[0],
                held_high=keys[1], budget=budget, layout=layout, page_rows=page_rows)


def _read(name, fmt, layers, batch, kv_heads, held, page_rows):
    """all rows of a batch as bf16 in the layout of the compact cache."""
    return dict(name=name, kind="read", format=fmt, layers=layers, batch=batch, kv_heads=kv_heads, held_low=held[0],
                held_high=held[1], page_rows=page_rows)


def _attention(name, fmt, batch, q_heads, kv_heads, held, new, softcap, page_rows):
    """attention of the new tokens of each sequence over what it held before and, causally, over themselves (their rows
    are in the pages)."""
    return dict(name=name, kind="attention", format=fmt, layers=1, batch=batch, q_heads=q_heads, kv_heads=kv_heads,
                held_low=held[0], held_high=held[1], new_low=new[0], new_high=new[1], softcap=softcap, page_rows=page_rows)


def listed():
    return [
        # one token of one sequence in one layer: the smallest call, all latency
        _append("append_layer", "bf16", 1, 1, 8, (983, 983), (1, 1), 64),
        # a token of each of 64 short sequences into 4 bits, small pages
        _append("append_batch_fp4", "fp4", 1, 64, 8, (16, 96), (1, 1), 16),
        # the next turns of 8 conversations behind what the eviction kept of the earlier ones
        _append("append_turn", "bf16", 1, 8, 8, (128, 983), (200, 2500), 64),
        # the benchmark's retained rows: all layers of the 8B shape, 983 rows of a 32k prompt
        _gather("gather_8b_32k", "bf16", 32, 1, 8, (32768, 32768), 983, "heads", 64),
        # a packed ragged batch evicted into 4 bits
        _gather("gather_ragged_fp4", "fp4", 32, 8, 8, (4096, 16384), 512, "tokens", 32),
        # one layer's compact rows out of 4 bits, to be scored again
        _read("read_layer_fp4", "fp4", 1, 1, 8, (983, 983), 64),
        # a batch that moves out of the pages, 8 layers at a time
        _read("read_batch", "bf16", 8, 16, 8, (512, 2048), 128),
        # decoding one token over a compacted 32k prompt: a model calls this once per layer
        _attention("attention_layer", "bf16", 1, 32, 8, (1046, 1046), (1, 1), 0.0, 64),
        # decoding one token of each of 64 sequences with a small budget in 4 bits, capped scores, small pages
        _attention("attention_batch_fp4", "fp4", 64, 32, 8, (256, 1100), (1, 1), 50.0, 16),
        # a 128k cache in 4 bits, 8 query heads per KV head
        _attention("attention_long_fp4", "fp4", 1, 64, 8, (131071, 131071), (1, 1), 0.0, 128),
        # four drafted tokens of each of 32 sequences, 8 query heads per KV head
        _attention("attention_verify", "bf16", 32, 64, 8, (1024, 8192), (4, 4), 0.0, 64),
        # the next turns of 8 conversations: as much arithmetic as a prompt
        _attention("attention_turn", "bf16", 8, 32, 8, (983, 983), (200, 2500), 0.0, 64),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    fmt = rng.choice(("bf16", "fp4"))
    kv_heads = rng.choice((8, 8, 8, 4, 2, 1, 5))
    page_rows = rng.choice((16, 16, 32, 64, 128, 256))
    kind = rng.choice(("append", "gather", "read", "attention", "attention", "attention"))

    def between(high):
        return (high, high) if rng.random() < 0.5 else (max(1, high // rng.randint(2, 8)), high)

    while True:
        layers = rng.choice((1, 1, 2, 8, 32))
        batch = _log_int(rng, 1, 64)
        if kind == "append":
            held = between(_log_int(rng, 1, 2048))
            new = (1, 1) if rng.random() < 0.4 else between(_log_int(rng, 2, 2500))
            # no more rows than the largest listed case writes, no more in the pools than the benchmark's
            if layers * batch * new[1] * kv_heads <= 150000 and layers * batch * (held[1] + new[1]) * kv_heads <= 400000:
                case = _append(None, fmt, layers, batch, kv_heads, held, new, page_rows)
                break
        elif kind == "gather":
            keys = between(_log_int(rng, 64, 32768))
            budget = min(_log_int(rng, 16, 4096), keys[1])
            if layers * batch * kv_heads * keys[1] <= 8.4e6 and layers * batch * kv_heads * budget <= 260000:
                case = _gather(None, fmt, layers, batch, kv_heads, keys, budget, rng.choice(("heads", "tokens")), page_rows)
                break
        elif kind == "read":
            held = between(_log_int(rng, 1, 8192))
            if layers * batch * kv_heads * held[1] <= 2.0e6:
                case = _read(None, fmt, layers, batch, kv_heads, held, page_rows)
                break
        else:
            group = rng.choice((4, 4, 8, 2, 1, 7))
            held = between(_log_int(rng, 16, 131071))
            draw_new = rng.random()
            new = (1, 1) if draw_new < 0.5 else between(_log_int(rng, 2, 16)) if draw_new < 0.75 else between(_log_int(rng, 16, 2500))
            rows = held[1] + new[1]
            if batch * kv_heads * rows <= 1.6e6 and batch * kv_heads * group * new[1] * rows <= 1.6e9:
                case = _attention(None, fmt, batch, kv_heads * group, kv_heads, held, new, rng.choice((0.0, 0.0, 30.0, 50.0)), page_rows)
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
    return held, _drawn(case, "new") if "new_low" in case else [0] * case["batch"]


def work(case):
    held, new = _rows(case)
    heads = case["layers"] * case["kv_heads"]
    row = 68 if case["format"] == "fp4" else 2 * HEAD_DIM
    value = 2 * HEAD_DIM
    rows_all = heads * (sum(held) + sum(new))
    read_back = 2 * rows_all * (row + value) if case["format"] == "fp4" else 0
    if case["kind"] == "append":
        n = heads * sum(new)
        return {"bytes": 2 * n * (value + row) + 4 * sum(new) + read_back, "flops": 3 * HEAD_DIM * n}
    if case["kind"] == "gather":
        return {"bytes": rows_all * (2 * (value + row) + 4) + read_back, "flops": 0}
    if case["kind"] == "read":
        return {"bytes": 2 * rows_all * (row + value), "flops": 0}
    pairs = sum(n * h + n * (n + 1) // 2 for h, n in zip(held, new)) * case["q_heads"]
    return {"bytes": 2 * rows_all * row + 2 * sum(new) * case["q_heads"] * value, "flops": 4 * HEAD_DIM * pairs}


# --- plain forms of the format -------------------------------------------------------------------------------------------
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


def _quantise(x):
    """bf16 [..., 128] -> codes uint8 [..., 64] and scale bytes uint8 [..., 4]."""
    g = x.to(torch.float32).unflatten(-1, (4, 32))
    largest = g.abs().amax(-1)
    bad = ~torch.isfinite(g).all(-1)
    m, e = torch.frexp(torch.where(bad, 1.0, largest))           # largest = m * 2^e, 1/2 <= m < 1: 7 * 2^(e - 3) = 0.875 * 2^e
    e = torch.where(m > 0.875, e - 2, e - 3)
    e = torch.where(largest == 0, -125, e).clamp(-125, 125)
    y = torch.where(bad.unsqueeze(-1), 0.0, g.abs()) * _power_of_two(-e.unsqueeze(-1))
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
    y = torch.clamp(torch.round(y / step) * step, max=6.0)
    code = torch.bucketize(y, torch.tensor(LEVELS, device=x.device)).to(torch.uint8)
    code = code + torch.where((g < 0) & ~bad.unsqueeze(-1), 8, 0).to(torch.uint8)
    code = code.flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), torch.where(bad, 255, e + 127).to(torch.uint8)


def _values(codes, scales):
    """float32 values [..., 128] of codes and scale bytes."""
    table = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=codes.device)
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).to(torch.int32)
    two = torch.where(scales == 255, float("nan"), _power_of_two(scales.to(torch.int32) - 127))
    return (table[c].unflatten(-1, (4, 32)) * two.unsqueeze(-1)).flatten(-2)


def _bf16(gen, *shape):
    """N(0, 1) in bf16."""
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)


def _model_keys(gen, *shape):
    """Keys as a model leaves them: some channels are several times as large as the others in every row."""
    gain = torch.ones(HEAD_DIM, device="cuda")
    gain[::17] = 4.0
    return _bf16(gen, *shape) * gain.to(torch.bfloat16)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    held, new = _rows(case)
    layers, batch, heads, page_rows = case["layers"], case["batch"], case["kv_heads"], case["page_rows"]
    rows = [h + n for h, n in zip(held, new)]
    pages_of = [(n + page_rows - 1) // page_rows for n in rows]
    max_pages = max(pages_of)
    n_pages = sum(pages_of) + max(1, sum(pages_of) // 8)
    fp4 = case["format"] == "fp4"
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
    written = case["kind"] in ("append", "gather")
    for name, keys in (("k", True), ("v", False)):
        x = torch.zeros(pool + (HEAD_DIM,), dtype=torch.bfloat16, device="cuda") if case["kind"] == "gather" else \
            (_model_keys if keys else _bf16)(gen, *pool, HEAD_DIM)
        if fp4:
            codes = torch.empty(pool + (HEAD_DIM // 2,), dtype=torch.uint8, device="cuda")
            scales = torch.empty(pool + (4,), dtype=torch.uint8, device="cuda")
            step = max(1, (1 << 26) // (heads * page_rows * HEAD_DIM))
            for layer in range(layers):
                for p in range(0, n_pages, step):
                    codes[layer, p:p + step], scales[layer, p:p + step] = _quantise(x[layer, p:p + step])
            state[name], state[name + "_scales"] = codes, scales
        else:
            state[name], state[name + "_scales"] = x, None
    if new[0] or max(new):
        total = sum(new)
        ragged = case["new_low"] != case["new_high"]
        state["cu_new"] = _int32([sum(new[:b]) for b in range(batch + 1)]) if ragged else None
        state["total_new"], state["max_new"] = total, max(new)
    if case["kind"] == "append":
        state["k_new"] = _model_keys(gen, layers, total, heads, HEAD_DIM)
        state["v_new"] = _bf16(gen, layers, total, heads, HEAD_DIM)
        # the positions go on behind the prompt that was evicted, far behind the rows that were kept of it
        first = [33 * h for h in held]
        state["positions"] = _int32([f + t for f, n in zip(first, new) for t in range(n)])
    if case["kind"] == "attention":
        state["q"] = _bf16(gen, 1, total, case["q_heads"], HEAD_DIM) * 1.5
        state["out"] = torch.empty_like(state["q"])
    if case["kind"] == "gather":
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
    if case["kind"] == "read" or (written and fp4):
        shape = (layers, batch, heads, max(rows), HEAD_DIM)
        state["k_out"] = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
        state["v_out"] = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
        state["filled"] = _int32(rows)
    if own:
        import paper_2603_11564_amd as D
        state["pages"] = D.make_pages(n_layers=layers, batch=batch, n_kv_heads=heads, page_rows=page_rows, n_pages=n_pages,
                                      max_pages=max_pages, format=case["format"], k=state["k"], v=state["v"],
                                      k_scales=state["k_scales"], v_scales=state["v_scales"], table=table)
        if max(new):
            q_heads = case.get("q_heads", heads)
            kv = (total * heads * HEAD_DIM, heads * HEAD_DIM, HEAD_DIM)
            state["step"] = D.make_step(n_q_heads=q_heads, total_new=total, max_new=max(new), cu_new=state["cu_new"],
                                        lengths=state["lengths"], k_strides=kv, v_strides=kv,
                                        q_strides=(total * q_heads * HEAD_DIM, q_heads * HEAD_DIM, HEAD_DIM),
                                        scale=SCALE, softcap=case.get("softcap", 0.0))
        if case["kind"] == "attention":
            n = D.paged_attention_workspace_bytes(state["pages"], state["step"])
            state["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
        if case["kind"] == "gather":
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
    if kind == "append":
        D.dapq_paged_append(s["pages"], s["step"], s["k_new"], s["v_new"], s["positions"], THETA, 0)
    elif kind == "gather":
        D.dapq_paged_gather(s["shape"], s["pages"], s["k_prompt"], s["v_prompt"], s["idx"], s["count"], s["case"]["budget"])
    if "k_out" in s:
        D.dapq_paged_read(s["pages"], s["filled"], max(s["rows"]), s["k_out"], s["v_out"])
        return s["k_out"], s["v_out"]
    return s["k"], s["v"]


# --- the same in elementary operations -------------------------------------------------------------------------------------
def _places(s, first, count):
    """Rows first[b] .. first[b] + count[b] - 1 of every sequence, one after the other: their pages and slots."""
    page_rows = s["case"]["page_rows"]
    total = sum(count)
    seq = torch.repeat_interleave(torch.arange(len(count), device="cuda"), torch.tensor(count, device="cuda"), output_size=total)
    start = torch.tensor([f - sum(count[:b]) for b, f in enumerate(first)], device="cuda")
    row = torch.arange(total, device="cuda") + start[seq]
    return seq, row, s["table"][seq, row // page_rows].long(), row % page_rows


def _put(s, name, page, slot, x):
    """x: bf16 [layer][row][head][d] into the pool."""
    if s[name + "_scales"] is None:
        s[name][:, page, :, slot] = x.transpose(0, 1)
    else:
        codes, scales = _quantise(x)
        s[name][:, page, :, slot] = codes.transpose(0, 1)
        s[name + "_scales"][:, page, :, slot] = scales.transpose(0, 1)


def _read_plain(s):
    seq, row, page, slot = _places(s, [0] * len(s["rows"]), s["rows"])
    out = []
    for name in ("k", "v"):
        x = s[name][:, page, :, slot]                               # [row][layer][head][...]
        if s[name + "_scales"] is not None:
            x = _values(x, s[name + "_scales"][:, page, :, slot]).to(torch.bfloat16)
        s[name + "_out"][:, seq, :, row] = x
        out.append(s[name + "_out"])
    return tuple(out)


def _rotated(x, positions):
    """x: bf16 [layer][row][head][d]; channel c is paired with c + 64.  Angles and products in 64 bits, rounded once."""
    half = HEAD_DIM // 2
    omega = THETA ** (-2.0 * torch.arange(half, device="cuda", dtype=torch.float64) / HEAD_DIM)
    angle = positions.to(torch.float64)[:, None, None] * omega
    a, b = x[..., :half].to(torch.float64), x[..., half:].to(torch.float64)
    return _bf16_once(torch.cat((a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()), -1))


def _attention_plain(s):
    case = s["case"]
    batch, heads = case["batch"], case["kv_heads"]
    group, longest, most_new = case["q_heads"] // heads, max(s["rows"]), s["max_new"]
    page_rows = case["page_rows"]
    row = torch.arange(longest, device="cuda")
    page = s["table"][:, row // page_rows].long().clamp(min=0)      # [seq][row]

    def rows_of(name):
        x = s[name][0, page, :, (row % page_rows).expand(batch, -1)]  # [seq][row][head][...]
        if s[name + "_scales"] is not None:
            x = _values(x, s[name + "_scales"][0, page, :, (row % page_rows).expand(batch, -1)])
        return x.to(torch.float32).transpose(1, 2)

    new = torch.tensor(s["new"], device="cuda")
    start = new.cumsum(0) - new
    token = torch.arange(most_new, device="cuda")
    at = (start[:, None] + token).clamp(max=s["total_new"] - 1)     # [seq][token]
    q = s["q"][0][at].to(torch.float32).unflatten(2, (heads, group)).permute(0, 2, 3, 1, 4).flatten(2, 3)  # [seq][head][group * token][d]
    x = torch.matmul(q, rows_of("k").transpose(-1, -2)) * SCALE
    if case["softcap"]:
        x = torch.tanh(x / case["softcap"]) * case["softcap"]
    visible = s["lengths"][:, None].long() + token + 1              # [seq][token]
    hidden = (row >= visible[..., None])[:, None, None].expand(-1, heads, group, -1, -1).flatten(2, 3)
    x = x.masked_fill(hidden, -math.inf)
    x = torch.exp(x - x.amax(-1, keepdim=True))
    x = torch.matmul(x / x.sum(-1, keepdim=True), rows_of("v"))
    x = x.unflatten(2, (group, most_new)).permute(0, 3, 1, 2, 4).flatten(2, 3)  # [seq][token][q head][d]
    s["out"][0] = x[token < new[:, None]].to(torch.bfloat16)
    return s["out"]


def run(state):
    if own:
        return _run_own(state)
    s, kind = state, state["case"]["kind"]
    if kind == "attention":
        return _attention_plain(s)
    if kind == "append":
        _, _, page, slot = _places(s, s["held"], s["new"])
        _put(s, "k", page, slot, _rotated(s["k_new"], s["positions"]))
        _put(s, "v", page, slot, s["v_new"])
    elif kind == "gather":
        seq, row, page, slot = _places(s, [0] * len(s["rows"]), s["rows"])
        token = (s["idx"][:, seq, :, row] + torch.tensor(s["cu"], device="cuda")[seq][:, None, None]).long()  # [row][layer][head]
        layer = torch.arange(s["case"]["layers"], device="cuda")[:, None]
        head = torch.arange(s["case"]["kv_heads"], device="cuda")
        for name in ("k", "v"):
            x = s[name + "_prompt"]
            x = x[layer, head, token] if s["case"]["layout"] == "heads" else x[layer, token, head]
            _put(s, name, page, slot, x.transpose(0, 1))
    if "k_out" in s:
        return _read_plain(s)
    return s["k"], s["v"]


# --- from the definition, in 64 bits ---------------------------------------------------------------------------------------
def _nearest_fp4(x):
    """float64 [..., 32] groups -> what FP4 keeps of them: the level whose distance is least, the even code of two."""
    largest = x.abs().amax(-1, keepdim=True)
    scale = torch.full_like(largest, 2.0 ** -125)
    for e in range(-124, 126):
        scale = torch.where(largest > 7.0 * 2.0 ** (e - 1), 2.0 ** e, scale)
    y = x.abs() / scale
    got = torch.zeros_like(y)
    for code in range(1, 8):
        middle = 0.5 * (LEVELS[code - 1] + LEVELS[code])
        got = torch.where((y >= middle) if code % 2 == 0 else (y > middle), LEVELS[code], got)
    return got * scale * torch.sign(x)


def _held_values(s, name, layer, b, n):
    """float64 [head][n][d]: the first n rows of sequence b in one layer."""
    page_rows = s["case"]["page_rows"]
    pages = s["table"][b, :(n + page_rows - 1) // page_rows].long()
    def rows(x):
        return x[layer].index_select(0, pages).permute(1, 0, 2, 3).flatten(1, 2)[:, :n]
    x = rows(s[name])
    if s[name + "_scales"] is None:
        return x.double()
    levels = torch.tensor(LEVELS, dtype=torch.float64, device="cuda")
    codes = torch.empty(x.shape[:2] + (HEAD_DIM,), dtype=torch.long, device="cuda")
    codes[..., 0::2], codes[..., 1::2] = (x & 15).long(), (x >> 4).long()
    powers = torch.tensor([2.0 ** (e - 127) for e in range(255)] + [math.nan], dtype=torch.float64, device="cuda")
    return levels[codes % 8] * (1 - 2 * (codes // 8)) * powers[rows(s[name + "_scales"]).long()].repeat_interleave(32, -1)


def _new_values(s, name, layer, b, fp4):
    """float64 [head][n][d]: the new rows of sequence b as the cache holds them (bf16: before their one rounding)."""
    at = sum(s["new"][:b])
    x = s[name + "_new"][layer, at:at + s["new"][b]].double()
    if name == "k":
        turn = torch.polar(torch.ones(64, dtype=torch.float64, device="cuda"),
                           s["positions"][at:at + s["new"][b], None, None].double()
                           * torch.exp(torch.arange(64, dtype=torch.float64, device="cuda") * (-math.log(THETA) / 64)))
        z = torch.complex(x[..., :64], x[..., 64:]) * turn
        x = torch.cat((z.real, z.imag), -1)
    x = x.transpose(0, 1)
    if not fp4:
        return x
    apart = x * (2.0 ** 45 + 1.0)                                    # the nearest number of 53 - 45 = 8 bits, as bf16 has
    return _nearest_fp4((apart - (apart - x)).unflatten(-1, (4, 32))).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    fp4, kind = case["format"] == "fp4", case["kind"]
    layers, batch, heads, page_rows = case["layers"], case["batch"], case["kv_heads"], case["page_rows"]
    if kind == "attention":
        group = case["q_heads"] // heads
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        for b in range(batch):
            n, held = s["new"][b], s["held"][b]
            at = sum(s["new"][:b])
            k, v = _held_values(s, "k", 0, b, held + n), _held_values(s, "v", 0, b, held + n)
            seen = torch.arange(held + n, device="cuda") <= held + torch.arange(n, device="cuda")[:, None]
            for h in range(case["q_heads"]):
                x = s["q"][0, at:at + n, h].double() @ k[h // group].T * SCALE
                if case["softcap"]:
                    x = case["softcap"] * torch.tanh(x / case["softcap"])
                out[0, at:at + n, h] = torch.softmax(x.masked_fill(~seen, -math.inf), -1) @ v[h // group]
        return out
    dense = "k_out" in s
    result = []
    for name in ("k", "v"):
        if dense:
            got = torch.zeros(s[name + "_out"].shape, dtype=torch.float64, device="cuda")
        else:
            got = s[name].double()
        for layer in range(layers):
            for b in range(batch):
                if kind == "gather":
                    n = s["held"][b]
                    rows = s["idx"][layer, b, :, :n].long() + s["cu"][b]
                    x = s[name + "_prompt"][layer]
                    x = x if case["layout"] == "heads" else x.transpose(0, 1)
                    x = torch.stack([x[h].index_select(0, rows[h]) for h in range(heads)]).double()
                    if fp4:
                        x = _nearest_fp4(x.unflatten(-1, (4, 32))).flatten(-2)
                    first = 0
                elif kind == "append":
                    x, first = _new_values(s, name, layer, b, fp4), s["held"][b]
                    if dense:
                        got[layer, b, :, :first] = _held_values(s, name, layer, b, first)
                else:
                    x, first = _held_values(s, name, layer, b, s["held"][b]), 0
                if dense:
                    got[layer, b, :, first:first + x.shape[1]] = x
                else:
                    place = torch.arange(first, first + x.shape[1], device="cuda")
                    got[layer, s["table"][b].long()[place // page_rows], :, place % page_rows] = x.transpose(0, 1)
        result.append(got)
    return tuple(result)
