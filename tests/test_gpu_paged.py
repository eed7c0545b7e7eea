"""The cache in pages on the GPU against its float64 definition: rows written, appended and read bit for bit, attention
within bounds that follow from its arithmetic."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2603_11564_amd as D  # noqa: E402
from dapq_harness import Problem  # noqa: E402
from oracle import dapq_oracle as O  # noqa: E402
from oracle import paged_oracle as PO  # noqa: E402
from paged_harness import (JUNK, SCALE, THETA, Cache, attend, attention_bound, dev_bits, dev_int, make_step, normal_bits, same_pool,  # noqa: E402
                           starts, strided)

pytestmark = pytest.mark.gpu
FORMATS = ("bf16", "fp4")


def special_rows(rng, n):
    """Rows [n][128] with groups that are zero, tiny, huge, not finite, and full of values half way between two levels."""
    x = rng.standard_normal((n, 128)) * np.exp(rng.uniform(-40, 40, (n, 4))).repeat(32, 1)
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 6.75])
    for i in range(n):
        g = slice(32 * (i % 4), 32 * (i % 4) + 32)
        kind = i % 9
        if kind == 0:
            x[i, g] = 0.0
        elif kind == 1:
            x[i, g] = rng.choice((-1.0, 1.0), 32) * rng.choice(ties, 32) * 2.0 ** rng.integers(-20, 20)
        elif kind == 2:
            x[i, g] = rng.standard_normal(32) * 2.0 ** -126
        elif kind == 3:
            x[i, g] = rng.uniform(-1, 1, 32) * 3.3e38
        elif kind == 4:
            x[i, 32 * (i % 4) + 7] = np.inf
        elif kind == 5:
            x[i, 32 * (i % 4) + 30] = np.nan
        elif kind == 6:
            x[i, g] = -0.0
    return O.f64_to_bf16_bits(x)


# --- gather -----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("layers,heads,lens,budget,page_rows,layout", [
    (1, 1, [1], 1, 16, "thd"),
    (2, 3, [50, 0, 33, 7], 20, 16, "thd"),
    (1, 8, [300], 983, 64, "hnd"),
    (3, 5, [40, 130], 65, 32, "thd"),
    (1, 2, [700], 600, 1024, "hnd"),
])
def test_gather(fmt, layers, heads, lens, budget, page_rows, layout):
    rng = np.random.default_rng(layers * 100 + budget)
    cu = starts(lens)
    tokens = int(cu[-1])
    k, v = (special_rows(rng, layers * tokens * heads).reshape(layers, tokens, heads, 128) for _ in range(2))
    prob = Problem(normal_bits(rng, layers, len(lens), heads, 1, 128), k, v, heads, cu if len(lens) > 1 else None, layout, SCALE)
    keep = [min(budget, n) for n in lens]
    idx = np.full((layers, len(lens), heads, budget), -7, dtype=np.int32)
    count = np.zeros((layers, len(lens), heads), dtype=np.int32)
    for layer, b, h in np.ndindex(count.shape):
        idx[layer, b, h, :keep[b]] = np.sort(rng.permutation(lens[b])[:keep[b]])
        count[layer, b, h] = keep[b]
    if keep[0] > 3:
        idx[0, 0, 0, 2], idx[0, 0, 0, 3] = lens[0], -1            # outside the prompt: left as they were
        count[0, 0, 0] = budget + 5 if keep[0] == budget else keep[0]  # (more than the budget: the budget)
    cache = Cache(rng, fmt, layers, heads, page_rows, keep)
    if keep[0] > page_rows:
        cache.table[0, 1] = cache.n_pages if layers > 1 else -3   # a page that there is not
    cache.to_device()
    D.dapq_paged_gather(prob.shape, cache.pages, prob.k, prob.v, torch.from_numpy(idx).cuda(), torch.from_numpy(count).cuda(), budget)
    same_pool(cache.from_device(), PO.gather(cache.pool, cache.table, k, v, cu, idx, count))


def test_gather_into_a_table_with_less_room():
    rng = np.random.default_rng(5)
    k, v = normal_bits(rng, 1, 100, 2, 128), normal_bits(rng, 1, 100, 2, 128)
    prob = Problem(normal_bits(rng, 1, 1, 2, 1, 128), k, v, 2, None, "thd", SCALE)
    cache = Cache(rng, "bf16", 1, 2, 16, [48], extra_entries=0).to_device()
    idx = np.tile(np.arange(100, dtype=np.int32), (1, 1, 2, 1))
    count = np.full((1, 1, 2), 100, dtype=np.int32)
    D.dapq_paged_gather(prob.shape, cache.pages, prob.k, prob.v, torch.from_numpy(idx).cuda(), torch.from_numpy(count).cuda(), 100)
    same_pool(cache.from_device(), PO.gather(cache.pool, cache.table, k, v, [0, 100], idx, count))


# --- append -----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("layers,heads,page_rows,lengths,new,ragged,pairing,pads", [
    (1, 8, 64, [983], [1], False, 0, (0, 0)),
    (1, 1, 16, [0], [1], True, 1, (0, 0)),
    (2, 3, 16, [0, 15, 16, 40], [17, 1, 0, 33], True, 0, (8, 16)),
    (1, 5, 32, [31, 5, 0], [4, 4, 4], False, 1, (0, 8)),
    (1, 11, 16, [7], [50], True, 0, (0, 0)),
    (3, 2, 128, [0, 0], [0, 130], True, None, (64, 0)),
    (1, 2, 16, list(range(150)), [1 + b % 3 for b in range(150)], True, 0, (0, 0)),
    (1, 2, 16, [3] * 200, [0] * 64 + [2] + [0] * 100 + [3] + [0] * 34, True, 0, (0, 0)),
])
def test_append(fmt, layers, heads, page_rows, lengths, new, ragged, pairing, pads):
    rng = np.random.default_rng(heads * 1000 + page_rows)
    total = sum(new)
    k, v = (special_rows(rng, layers * total * heads).reshape(layers, total, heads, 128) for _ in range(2))
    positions = None if pairing is None else rng.integers(0, 1 << 20, total).astype(np.int32)
    cache = Cache(rng, fmt, layers, heads, page_rows, [h + n for h, n in zip(lengths, new)]).fill(rng, [min(h, 20) for h in lengths]).to_device()
    dk, ks = strided(k, *pads)
    dv, vs = strided(v, pads[1], pads[0])
    step = make_step(lengths, new, ragged, heads, k_strides=ks, v_strides=vs)
    D.dapq_paged_append(cache.pages, step, dk, dv, None if positions is None else dev_int(positions), THETA, pairing or 0)
    with np.errstate(invalid="ignore"):
        want = PO.append(cache.pool, cache.table, lengths, starts(new), max(new), k, v, positions, THETA, "interleaved" if pairing else "half")
    got = cache.from_device()
    if fmt == "bf16":                                             # (NaNs are NaNs)
        for name in got:
            for a in (got[name], want[name]):
                a[(a & 0x7fff) > 0x7f80] = JUNK
    same_pool(got, want)


def test_append_what_has_no_place():
    """More tokens than max_new, rows past the table, pages that there are not, negative lengths: left out, the rest is there."""
    rng = np.random.default_rng(3)
    lengths, new = [10, 40, 14, -2, 2 ** 31 - 3], [9, 20, 6, 4, 5]
    k, v = normal_bits(rng, 1, 44, 2, 128), normal_bits(rng, 1, 44, 2, 128)
    cache = Cache(rng, "fp4", 1, 2, 16, [32, 48, 32, 16, 48], extra_entries=0)
    cache.table[2, 1], cache.table[0, 0] = 1 << 30, -2 ** 31
    cache.to_device()
    (dk, ks), (dv, vs) = strided(k), strided(v)
    positions = rng.integers(0, 1 << 17, 44).astype(np.int32)
    step = make_step(lengths, new, True, 2, max_new=12, k_strides=ks, v_strides=vs)
    D.dapq_paged_append(cache.pages, step, dk, dv, dev_int(positions), THETA)
    same_pool(cache.from_device(), PO.append(cache.pool, cache.table, lengths, starts(new), 12, k, v, positions, THETA))


# --- read -------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("layers,heads,page_rows,lengths,max_rows", [
    (1, 1, 16, [1], 1), (2, 3, 16, [0, 17, 64, 33], 40), (1, 8, 64, [200], 200), (1, 2, 512, [700, 3], 1000)])
def test_read(fmt, layers, heads, page_rows, lengths, max_rows):
    rng = np.random.default_rng(max_rows)
    cache = Cache(rng, fmt, layers, heads, page_rows, lengths).fill(rng, lengths)
    if lengths[-1] > page_rows:
        cache.table[-1, 0] = -1
    cache.to_device()
    outs = [dev_bits(np.full((layers, len(lengths), heads, max_rows, 128), JUNK, np.uint16)) for _ in range(2)]
    D.dapq_paged_read(cache.pages, dev_int([n + (5000 if b == 1 else 0) for b, n in enumerate(lengths)]), max_rows, *outs)
    lengths = [n + (5000 if b == 1 else 0) for b, n in enumerate(lengths)]
    want = PO.read(cache.pool, cache.table, lengths, max_rows, JUNK)
    for got, ref in zip(outs, want):
        got = got.view(torch.int16).cpu().numpy().view(np.uint16)
        got[(got & 0x7fff) > 0x7f80] = JUNK
        ref[(ref & 0x7fff) > 0x7f80] = JUNK
        assert np.array_equal(got, ref)


def test_every_code_and_scale_is_read_exactly():
    """Codes 0..15 with every scale byte that the calls write, and 255."""
    rng = np.random.default_rng(1)
    cache = Cache(rng, "fp4", 1, 1, 256, [512], extra_entries=0)
    cache.pool["k"][:] = rng.integers(0, 256, cache.pool["k"].shape)
    for page in range(cache.n_pages):
        cache.pool["k_scales"][0, page, 0] = (np.arange(2, 258)[:, None] + np.arange(4) * 64 - 2) % 251 + 2
    cache.pool["k_scales"][0, 0, 0, 7] = 255
    cache.pool["v"][:], cache.pool["v_scales"][:] = cache.pool["k"], cache.pool["k_scales"]
    cache.to_device()
    outs = [torch.zeros((1, 1, 1, 512, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    D.dapq_paged_read(cache.pages, dev_int([512]), 512, *outs)
    want = PO.read(cache.pool, cache.table, [512], 512, 0)
    for got, ref in zip(outs, want):
        np.testing.assert_array_equal(got.double().cpu().numpy(), O.bf16_bits_to_f64(ref))


# --- attention --------------------------------------------------------------------------------------------------------------
def check_attention(cache, lengths, new, q_bits, softcap=0.0, scale=SCALE, **kw):
    got = attend(cache, lengths, new, q_bits, scale=scale, softcap=softcap, **kw)
    out, weighted, size = PO.attention(cache.pool, cache.table, lengths, starts(new), O.bf16_bits_to_f64(q_bits), float(np.float32(scale)), softcap)
    error = np.abs(got - out)
    group = q_bits.shape[2] // cache.heads
    bound = attention_bound(out, weighted, size, group * max(new))
    worst = np.unravel_index(np.nanargmax(error / bound), error.shape)
    assert np.isfinite(got).all() and (error <= bound).all(), (worst, got[worst], out[worst], bound[worst])
    return got


ATTENTION = [  # layers, kv heads, group, page_rows, lengths, new
    (1, 1, 1, 16, [0], [1]),
    (1, 8, 4, 64, [982], [1]),
    (1, 2, 4, 16, [0, 1, 15, 16, 31, 32, 33, 500], [1] * 8),
    (2, 3, 5, 32, [70, 0, 9], [1, 1, 1]),
    (1, 1, 8, 16, [100, 3], [1, 1]),
    (1, 2, 16, 128, [300], [1]),
    (1, 1, 17, 16, [40], [1]),
    (1, 1, 64, 16, [90], [1]),
    (1, 2, 4, 16, [33, 0, 250], [4, 4, 4]),
    (1, 2, 8, 32, [60, 17], [4, 2]),
    (2, 1, 3, 16, [0, 5, 40], [37, 0, 20]),
    (1, 2, 4, 64, [100, 0], [70, 130]),
    (1, 1, 7, 16, [0, 300], [1, 90]),
    (1, 1, 1, 16, [3000], [2]),
    (1, 2, 4, 16, [5 * b for b in range(70)], [b % 3 for b in range(70)]),
]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("softcap", [0.0, 20.0])
@pytest.mark.parametrize("case", range(len(ATTENTION)))
def test_attention(fmt, softcap, case):
    layers, heads, group, page_rows, lengths, new = ATTENTION[case]
    rng = np.random.default_rng(100 + case)
    rows = [h + n for h, n in zip(lengths, new)]
    cache = Cache(rng, fmt, layers, heads, page_rows, rows).fill(rng, rows, gain=2.0).to_device()
    q = normal_bits(rng, layers, sum(new), heads * group, 128)
    check_attention(cache, lengths, new, q, softcap, ragged=len(set(new)) > 1, pads=(8, 16) if case % 2 else (0, 0))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("case", range(len(ATTENTION)))
def test_attention_through_a_wide_table(fmt, case):
    """A table of 20000 rows a sequence, most of which have no page: the parts that rows are shared out in follow the lengths, not the table."""
    layers, heads, group, page_rows, lengths, new = ATTENTION[case]
    rng = np.random.default_rng(300 + case)
    rows = [h + n for h, n in zip(lengths, new)]
    cache = Cache(rng, fmt, layers, heads, page_rows, rows, extra_entries=20000 // page_rows).fill(rng, rows, gain=2.0).to_device()
    check_attention(cache, lengths, new, normal_bits(rng, layers, sum(new), heads * group, 128), ragged=len(set(new)) > 1)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("page_rows", [16, 32, 64, 128, 256, 512, 1024])
@pytest.mark.parametrize("new", [1, 30])
def test_pages_of_all_sizes(fmt, page_rows, new):
    rng = np.random.default_rng(page_rows)
    rows = [1030 + new, 250 + new]
    cache = Cache(rng, fmt, 1, 1, page_rows, rows).fill(rng, rows).to_device()
    q = normal_bits(rng, 1, 2 * new, 2, 128)
    got = check_attention(cache, [1030, 250], [new, new], q, ragged=False)
    assert np.array_equal(attend(cache, [1030, 250], [new, new], q, max_new=1 << 30, ragged=False), got)


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_long_sequence_among_many(fmt):
    """150 sequences, one of which has most of the rows, some none: parts of all lengths, also of sequences past the first 64."""
    rng = np.random.default_rng(301)
    lengths = [int(n) for n in rng.integers(0, 40, 150)]
    lengths[3], lengths[100] = 700, 2500
    new = [int(n) for n in rng.integers(0, 3, 150)]
    new[100] = 2
    rows = [h + n for h, n in zip(lengths, new)]
    cache = Cache(rng, fmt, 1, 1, 16, rows, extra_entries=1000).fill(rng, rows).to_device()
    for group in (4, 16):
        check_attention(cache, lengths, new, normal_bits(rng, 1, sum(new), group, 128))


@pytest.mark.parametrize("softcap", [0.01, 1.0, 64.0, 65.0, 300.0, 1e6, 1e30])
@pytest.mark.parametrize("new", [1, 9])
def test_caps_of_all_sizes(softcap, new):
    """Scores far above the cap, around it and far below it (there the cap changes nothing)."""
    rng = np.random.default_rng(71)
    cache = Cache(rng, "bf16", 1, 1, 32, [150 + new]).fill(rng, [150 + new], gain=3.0).to_device()
    check_attention(cache, [150], [new], normal_bits(rng, 1, new, 4, 128), softcap, scale=0.5)


@pytest.mark.parametrize("softcap", [2.0 ** -100, 2.0 ** 108])
@pytest.mark.parametrize("new", [1, 9])
def test_caps_at_the_ends_of_their_range(softcap, new):
    """Next to the smallest and the largest caps that are taken with this scale, also where a score is 0."""
    rng = np.random.default_rng(72)
    cache = Cache(rng, "bf16", 1, 1, 32, [150 + new]).fill(rng, [150 + new], gain=3.0).to_device()
    q = normal_bits(rng, 1, new, 4, 128)
    q[:, :, 1] = 0
    check_attention(cache, [150], [new], q, softcap, scale=0.5)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [40, 3, 33, 20]])
def test_attention_with_pages_missing(fmt, new):
    """Rows on no page are left out, whatever the other pages hold; a query without any row gets zeros."""
    rng = np.random.default_rng(9)
    lengths = [100, 40, 64, 20]
    rows = [h + n for h, n in zip(lengths, new)]
    cache = Cache(rng, fmt, 1, 2, 16, rows)
    cache.table[0, 1], cache.table[0, 2], cache.table[1, 0], cache.table[2, :] = -1, cache.n_pages, 1 << 30, -5
    cache.table[3, 1:] = -1
    cache.fill(rng, rows).to_device()
    got = check_attention(cache, lengths, new, normal_bits(rng, 1, sum(new), 8, 128))
    assert not got[0, starts(new)[2]:starts(new)[3]].any()


@pytest.mark.parametrize("fmt", FORMATS)
def test_attention_without_visible_rows(fmt):
    """Lengths of -1 and less leave the first tokens of a sequence without a row, and the table's end cuts the others."""
    rng = np.random.default_rng(2)
    cache = Cache(rng, fmt, 1, 1, 16, [32, 32, 32], extra_entries=0).fill(rng, [32, 32, 32]).to_device()
    q = normal_bits(rng, 1, 9, 2, 128)
    got = attend(cache, [-2, 31, 2 ** 31 - 2], [3, 3, 3], q)
    want, weighted, size = PO.attention(cache.pool, cache.table, [-2, 31, 31], [0, 3, 6, 9], O.bf16_bits_to_f64(q), SCALE)
    assert not got[0, :2].any() and (np.abs(got - want) <= attention_bound(want, weighted, size, 6)).all()


@pytest.mark.parametrize("new", [1, 20])
def test_attention_of_extreme_scores(new):
    """One key far above all others, keys of -inf, and logits of some hundreds with a scale of one."""
    rng = np.random.default_rng(4)
    lengths = [200]
    cache = Cache(rng, "bf16", 1, 2, 16, [200 + new]).fill(rng, [200 + new], gain=4.0)
    q = normal_bits(rng, 1, new, 4, 128)
    page, slot = PO.place(cache.table, cache.n_pages, 16, 0, 170)
    cache.pool["k"][0, page, 0, slot] = O.f64_to_bf16_bits(O.bf16_bits_to_f64(q[0, 0, 0]) * 3)
    cache.to_device()
    check_attention(cache, lengths, [new], q, scale=1.0)
    check_attention(cache, lengths, [new], q, scale=1.0, softcap=5.0)
    # a key whose logits are -inf (and +inf for others) weighs nothing where it is -inf
    cache.pool["k"][0, page, :, slot] = O.f64_to_bf16_bits(np.full(128, 0.0))
    cache.pool["k"][0, page, :, slot, 0] = O.f64_to_bf16_bits(np.array([-np.inf]))
    q[..., 0] = O.f64_to_bf16_bits(np.array([0.5]))
    cache.to_device()
    check_attention(cache, lengths, [new], q)


def test_attention_of_no_numbers():
    """A NaN in a visible key or value reaches the rows that see it and no others."""
    rng = np.random.default_rng(6)
    cache = Cache(rng, "bf16", 1, 2, 16, [60, 60]).fill(rng, [60, 60])
    page, slot = PO.place(cache.table, cache.n_pages, 16, 0, 52)
    cache.pool["k"][0, page, 0, slot, 3] = JUNK
    cache.to_device()
    q = normal_bits(rng, 1, 20, 4, 128)
    got = attend(cache, [50, 50], [10, 10], q)
    nan = np.isnan(got)
    assert nan[0, 2:10, :2].all() and not nan[0, :2].any() and not nan[0, 10:].any() and not nan[0, :, 2:].any()


@pytest.mark.parametrize("group,new", [(1, 1), (4, 1), (2, 3), (8, 2), (4, 7), (2, 60)])
def test_values_that_are_not_finite(group, new):  # (2 x 60: turns)
    """An infinite value or a NaN among the values of the new tokens reaches the tokens from its own on; what nobody sees reaches nobody."""
    rng = np.random.default_rng(60 + new)
    before = 45
    cache = Cache(rng, "bf16", 1, 2, 16, [before + new + 30]).fill(rng, [before + new])
    plant = {5: (0, np.inf), 20: (1, np.nan), before: (2, -np.inf), before + new // 2: (3, np.nan), before + new - 1: (4, np.inf)}
    for row, (channel, value) in plant.items():
        page, slot = PO.place(cache.table, cache.n_pages, 16, 0, row)
        cache.pool["v"][0, page, 1, slot, channel] = O.f64_to_bf16_bits(np.array([value]))[0]
    cache.to_device()
    q = normal_bits(rng, 1, new, 2 * group, 128)
    got = attend(cache, [before], [new], q)
    with np.errstate(invalid="ignore"):
        want, weighted, size = PO.attention(cache.pool, cache.table, [before], [0, new], O.bf16_bits_to_f64(q), SCALE)
    finite = np.isfinite(want)
    assert not finite[0, :, group:, :2].any() and finite[0, :, :group].all() and finite[0, :, :, 5:].all()
    assert np.array_equal(np.isnan(got), np.isnan(want)) and (got[np.isinf(want)] == want[np.isinf(want)]).all()
    with np.errstate(invalid="ignore"):
        assert (np.abs(got - want) <= attention_bound(want, weighted, size, group * new))[finite].all()


@pytest.mark.parametrize("new", [[2, 40], [0, 0]])
def test_tokens_past_max_new_are_left_out(new):
    rng = np.random.default_rng(8)
    cache = Cache(rng, "bf16", 1, 1, 16, [60, 80]).fill(rng, [60, 80]).to_device()
    q = normal_bits(rng, 1, max(sum(new), 1), 2, 128)[:, :sum(new)]
    if not sum(new):
        q = q.reshape(1, 0, 2, 128)
        step = make_step([5, 5], new, True, 2, max_new=0, q_strides=(256, 256, 128))
        D.dapq_paged_attention(cache.pages, step, dev_bits(normal_bits(rng, 1, 1, 2, 128)), torch.zeros(256, dtype=torch.bfloat16, device="cuda"),
                               torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"))
        return
    got = attend(cache, [30, 30], new, q, max_new=7)
    want, weighted, size = PO.attention(cache.pool, cache.table, [30, 30], [0, 2, 42], O.bf16_bits_to_f64(q), SCALE)
    seen = list(range(2)) + list(range(2, 9))
    assert (np.abs(got - want) <= attention_bound(want, weighted, size, 100))[0, seen].all()
    assert np.isnan(got[0, 9:]).all()                            # (what the buffer held)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("heads,group,page_rows,lengths,new", [
    (1, 4, 16, [1000], [16]), (2, 1, 64, [700, 0, 130], [33, 50, 200]), (1, 8, 32, [0], [129]), (3, 5, 16, [64, 1], [64, 63]),
    (1, 2, 128, [0] * 70, [b % 5 * 20 for b in range(70)])])
def test_turns(fmt, heads, group, page_rows, lengths, new):
    """Blocks of columns that end in a token, rows shared out and not, tiles and pages of all sizes, a page missing."""
    rng = np.random.default_rng(500 + heads)
    rows = [h + n for h, n in zip(lengths, new)]
    cache = Cache(rng, fmt, 1, heads, page_rows, rows).fill(rng, rows, gain=2.0)
    if rows[0] > 3 * page_rows:
        cache.table[0, 2] = -1
    cache.to_device()
    check_attention(cache, lengths, new, normal_bits(rng, 1, sum(new), heads * group, 128), softcap=15.0 if heads == 3 else 0.0, ragged=len(new) > 1)


def test_turns_past_max_new_are_left_out():
    rng = np.random.default_rng(18)
    cache = Cache(rng, "bf16", 1, 1, 16, [160, 180]).fill(rng, [160, 180]).to_device()
    q = normal_bits(rng, 1, 150, 4, 128)
    got = attend(cache, [30, 30], [60, 90], q, max_new=35)
    want, weighted, size = PO.attention(cache.pool, cache.table, [30, 30], [0, 60, 150], O.bf16_bits_to_f64(q), SCALE)
    seen = list(range(35)) + list(range(60, 95))
    assert (np.abs(got - want) <= attention_bound(want, weighted, size, 140))[0, seen].all()
    assert np.isnan(got[0, 35:60]).all() and np.isnan(got[0, 95:]).all()


def test_many_rows_are_the_mean_of_their_values():
    """40000 rows with keys of zero: the output is the mean of the values (here whole numbers below 256, whose sums fp32 holds exactly)."""
    rng = np.random.default_rng(12)
    n = 40000
    cache = Cache(rng, "bf16", 1, 2, 64, [n], extra_entries=0)
    cache.pool["k"][:] = 0
    cache.pool["v"][:] = O.f64_to_bf16_bits(rng.integers(-4, 5, cache.pool["v"].shape).astype(np.float64))
    cache.to_device()
    order = cache.table[0]
    v = O.bf16_bits_to_f64(cache.pool["v"][0, order]).transpose(1, 0, 2, 3).reshape(2, -1, 128)[:, :n].mean(1)
    got = attend(cache, [n - 1], [1], normal_bits(rng, 1, 1, 8, 128))
    want = np.repeat(v, 4, 0)
    assert (np.abs(got[0, 0] - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -20).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_pools_of_more_than_four_gigabytes(fmt):
    """Pages at the far end of a pool whose rows' bytes pass 32 bits."""
    rng = np.random.default_rng(7)
    heads, page_rows, row = 8, 256, 256 if fmt == "bf16" else 64
    n_pages = (5 << 30) // (heads * page_rows * row)
    rows = 700
    small = Cache(rng, fmt, 1, heads, page_rows, [rows], spare=0, extra_entries=0).fill(rng, [rows])
    far = {n: torch.zeros((1, n_pages) + a.shape[2:], dtype=torch.uint8 if a.dtype == np.uint8 else torch.int16, device="cuda") for n, a in small.pool.items()}
    for n, a in small.pool.items():
        far[n][:, -small.n_pages:] = torch.from_numpy(a.view(np.int16 if a.dtype == np.uint16 else a.dtype)).cuda()
    table = dev_int((small.table[0] + n_pages - small.n_pages).tolist())
    small.pages = D.make_pages(n_layers=1, batch=1, n_kv_heads=heads, page_rows=page_rows, n_pages=n_pages, max_pages=small.max_pages, format=fmt,
                               k=far["k"], v=far["v"], k_scales=far.get("k_scales"), v_scales=far.get("v_scales"), table=table)
    q = normal_bits(rng, 1, 12, heads * 4, 128)
    check_attention(small, [rows - 12], [12], q)
    k, v = normal_bits(rng, 1, 5, heads, 128), normal_bits(rng, 1, 5, heads, 128)
    (dk, ks), (dv, vs) = strided(k), strided(v)
    D.dapq_paged_append(small.pages, make_step([rows - 5], [5], False, heads, k_strides=ks, v_strides=vs), dk, dv, dev_int(range(5)), THETA)
    want = PO.append(small.pool, small.table, [rows - 5], [0, 5], 5, k, v, np.arange(5), THETA)
    for n, a in want.items():
        assert np.array_equal(far[n][:, -small.n_pages:].cpu().numpy().view(a.dtype), a)
    assert not far["k"][:, :-small.n_pages].any()
    outs = [torch.zeros((1, 1, heads, rows, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    D.dapq_paged_read(small.pages, dev_int([rows]), rows, *outs)
    for got, ref in zip(outs, PO.read(want, small.table, [rows], rows, 0)):
        assert np.array_equal(got.view(torch.int16).cpu().numpy().view(np.uint16), ref)


# --- together ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", FORMATS)
def test_evict_decode_and_evict_again(fmt):
    """A prompt is scored and evicted into pages; three steps of decoding append and attend; the rows are read back, agree with what the compact
    cache of dapq_gather and the rotation of dapq_rope_apply give, and are scored and evicted again."""
    rng = np.random.default_rng(21)
    layers, heads, group, length, budget, page_rows = 2, 2, 4, 300, 60, 16
    k, v = normal_bits(rng, layers, length, heads, 128), normal_bits(rng, layers, length, heads, 128)
    prob = Problem(normal_bits(rng, layers, 1, heads * group, 16, 128), k, v, heads, None, "thd", SCALE)
    idx, count, _ = prob.pool_topk(prob.score(), 7, budget)
    cache = Cache(rng, fmt, layers, heads, page_rows, [budget + 20]).to_device()
    D.dapq_paged_gather(prob.shape, cache.pages, prob.k, prob.v, idx, count, budget)
    compact = prob.gather(idx, count, budget)
    expect = PO.gather(cache.pool, cache.table, k, v, [0, length], idx.cpu().numpy(), count.cpu().numpy())
    lengths = dev_int([budget])
    rows, position = budget, length
    for new in (1, 3, 1):
        kn, vn = normal_bits(rng, layers, new, heads, 128), normal_bits(rng, layers, new, heads, 128)
        (dk, ks), (dv, vs) = strided(kn), strided(vn)
        q = normal_bits(rng, layers, new, heads * group, 128)
        dq, qs = strided(q)
        step = D.make_step(n_q_heads=heads * group, total_new=new, max_new=new, lengths=lengths, k_strides=ks, v_strides=vs, q_strides=qs, scale=SCALE)
        positions = np.arange(position, position + new)
        out = torch.empty((layers, new, heads * group, 128), dtype=torch.bfloat16, device="cuda")
        work = torch.empty(D.paged_attention_workspace_bytes(cache.pages, step), dtype=torch.uint8, device="cuda")
        D.dapq_paged_append(cache.pages, step, dk, dv, dev_int(positions), THETA)
        D.dapq_paged_attention(cache.pages, step, dq, out, work)
        expect = PO.append(expect, cache.table, [rows], [0, new], new, kn, vn, positions, THETA)
        want, weighted, size = PO.attention(expect, cache.table, [rows], [0, new], O.bf16_bits_to_f64(q), SCALE)
        assert (np.abs(out.double().cpu().numpy() - want) <= attention_bound(want, weighted, size, new * group)).all()
        lengths += new
        rows, position = rows + new, position + new
    same_pool(cache.from_device(), expect)
    outs = [torch.zeros((layers, 1, heads, rows, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    D.dapq_paged_read(cache.pages, lengths, rows, *outs)
    if fmt == "bf16":
        assert torch.equal(outs[0][..., :budget, :], compact[0]) and torch.equal(outs[1][..., :budget, :], compact[1])
    # again, over the rows that were read: [layer][seq][head][row][d]
    strides = (heads * rows * 128, 0, rows * 128, 128)
    shape = D.make_shape(n_layers=layers, batch=1, n_q_heads=heads * group, n_kv_heads=heads, n_pseudo=16, total_tokens=rows, k_strides=strides,
                         v_strides=strides, q_strides=(heads * group * 16 * 128, heads * group * 16 * 128, 16 * 128, 128), scale=SCALE)
    S = torch.empty((layers, heads, rows), dtype=torch.float32, device="cuda")
    D.dapq_score(shape, prob.q, outs[0], S, torch.empty(max(256, D.workspace_bytes(shape)), dtype=torch.uint8, device="cuda"))
    idx2 = torch.zeros((layers, 1, heads, 20), dtype=torch.int32, device="cuda")
    count2 = torch.zeros((layers, 1, heads), dtype=torch.int32, device="cuda")
    D.dapq_pool_topk(shape, S, 7, 20, None, idx2, count2)
    D.dapq_paged_gather(shape, cache.pages, *outs, idx2, count2, 20)
    kd, vd = (o[:, 0].transpose(1, 2).contiguous().view(torch.int16).cpu().numpy().view(np.uint16) for o in outs)
    same_pool(cache.from_device(), PO.gather(expect, cache.table, kd, vd, [0, rows], idx2.cpu().numpy(), count2.cpu().numpy()))


@pytest.mark.parametrize("fmt", FORMATS)
def test_decoding_replayed_from_a_graph(fmt):
    """One step (append and attention, then the lengths and positions go on) recorded once and replayed; every replay is the eager step, bit for bit."""
    rng = np.random.default_rng(31)
    heads, group, page_rows, first = 2, 4, 16, [40, 3, 900]
    steps = 20

    def fresh():
        cache = Cache(np.random.default_rng(1), fmt, 1, heads, page_rows, [n + steps + 1 for n in first]).fill(np.random.default_rng(2), first).to_device()
        return cache, dev_int(first), dev_int([1000 + n for n in first])

    kn, vn = (torch.zeros((1, 3, heads, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q, out = (torch.zeros((1, 3, heads * group, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    data = [[dev_bits(normal_bits(rng, *t.shape)) for t in (kn, vn, q)] for _ in range(steps)]

    def make(cache, lengths):
        step = D.make_step(n_q_heads=heads * group, total_new=3, max_new=1, lengths=lengths, k_strides=(0, heads * 128, 128),
                           v_strides=(0, heads * 128, 128), q_strides=(0, heads * group * 128, 128), scale=SCALE)
        work = torch.full((D.paged_attention_workspace_bytes(cache.pages, step),), 0xA5, dtype=torch.uint8, device="cuda")

        def go(positions):
            D.dapq_paged_append(cache.pages, step, kn, vn, positions, THETA)
            D.dapq_paged_attention(cache.pages, step, q, out, work)
            lengths.add_(1)
            positions.add_(1)
        return go, work

    def load(i):
        for t, src in zip((kn, vn, q), data[i]):
            t.copy_(src)

    cache, lengths, positions = fresh()
    go, _ = make(cache, lengths)
    want = []
    for i in range(steps):
        load(i)
        go(positions)
        want.append(out.clone())
    eager = cache.from_device()
    cache, lengths, positions = fresh()
    go, work = make(cache, lengths)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    load(0)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        go(positions)
    lengths.copy_(dev_int(first))
    positions.copy_(dev_int([1000 + n for n in first]))
    for i in range(steps):
        load(i)
        work.fill_(0x5A)
        out.fill_(7.0)
        graph.replay()
        if i % 3 == 0:
            torch.cuda.synchronize()
        assert torch.equal(out, want[i]), i
    same_pool(cache.from_device(), eager)


def test_two_calls_at_once():
    """On two streams, with a workspace each, over pages that two sequences share."""
    rng = np.random.default_rng(42)
    cache = Cache(rng, "bf16", 1, 2, 16, [900, 900]).fill(rng, [900, 900])
    cache.table[1] = cache.table[0]
    cache.to_device()
    q = [normal_bits(rng, 1, 2, 8, 128) for _ in range(2)]
    want = [attend(cache, [898, 400], [1, 1], x) for x in q]
    assert not np.array_equal(want[0], want[1])
    calls = []
    for x in q:
        dq, strides = strided(x)
        step = make_step([898, 400], [1, 1], False, n_q_heads=8, q_strides=strides)
        calls.append((torch.cuda.Stream(), dq, step, torch.zeros((1, 2, 8, 128), dtype=torch.bfloat16, device="cuda"),
                      torch.empty(D.paged_attention_workspace_bytes(cache.pages, step), dtype=torch.uint8, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(20):
        for stream, dq, step, out, work in calls:
            D.dapq_paged_attention(cache.pages, step, dq, out, work, stream=stream)
    torch.cuda.synchronize()
    for call, ref in zip(calls, want):
        assert np.array_equal(call[3].double().cpu().numpy(), ref)


def test_on_another_stream():
    rng = np.random.default_rng(41)
    cache = Cache(rng, "fp4", 1, 2, 16, [600]).fill(rng, [600]).to_device()
    q = normal_bits(rng, 1, 1, 8, 128)
    want = attend(cache, [599], [1], q)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        got = attend(cache, [599], [1], q)
    assert np.array_equal(got, want)
