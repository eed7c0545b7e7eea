"""Pages of 8 bits on the GPU against their float64 definition: the tests of the other formats in this one, every code and scale byte, values that
are no bf16 number."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2603_11564_amd as D  # noqa: E402
import test_gpu_paged as P  # noqa: E402
from dapq_harness import Problem  # noqa: E402
from oracle import dapq_oracle as O  # noqa: E402
from oracle import paged_oracle as PO  # noqa: E402
from paged_harness import SCALE, THETA, Cache, attend, attention_bound, dev_bits, dev_int, make_step, normal_bits, same_pool, starts, strided  # noqa: E402

pytestmark = pytest.mark.gpu
COLUMNS = [(1, 1), (4, 1), (2, 3), (4, 2), (8, 2), (3, 5), (4, 7), (16, 2), (2, 17), (2, 60), (8, 40)]  # (query heads of a KV head, new tokens)


def special_rows(rng, n):
    """Rows [n][128] with groups that are zero, tiny, huge (up to the largest bf16), not finite, and full of values half way between two levels."""
    x = rng.standard_normal((n, 128)) * np.exp(rng.uniform(-40, 40, (n, 4))).repeat(32, 1)
    ties = (PO.E4M3_LEVELS[:-1] + PO.E4M3_LEVELS[1:]) / 2
    for i in range(n):
        g = slice(32 * (i % 4), 32 * (i % 4) + 32)
        kind = i % 10
        if kind == 0:
            x[i, g] = 0.0
        elif kind == 1:
            x[i, g] = rng.choice((-1.0, 1.0), 32) * rng.choice(ties, 32) * 2.0 ** rng.integers(-20, 20)
            x[i, g.start] = rng.choice((448.0, 464.0, 468.0, 232.0)) * 2.0 ** rng.integers(-20, 20)
        elif kind == 2:
            x[i, g] = rng.standard_normal(32) * 2.0 ** -118
        elif kind == 3:
            x[i, g] = rng.uniform(-1, 1, 32) * 3.389e38
            x[i, g.start] = 3.3895e38
        elif kind == 4:
            x[i, 32 * (i % 4) + 7] = np.inf
        elif kind == 5:
            x[i, 32 * (i % 4) + 30] = np.nan
        elif kind == 6:
            x[i, g] = -0.0
        elif kind == 7:
            x[i, g] = rng.standard_normal(32) * 2.0 ** -128
    return O.f64_to_bf16_bits(x)


# --- rows -------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("layers,heads,lens,budget,page_rows,layout", [
    (1, 1, [1], 1, 16, "thd"), (2, 3, [50, 0, 33, 7], 20, 16, "thd"), (1, 8, [300], 983, 64, "hnd"), (3, 5, [40, 130], 65, 32, "thd"),
    (1, 2, [700], 600, 1024, "hnd")])
def test_gather(layers, heads, lens, budget, page_rows, layout):
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
    cache = Cache(rng, "e4m3", layers, heads, page_rows, keep).to_device()
    D.dapq_paged_gather(prob.shape, cache.pages, prob.k, prob.v, torch.from_numpy(idx).cuda(), torch.from_numpy(count).cuda(), budget)
    same_pool(cache.from_device(), PO.gather(cache.pool, cache.table, k, v, cu, idx, count))


@pytest.mark.parametrize("layers,heads,page_rows,lengths,new,ragged,pairing,pads", [
    (1, 8, 64, [983], [1], False, 0, (0, 0)), (1, 1, 16, [0], [1], True, 1, (0, 0)), (2, 3, 16, [0, 15, 16, 40], [17, 1, 0, 33], True, 0, (8, 16)),
    (1, 5, 32, [31, 5, 0], [4, 4, 4], False, 1, (0, 8)), (1, 11, 16, [7], [50], True, 0, (0, 0)), (3, 2, 128, [0, 0], [0, 130], True, None, (64, 0)),
    (1, 32, 16, [3, 9], [300, 400], True, 0, (0, 0)), (1, 2, 16, list(range(150)), [1 + b % 3 for b in range(150)], True, 0, (0, 0))])
def test_append(layers, heads, page_rows, lengths, new, ragged, pairing, pads):
    rng = np.random.default_rng(heads * 1000 + page_rows)
    total = sum(new)
    k, v = (special_rows(rng, layers * total * heads).reshape(layers, total, heads, 128) for _ in range(2))
    positions = None if pairing is None else rng.integers(0, 1 << 20, total).astype(np.int32)
    cache = Cache(rng, "e4m3", layers, heads, page_rows, [h + n for h, n in zip(lengths, new)]).fill(rng, [min(h, 20) for h in lengths]).to_device()
    (dk, ks), (dv, vs) = strided(k, *pads), strided(v, pads[1], pads[0])
    step = make_step(lengths, new, ragged, heads, k_strides=ks, v_strides=vs)
    D.dapq_paged_append(cache.pages, step, dk, dv, None if positions is None else dev_int(positions), THETA, pairing or 0)
    with np.errstate(invalid="ignore"):
        want = PO.append(cache.pool, cache.table, lengths, starts(new), max(new), k, v, positions, THETA, "interleaved" if pairing else "half")
    same_pool(cache.from_device(), want)


def test_every_code_and_scale_byte_is_read_exactly():
    """All 256 scale bytes, each with all 256 codes (K has the codes without a sign, V those with one); what lies past bf16 is infinite."""
    cache = Cache(np.random.default_rng(0), "e4m3", 1, 1, 16, [1024], extra_entries=0)
    for row in range(1024):
        page, slot = PO.place(cache.table, cache.n_pages, 16, 0, row)
        for name, sign in (("k", 0), ("v", 128)):
            cache.pool[name][0, page, 0, slot] = np.arange(128) + sign
            cache.pool[name + "_scales"][0, page, 0, slot] = (row // 4 + (row + np.arange(4)) % 4 * 64) & 255
    cache.to_device()
    outs = [torch.zeros((1, 1, 1, 1024, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    D.dapq_paged_read(cache.pages, dev_int([1024]), 1024, *outs)
    with np.errstate(over="ignore"):
        want = PO.read(cache.pool, cache.table, [1024], 1024, 0)
    for got, ref in zip(outs, want):
        np.testing.assert_array_equal(got.double().cpu().numpy(), O.bf16_bits_to_f64(ref))


@pytest.mark.parametrize("layers,heads,page_rows,lengths,max_rows", [
    (1, 1, 16, [1], 1), (2, 3, 16, [0, 17, 64, 33], 40), (1, 8, 64, [200], 200), (1, 2, 512, [700, 3], 1000), (2, 8, 64, [2100], 2100)])
def test_read(layers, heads, page_rows, lengths, max_rows):
    P.test_read("e4m3", layers, heads, page_rows, lengths, max_rows)


# --- attention, as in the other formats -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("softcap,case", [(c, i) for c in (0.0, 20.0) for i in range(len(P.ATTENTION))] + [(100.0, i) for i in (1, 4, 8, 9, 11)])
def test_attention(softcap, case):
    P.test_attention("e4m3", softcap, case)


@pytest.mark.parametrize("case", range(len(P.ATTENTION)))
def test_attention_through_a_wide_table(case):
    P.test_attention_through_a_wide_table("e4m3", case)


@pytest.mark.parametrize("page_rows", [16, 32, 64, 128, 256, 512, 1024])
@pytest.mark.parametrize("new", [1, 30])
def test_pages_of_all_sizes(page_rows, new):
    P.test_pages_of_all_sizes("e4m3", page_rows, new)


def test_a_long_sequence_among_many():
    P.test_a_long_sequence_among_many("e4m3")


@pytest.mark.parametrize("new", [[1, 1, 1, 1], [40, 3, 33, 20]])
def test_attention_with_pages_missing(new):
    P.test_attention_with_pages_missing("e4m3", new)


def test_attention_without_visible_rows():
    P.test_attention_without_visible_rows("e4m3")


@pytest.mark.parametrize("heads,group,page_rows,lengths,new", [
    (1, 4, 16, [1000], [16]), (2, 1, 64, [700, 0, 130], [33, 50, 200]), (1, 8, 32, [0], [129]), (3, 5, 16, [64, 1], [64, 63])])
def test_turns(heads, group, page_rows, lengths, new):
    P.test_turns("e4m3", heads, group, page_rows, lengths, new)


def test_pools_of_more_than_four_gigabytes():
    P.test_pools_of_more_than_four_gigabytes("e4m3")


def test_evict_decode_and_evict_again():
    P.test_evict_decode_and_evict_again("e4m3")


def test_decoding_replayed_from_a_graph():
    P.test_decoding_replayed_from_a_graph("e4m3")


# --- pages that hold what the calls themselves never write ----------------------------------------------------------------------
def as_bf16(cache):
    """The cache's values as a pool of bf16 rows."""
    with np.errstate(over="ignore"):
        return {n: O.f64_to_bf16_bits(PO.e4m3_values(cache.pool[n], cache.pool[n + "_scales"])) for n in ("k", "v")}


def plant(rng, cache, name, head, row, group, byte, codes):
    """A group of 32 channels with one scale byte and magnitudes out of `codes`, of either sign."""
    page, slot = PO.place(cache.table, cache.n_pages, cache.page_rows, 0, row)
    cache.pool[name][0, page, head, slot, 32 * group:32 * group + 32] = rng.choice(codes, 32) + rng.choice((0, 128), 32)
    cache.pool[name + "_scales"][0, page, head, slot, group] = byte


def check(cache, before, new, q_bits, group):
    got = attend(cache, [before], [new], q_bits)
    with np.errstate(invalid="ignore"):
        want, weighted, size = PO.attention(as_bf16(cache), cache.table, [before], [0, new], O.bf16_bits_to_f64(q_bits), SCALE)
        finite = np.isfinite(want)
        assert np.array_equal(np.isnan(got), np.isnan(want)) and (got[np.isinf(want)] == want[np.isinf(want)]).all()
        assert (np.abs(got - want) <= attention_bound(want, weighted, size, group * new))[finite].all()
    return want


def cache_of(rng, before, new, wide):
    """Rows for the tokens and junk behind them.  wide: a table in which rows are shared out."""
    return Cache(rng, "e4m3", 1, 2, 16, [before + new + 30], extra_entries=1250 if wide else 1).fill(rng, [before + new])


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("group,new", COLUMNS)
def test_the_largest_scales(group, new, wide):
    """Finite values next to the largest bf16: below 2^(374 - s) of the codes at scale byte s, all of them up to 246."""
    rng = np.random.default_rng(80 + new)
    before = 45
    for bytes_of in ((246, 247, 250, 254), (254, 251, 247, 246), (253, 246, 254, 249)):
        cache = cache_of(rng, before, new, wide)
        for g, (row, byte) in enumerate(zip((5, before, before + new // 2, before + new - 1), bytes_of)):
            plant(rng, cache, "v", 1, row, g, byte, range(127 if byte == 246 else 0x80 - 8 * (byte - 246)))
        cache.to_device()
        want = check(cache, before, new, np.zeros((1, new, 2 * group, 128), np.uint16), group)
        assert np.isfinite(want).all() and (np.abs(want[0, -1, group:]).reshape(group, 4, 32).max(-1) > 2.0 ** 110).all()


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("group,new", COLUMNS)
def test_values_past_the_largest_scales(group, new, wide):
    """Groups whose larger codes are infinite, beside finite ones of the same group: each reaches the tokens that see it."""
    rng = np.random.default_rng(180 + new)
    before = 45
    cache = cache_of(rng, before, new, wide)
    infinite = []
    for g, (row, byte) in enumerate(zip((5, before, before + new // 2, before + new - 1), (250, 247, 254, 252))):
        plant(rng, cache, "v", 1, row, g, byte, range(0x38, 127))
        page, slot = PO.place(cache.table, cache.n_pages, 16, 0, row)
        infinite.append((cache.pool["v"][0, page, 1, slot, 32 * g:32 * g + 32] & 127) >= 0x80 - 8 * (byte - 246))
    cache.to_device()
    want = check(cache, before, new, np.zeros((1, new, 2 * group, 128), np.uint16), group)
    # (at 247 seven of the 71 codes are infinite, and a draw of 32 may have none of them)
    assert (np.isinf(want[0, -1, group:].reshape(group, 4, 32)) == infinite).all() and np.isfinite(want[0, :, :group]).all()


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("group,new", COLUMNS)
@pytest.mark.parametrize("byte,codes", [(255, (0,)), (255, range(128)), (127, (127,)), (127, (20, 30, 127))])
def test_groups_without_a_number(group, new, wide, byte, codes):
    """Scale byte 255, or the code without a number, among the values of rows that all tokens see, that some see and that none does: NaN for the tokens that
    see it, in its channels."""
    rng = np.random.default_rng(280 + new)
    before = 45
    cache = cache_of(rng, before, new, wide)
    rows = (5, before, before + new // 2, before + new - 1)
    for g, row in enumerate(rows):
        plant(rng, cache, "v", 1, row, g, byte, codes)
    cache.to_device()
    want = check(cache, before, new, normal_bits(rng, 1, new, 2 * group, 128), group)
    nan = np.isnan(want[0, :, group:]).reshape(new, group, 4, 32)
    for g, row in enumerate(rows):
        t = max(0, row - before)
        assert nan[t:, :, g].any(-1).all() and not nan[:t, :, g].any()
        if len(codes) == 1 or byte == 255:
            assert nan[t:, :, g].all()
    assert np.isfinite(want[0, :, :group]).all()


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("group,new", COLUMNS)
@pytest.mark.parametrize("byte,code", [(255, 0), (127, 127)])
def test_keys_without_a_number(group, new, wide, byte, code):
    rng = np.random.default_rng(380 + new)
    before = 45
    cache = cache_of(rng, before, new, wide)
    plant(rng, cache, "k", 0, before + new // 2, 2, byte, (code,))
    cache.to_device()
    want = check(cache, before, new, normal_bits(rng, 1, new, 2 * group, 128), group)
    assert np.isnan(want[0, new // 2:, :group]).all() and np.isfinite(want[0, :new // 2]).all() and np.isfinite(want[0, :, group:]).all()


@pytest.mark.parametrize("group,new", COLUMNS)
def test_the_smallest_scales(group, new):
    """Values below the smallest normal number, as the calls never write them."""
    rng = np.random.default_rng(480 + new)
    before = 45
    cache = cache_of(rng, before, new, False)
    for row in range(before + new):
        for g, byte in enumerate((0, 1, 3, 9)):
            plant(rng, cache, "v", 1, row, g, byte, range(127))
    cache.to_device()
    q = normal_bits(rng, 1, new, 2 * group, 128)
    got = attend(cache, [before], [new], q)
    want, weighted, size = PO.attention(as_bf16(cache), cache.table, [before], [0, new], O.bf16_bits_to_f64(q), SCALE)
    assert (np.abs(got - want) <= attention_bound(want, weighted, size, group * new)).all()


def test_append_what_has_no_place():
    """More tokens than max_new, rows past the table, pages that there are not, negative lengths: left out, the rest is there."""
    rng = np.random.default_rng(3)
    lengths, new = [10, 40, 14, -2, 2 ** 31 - 3], [9, 20, 6, 4, 5]
    k, v = normal_bits(rng, 1, 44, 2, 128), normal_bits(rng, 1, 44, 2, 128)
    cache = Cache(rng, "e4m3", 1, 2, 16, [32, 48, 32, 16, 48], extra_entries=0)
    cache.table[2, 1], cache.table[0, 0] = 1 << 30, -2 ** 31
    cache.to_device()
    (dk, ks), (dv, vs) = strided(k), strided(v)
    positions = rng.integers(0, 1 << 17, 44).astype(np.int32)
    step = make_step(lengths, new, True, 2, max_new=12, k_strides=ks, v_strides=vs)
    D.dapq_paged_append(cache.pages, step, dk, dv, dev_int(positions), THETA)
    same_pool(cache.from_device(), PO.append(cache.pool, cache.table, lengths, starts(new), 12, k, v, positions, THETA))
