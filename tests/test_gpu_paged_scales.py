"""FP4 pages that hold what the calls themselves never write, every scale byte of the format: rows read back, and values behind scales whose
larger codes are infinite, in rows that all tokens see and in rows that only the later ones do."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2603_11564_amd as D  # noqa: E402
from oracle import dapq_oracle as O  # noqa: E402
from oracle import paged_oracle as PO  # noqa: E402
from paged_harness import SCALE, Cache, attend, attention_bound, dev_int, normal_bits  # noqa: E402

pytestmark = pytest.mark.gpu
COLUMNS = [(1, 1), (4, 1), (2, 3), (4, 2), (8, 2), (3, 5), (4, 7), (16, 2), (2, 17), (2, 60), (8, 40)]  # (query heads of a KV head, new tokens)
FINITE = {252: (0, 1, 2, 3, 4, 5, 6, 7), 253: (0, 1, 2, 3, 4, 5), 254: (0, 1, 2, 3)}             # magnitudes' codes: 4 * 2^126 is past bf16, 2 * 2^127 too


def test_every_scale_byte_is_read_exactly():
    """All 256 scale bytes in every group, each with all codes; what lies past bf16 is infinite."""
    cache = Cache(np.random.default_rng(0), "fp4", 1, 1, 16, [256], extra_entries=0)
    for name in ("k", "v"):
        for row in range(256):
            page, slot = PO.place(cache.table, cache.n_pages, 16, 0, row)
            cache.pool[name][0, page, 0, slot] = (np.arange(64) * 2 % 16 | ((np.arange(64) * 2 + 1) % 16) << 4)
            cache.pool[name + "_scales"][0, page, 0, slot] = (row + np.arange(4) * 64 + (name == "v") * 5) & 255
    cache.to_device()
    outs = [torch.zeros((1, 1, 1, 256, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    D.dapq_paged_read(cache.pages, dev_int([256]), 256, *outs)
    with np.errstate(over="ignore"):
        want = PO.read(cache.pool, cache.table, [256], 256, 0)
    for got, ref in zip(outs, want):
        np.testing.assert_array_equal(got.double().cpu().numpy(), O.bf16_bits_to_f64(ref))


def as_bf16(cache):
    """The cache's values as a pool of bf16 rows."""
    with np.errstate(over="ignore"):
        return {n: O.f64_to_bf16_bits(PO.fp4_values(cache.pool[n], cache.pool[n + "_scales"])) for n in ("k", "v")}


def plant(rng, cache, name, head, row, group, byte, codes):
    """A group of 32 channels with one scale byte and magnitudes out of `codes`, of either sign."""
    page, slot = PO.place(cache.table, cache.n_pages, cache.page_rows, 0, row)
    c = rng.choice(codes, 32) + rng.choice((0, 8), 32)
    cache.pool[name][0, page, head, slot, 16 * group:16 * group + 16] = c[0::2] | c[1::2] << 4
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
    return Cache(rng, "fp4", 1, 2, 16, [before + new + 30], extra_entries=1250 if wide else 1).fill(rng, [before + new])


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("group,new", COLUMNS)
def test_the_largest_scales(group, new, wide):
    """Finite values next to the largest bf16, in the rows of the first, a middle and the last token and in one before them.  With queries of 0 every weight is 1,
    and a channel has one such value, so that its sum stays in the range of fp32."""
    rng = np.random.default_rng(80 + new)
    before = 45
    for bytes_of in ((254, 253, 254, 253), (253, 254, 253, 254), (252, 252, 253, 254)):
        cache = cache_of(rng, before, new, wide)
        for g, (row, byte) in enumerate(zip((5, before, before + new // 2, before + new - 1), bytes_of)):
            plant(rng, cache, "v", 1, row, g, byte, FINITE[byte])
        cache.to_device()
        want = check(cache, before, new, np.zeros((1, new, 2 * group, 128), np.uint16), group)
        assert np.isfinite(want).all() and (np.abs(want[0, -1, group:]).reshape(group, 4, 32).max(-1) > 2.0 ** 110).all()


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("group,new", COLUMNS)
def test_the_smallest_scales(fmt, group, new):
    """Values below the smallest normal number, in both formats."""
    rng = np.random.default_rng(480 + new)
    before = 45
    cache = cache_of(rng, before, new, False)
    for row in range(before + new):
        for g, byte in enumerate((0, 1, 2, 8)):
            plant(rng, cache, "v", 1, row, g, byte, range(8))
    if fmt == "bf16":
        cache.pool.update(as_bf16(cache))
        del cache.pool["k_scales"], cache.pool["v_scales"]
        cache.fmt = fmt
    cache.to_device()
    q = normal_bits(rng, 1, new, 2 * group, 128)
    got = attend(cache, [before], [new], q)
    want, weighted, size = PO.attention(cache.pool, cache.table, [before], [0, new], O.bf16_bits_to_f64(q), SCALE)
    assert (np.abs(got - want) <= attention_bound(want, weighted, size, group * new)).all()


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("group,new", COLUMNS)
def test_values_past_the_largest_scales(group, new, wide):
    """Groups whose larger codes are infinite, beside finite ones of the same group: each reaches the tokens that see it."""
    rng = np.random.default_rng(180 + new)
    before = 45
    cache = cache_of(rng, before, new, wide)
    for g, (row, byte) in enumerate(zip((5, before, before + new // 2, before + new - 1), (253, 254, 253, 254))):
        plant(rng, cache, "v", 1, row, g, byte, range(8))
    cache.to_device()
    want = check(cache, before, new, np.zeros((1, new, 2 * group, 128), np.uint16), group)
    last = np.isinf(want[0, -1, group:].reshape(group, 4, 32))
    assert last.any(-1).all() and not last.all(-1).any() and np.isfinite(want[0, :, :group]).all()


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("group,new", COLUMNS)
def test_groups_without_a_number(group, new, wide):
    """Scale byte 255 among the values, of rows that all tokens see, that some see and that none does: NaN for the tokens that see it, in its channels."""
    rng = np.random.default_rng(280 + new)
    before = 45
    cache = cache_of(rng, before, new, wide)
    for g, row in enumerate((5, before, before + new // 2, before + new - 1)):
        plant(rng, cache, "v", 1, row, g, 255, range(8) if new % 2 else (0,))
    cache.to_device()
    want = check(cache, before, new, normal_bits(rng, 1, new, 2 * group, 128), group)
    nan = np.isnan(want[0, :, group:]).reshape(new, group, 4, 32)
    first_seen = (0, 0, new // 2, new - 1)
    for g, t in enumerate(first_seen):
        assert nan[t:, :, g].all() and not nan[:t, :, g].any()
    assert np.isfinite(want[0, :, :group]).all()


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("group,new", COLUMNS)
def test_keys_without_a_number(group, new, wide):
    """Scale byte 255 in a key: NaN for the tokens that see it and for no others."""
    rng = np.random.default_rng(380 + new)
    before = 45
    cache = cache_of(rng, before, new, wide)
    plant(rng, cache, "k", 0, before + new // 2, 2, 255, (0,))
    cache.to_device()
    want = check(cache, before, new, normal_bits(rng, 1, new, 2 * group, 128), group)
    assert np.isnan(want[0, new // 2:, :group]).all() and np.isfinite(want[0, :new // 2]).all() and np.isfinite(want[0, :, group:]).all()
