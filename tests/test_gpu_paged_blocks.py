"""Chosen blocks of a cache in pages on the GPU against their float64 definition: bounds and choices bit for bit, attention within bounds that follow from
its arithmetic."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2603_11564_amd as D  # noqa: E402
import test_gpu_paged_e4m3 as E4M3  # noqa: E402
import test_gpu_paged_scales as SCALES  # noqa: E402
from dapq_harness import Problem  # noqa: E402
from oracle import blocks_oracle as BO  # noqa: E402
from oracle import dapq_oracle as O  # noqa: E402
from oracle import paged_oracle as PO  # noqa: E402
from paged_harness import JUNK, SCALE, THETA, Cache, attend, attention_bound, dev_bits, dev_int, make_step, normal_bits, same_pool, starts, strided  # noqa: E402

pytestmark = pytest.mark.gpu
FORMATS = ("bf16", "fp4", "e4m3")


class Bounds:
    """The bounds of a cache's blocks on the host, 85 and -86 where nobody wrote, and on the device."""

    def __init__(self, cache, block_rows):
        shape = cache.pool["k"].shape[:3] + (cache.page_rows // block_rows,)
        self.block_rows = block_rows
        self.bounds, self.scales = np.full(shape + (2, 128), 85, np.int8), np.full(shape, 127, np.uint8)
        self.bounds[..., 1, :] = -86

    def to_device(self):
        self.dev, self.dev_scales = torch.from_numpy(self.bounds.copy()).cuda(), torch.from_numpy(self.scales.copy()).cuda()
        return self

    def blocks(self, **kw):
        return D.make_blocks(block_rows=self.block_rows, bounds=self.dev, scales=self.dev_scales, **kw)

    def random(self, rng, distinct=True):
        """Bounds of blocks that are alike or not, in a few scales."""
        mid, half = rng.integers(-60, 61, self.bounds.shape[:-2] + (128,)), rng.integers(0, 60, self.bounds.shape[:-2] + (128,))
        if not distinct:
            mid, half = mid[:, :1, :, :1] // 20 * 20 + 0 * mid, half[:, :1, :, :1] + 0 * half
        self.bounds[..., 0, :], self.bounds[..., 1, :] = mid + half, mid - half
        self.scales[:] = rng.integers(120, 124, self.scales.shape) if distinct else 122
        return self


# --- bounds -----------------------------------------------------------------------------------------------------------------
def check_bounds(cache, b, first, lengths, max_rows):
    b.to_device()
    D.dapq_paged_bounds(cache.pages, b.blocks(), None if first is None else dev_int(first), dev_int(lengths), max_rows)
    want, scales = BO.bounds(cache.pool, cache.table, b.block_rows, first, lengths, max_rows, b.bounds, b.scales)
    assert np.array_equal(b.dev_scales.cpu().numpy(), scales)
    assert np.array_equal(b.dev.cpu().numpy(), want)
    return want, scales


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("layers,heads,page_rows,block_rows,first,lengths,max_rows", [
    (1, 1, 16, 16, None, [16], 16),
    (1, 8, 64, 16, [31], [32], 1),
    (2, 3, 32, 16, [0, 15, 16, 17, 40, 5], [16, 16, 31, 33, 100, 5], 60),
    (1, 2, 64, 32, [-5, 64, 10], [70, 64, 200], 300),
    (1, 5, 128, 128, None, [300, 127, 128, 0], 300),
    (3, 1, 1024, 256, [0, 700], [1024, 1100], 1024),
    (1, 2, 16, 16, [0] * 70, [b for b in range(70)], 70),
    (1, 1, 256, 64, [100, 100], [1000, 400], 200),
])
def test_bounds(fmt, layers, heads, page_rows, block_rows, first, lengths, max_rows):
    """Only the blocks that the rows complete are written."""
    rng = np.random.default_rng(page_rows + block_rows)
    cache = Cache(rng, fmt, layers, heads, page_rows, lengths).fill(rng, lengths, gain=3.0).to_device()
    check_bounds(cache, Bounds(cache, block_rows), first, lengths, max_rows)


def test_bounds_of_keys_of_all_sizes():
    """Keys from subnormal to the largest, single outliers, zeros, equal rows, values on whole numbers of the unit, infinities and NaN."""
    rng = np.random.default_rng(5)
    n = 16 * 200
    cache = Cache(rng, "bf16", 1, 1, 64, [n], extra_entries=0)
    for b in range(n // 16):
        x = rng.standard_normal((16, 128)) * np.exp(rng.uniform(-88, 88)) * np.exp(rng.uniform(-8, 8, 128) * (b % 3))
        if b % 10 == 0:
            x[:] = 0.0
        elif b % 10 == 1:
            x = rng.integers(-127, 128, (16, 128)) * 2.0 ** float(rng.integers(-40, 40))
        elif b % 10 == 2:
            x[rng.integers(16), rng.integers(128)] = rng.choice([np.inf, -np.inf, np.nan])
        elif b % 10 == 3:
            x[:] = x[0]
        elif b % 10 == 4:
            x = rng.uniform(-1, 1, (16, 128)) * 3.38e38
        elif b % 10 == 5:
            x = rng.standard_normal((16, 128)) * 2.0 ** -128
        for i in range(16):
            page, slot = PO.place(cache.table, cache.n_pages, 64, 0, 16 * b + i)
            cache.pool["k"][0, page, 0, slot] = O.f64_to_bf16_bits(x[i])
    cache.to_device()
    for block_rows in (16, 64):
        _, scales = check_bounds(cache, Bounds(cache, block_rows), [0], [n], n)
        # (four kinds of rows share a block of 64, one of which is never all zero or tiny)
        assert ({77, 177, 255} if block_rows == 16 else {177, 255}) <= set(np.unique(scales).tolist())


@pytest.mark.parametrize("fmt", ["fp4", "e4m3"])
def test_bounds_of_codes_of_all_scales(fmt):
    rng = np.random.default_rng(6)
    n = 16 * 100
    cache = Cache(rng, fmt, 1, 1, 32, [n], extra_entries=0)
    cache.pool["k"][:] = rng.integers(0, 127 if fmt == "e4m3" else 256, cache.pool["k"].shape)
    cache.pool["k_scales"][:] = rng.integers(0, 256, cache.pool["k_scales"].shape[:2] + (1, 1, 1))
    cache.to_device()
    with np.errstate(over="ignore"):
        values = {"k": O.f64_to_bf16_bits(PO.code_values(cache.pool["k"], cache.pool["k_scales"]))}
    b = Bounds(cache, 16).to_device()
    D.dapq_paged_bounds(cache.pages, b.blocks(), None, dev_int([n]), n)
    want, scales = BO.bounds(values, cache.table, 16, None, [n], n, b.bounds, b.scales)
    assert np.array_equal(b.dev_scales.cpu().numpy(), scales) and np.array_equal(b.dev.cpu().numpy(), want)


def test_bounds_of_what_has_no_place():
    """Pages that there are not, lengths past the table and below zero; shared pages share their bounds."""
    rng = np.random.default_rng(7)
    cache = Cache(rng, "bf16", 1, 2, 16, [64, 64, 64, 64], extra_entries=0).fill(rng, [64] * 4)
    cache.table[0, 1], cache.table[1, 0], cache.table[1, 3], cache.table[2] = -1, cache.n_pages, -2 ** 31, cache.table[3]
    cache.to_device()
    check_bounds(cache, Bounds(cache, 16), [0, -2 ** 31, 2 ** 31 - 1, 48], [2 ** 31 - 1, 64, 2 ** 31 - 1, 64], 2 ** 31 - 1)
    check_bounds(cache, Bounds(cache, 16), None, [-5, 0, -2 ** 31, 15], 100)


# --- selection --------------------------------------------------------------------------------------------------------------
def choose(cache, b, lengths, new, q_bits, n_select, n_first=1, n_last=1, ragged=True, max_new=None, pads=(0, 0), stream=None):
    """dapq_paged_select on the device: idx and count as it leaves them, -7 where it writes nothing."""
    q, strides = strided(q_bits, *pads)
    step = make_step(lengths, new, ragged, n_q_heads=q_bits.shape[2], q_strides=strides, max_new=max_new)
    blocks = b.blocks(n_select=n_select, n_first=n_first, n_last=n_last)
    idx = torch.full((cache.layers, sum(new), cache.heads, n_select), -7, dtype=torch.int32, device="cuda")
    count = torch.full((cache.layers, sum(new), cache.heads), -7, dtype=torch.int32, device="cuda")
    n = D.paged_select_workspace_bytes(cache.pages, blocks, step)
    work = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    D.dapq_paged_select(cache.pages, blocks, step, q, idx, count, work, stream=stream)
    torch.cuda.synchronize()
    return idx.cpu().numpy(), count.cpu().numpy()


def check_choice(cache, b, lengths, new, q_bits, n_select, n_first=1, n_last=1, max_new=None, **kw):
    idx, count = choose(cache, b, lengths, new, q_bits, n_select, n_first, n_last, max_new=max_new, **kw)
    want = BO.select(cache.table, cache.n_pages, cache.page_rows, b.bounds, b.scales, b.block_rows, n_select, n_first, n_last, lengths, starts(new),
                     max(new) if max_new is None else max_new, O.bf16_bits_to_f64(q_bits))
    for at in np.ndindex(count.shape):
        chosen = want.get(at)
        if chosen is None:
            assert count[at] == -7 and (idx[at] == -7).all()
            continue
        assert count[at] == len(chosen), (at, count[at], len(chosen))
        assert idx[at][:len(chosen)].tolist() == chosen and (idx[at][len(chosen):] == -7).all(), at
    return idx, count


SELECT = [  # layers, kv heads, group, page_rows, block_rows, lengths, new, n_select, n_first, n_last
    (1, 1, 1, 16, 16, [0], [1], 1, 0, 1),
    (1, 8, 4, 64, 16, [1999], [1], 16, 1, 1),
    (2, 3, 5, 32, 16, [700, 0, 15, 16, 17], [1] * 5, 7, 2, 3),
    (1, 2, 4, 64, 32, [900, 33, 500], [4, 4, 4], 9, 1, 2),
    (1, 1, 8, 16, 16, [333, 90], [2, 3], 20, 0, 20),
    (1, 2, 7, 128, 64, [3000, 100], [3, 1], 5, 1, 1),
    (2, 1, 16, 64, 64, [1500], [5], 8, 0, 1),
    (1, 1, 17, 32, 32, [640], [2], 4, 1, 1),
    (1, 2, 40, 16, 16, [300, 20], [2, 1], 6, 1, 1),
    (1, 2, 2, 16, 16, [5 * b for b in range(70)], [b % 3 for b in range(70)], 4, 1, 1),
    (1, 2, 4, 64, 16, [100, 0], [70, 130], 3, 1, 1),
    (1, 1, 3, 1024, 16, [20000], [1], 300, 4, 4),
    (1, 1, 1, 256, 256, [9000], [1], 4096, 0, 1),
]


@pytest.mark.parametrize("distinct", [True, False])
@pytest.mark.parametrize("case", range(len(SELECT)))
def test_selection(case, distinct):
    """distinct: bounds of all sizes; else blocks that are all alike but one in each page, so that ties decide."""
    layers, heads, group, page_rows, block_rows, lengths, new, n_select, n_first, n_last = SELECT[case]
    rng = np.random.default_rng(900 + case)
    cache = Cache(rng, "bf16", layers, heads, page_rows, [h + n for h, n in zip(lengths, new)]).to_device()
    b = Bounds(cache, block_rows).random(rng, distinct).to_device()
    q = normal_bits(rng, layers, sum(new), heads * group, 128)
    check_choice(cache, b, lengths, new, q, n_select, n_first, n_last, ragged=len(set(new)) > 1, pads=(8, 16) if case % 2 else (0, 0))


@pytest.mark.parametrize("n_select", [1, 2, 3, 63, 64, 65, 255, 256, 1000, 4096])
def test_numbers_of_blocks(n_select):
    """One token of 2500 blocks, and of as many as are chosen, one more and one fewer, through tables of several widths."""
    rng = np.random.default_rng(n_select)
    for rows, wide in ((40000, 1), (16 * n_select, 600), (16 * n_select + 1, 1), (16 * n_select + 16, 5000), (max(1, 16 * n_select - 16), 1)):
        cache = Cache(rng, "bf16", 1, 1, 16, [rows], extra_entries=wide).to_device()
        b = Bounds(cache, 16).random(rng).to_device()
        check_choice(cache, b, [rows - 1], [1], normal_bits(rng, 1, 1, 4, 128), n_select, 0, 1)


@pytest.mark.parametrize("blocks,new", [(60, 1), (300, 1), (300, 2), (2100, 1), (2100, 2)])
def test_many_items(blocks, new):
    """A workgroup scores all blocks of an item and chooses: tables of up to 256, 2048 and 8192 blocks, sequences of all lengths in them."""
    rng = np.random.default_rng(blocks + new)
    lengths = [16 * blocks - 5 - new] + [int(n) for n in rng.integers(1, 900, 32)]
    lengths[20] = 0
    cache = Cache(rng, "bf16", 1, 8, 16, [n + new for n in lengths]).to_device()
    b = Bounds(cache, 16).random(rng).to_device()
    check_choice(cache, b, lengths, [new] * 33, normal_bits(rng, 1, 33 * new, 32, 128), 9, 1, 2, ragged=False)


@pytest.mark.parametrize("group,new", [(8, 4), (8, 5), (16, 2), (16, 7), (4, 9), (5, 3), (12, 16)])
def test_many_items_of_several_column_tiles(group, new):
    """Two tokens of a column tile and fewer: a workgroup has one; sequences with fewer tokens than others."""
    rng = np.random.default_rng(group * 100 + new)
    lengths = [int(n) for n in rng.integers(0, 700, 20)]
    tokens = [int(n) for n in rng.integers(0, new + 1, 20)]
    tokens[4] = new
    cache = Cache(rng, "bf16", 1, 4, 32, [n + new for n in lengths]).to_device()
    b = Bounds(cache, 16).random(rng).to_device()
    check_choice(cache, b, lengths, tokens, normal_bits(rng, 1, sum(tokens), 4 * group, 128), 6, 1, 1)
    new_all = [new] * 20
    check_choice(cache, b, lengths, new_all, normal_bits(rng, 1, 20 * new, 4 * group, 128), 6, 0, 1, ragged=False)


@pytest.mark.parametrize("rows,wide", [(500, 17000), (66000, 2000), (131000, 1), (270000, 1)])
def test_very_many_blocks(rows, wide):
    """Tables of more than 4096, 8192 and 16384 blocks, the last of which are read again for every round of a choice; all alike in a second go."""
    rng = np.random.default_rng(98)
    cache = Cache(rng, "bf16", 1, 1, 16, [rows], extra_entries=wide).to_device()
    for distinct in (True, False):
        b = Bounds(cache, 16).random(rng, distinct).to_device()
        check_choice(cache, b, [rows - 3], [3], normal_bits(rng, 1, 3, 2, 128), 300, 2, 1, ragged=False)


def test_selection_with_pages_missing():
    rng = np.random.default_rng(91)
    lengths, new = [500, 200, 64, 20], [1, 3, 2, 1]
    cache = Cache(rng, "bf16", 1, 2, 32, [h + n for h, n in zip(lengths, new)])
    cache.table[0, 1], cache.table[0, 2], cache.table[1, 0], cache.table[1, -2], cache.table[2, :] = -1, cache.n_pages, 1 << 30, -2 ** 31, -5
    cache.to_device()
    b = Bounds(cache, 16).random(rng).to_device()
    for n in (4, 30):
        _, count = check_choice(cache, b, lengths, new, normal_bits(rng, 1, 7, 8, 128), n, 2, 2)
        assert not count[0, 4:6].any()


def test_selection_without_visible_rows():
    """Lengths of -1 and less leave the first tokens of a sequence without a row, and the table's end cuts the others."""
    rng = np.random.default_rng(92)
    cache = Cache(rng, "bf16", 1, 1, 16, [160, 160, 160], extra_entries=0).to_device()
    b = Bounds(cache, 16).random(rng).to_device()
    _, count = check_choice(cache, b, [-2, 31, 2 ** 31 - 2], [3, 3, 3], normal_bits(rng, 1, 9, 2, 128), 4)
    assert count[0, :, 0].tolist() == [0, 0, 1, 2, 3, 3, 4, 4, 4]     # (33 rows: 3 blocks)


def test_blocks_that_are_not_finite_and_queries_that_are_not():
    """Scale byte 255 goes before all scores; a query with an infinity or a NaN scores 0 everywhere, queries of zero do, and huge and tiny ones
    are in units of their own."""
    rng = np.random.default_rng(93)
    cache = Cache(rng, "bf16", 1, 2, 16, [1000]).to_device()
    b = Bounds(cache, 16).random(rng)
    for block in (7, 30, 31, 55):
        page, _ = PO.place(cache.table, cache.n_pages, 16, 0, 16 * block)
        b.scales[0, page, :, 0] = 255
    b.to_device()
    q = normal_bits(rng, 1, 12, 8, 128)
    q[0, 1, 0, 5], q[0, 2, :, 77], q[0, 3, 2, 0] = 0x7f80, JUNK, 0xff80
    q[0, 4], q[0, 5, :4] = 0, 0
    q[0, 6] = O.f64_to_bf16_bits(rng.standard_normal((8, 128)) * 1e30)
    q[0, 7] = O.f64_to_bf16_bits(rng.standard_normal((8, 128)) * 1e-30)
    q[0, 8] = O.f64_to_bf16_bits(rng.standard_normal((8, 128)) * 2.0 ** -130)
    q[0, 9] = O.f64_to_bf16_bits(np.full((8, 128), 3.3e38))
    q[0, 10] = O.f64_to_bf16_bits(rng.integers(-4, 5, (8, 128)) + 0.5)                # (halves of the unit once the largest is 127)
    q[0, 10, :, 0] = O.f64_to_bf16_bits(np.full(8, 127.0))
    for n in (3, 5, 8):
        check_choice(cache, b, [980], [12], q, n, 1, 1)


@pytest.mark.parametrize("scale", [77, 100, 177])
def test_scales_at_the_ends_of_their_range(scale):
    rng = np.random.default_rng(94)
    cache = Cache(rng, "bf16", 1, 1, 16, [800]).to_device()
    b = Bounds(cache, 16).random(rng)
    b.scales[:] = scale
    b.to_device()
    for gain in (1e-30, 1.0, 1e20):
        check_choice(cache, b, [790], [2], O.f64_to_bf16_bits(rng.standard_normal((1, 2, 4, 128)) * gain), 6)


def test_tokens_past_max_new_are_left_out():
    rng = np.random.default_rng(95)
    cache = Cache(rng, "bf16", 2, 2, 16, [300, 380]).to_device()
    b = Bounds(cache, 16).random(rng).to_device()
    check_choice(cache, b, [200, 290], [2, 40], normal_bits(rng, 2, 42, 4, 128), 5, max_new=7)


def test_bounds_that_nobody_reads():
    """Bounds of the first and last blocks, and of what is on no page or past the lengths, may hold anything."""
    rng = np.random.default_rng(96)
    cache = Cache(rng, "bf16", 1, 1, 16, [400]).to_device()
    b = Bounds(cache, 16).random(rng).to_device()
    q = normal_bits(rng, 1, 2, 4, 128)
    want = choose(cache, b, [298], [2], q, 8, 2, 3)
    for block in [0, 1] + list(range(18, 25)):                       # 300 rows: 19 blocks, of which both tokens keep 17, 18 and one 16 or its own
        page, _ = PO.place(cache.table, cache.n_pages, 16, 0, 16 * block)
        b.bounds[0, page], b.scales[0, page] = rng.integers(-128, 128, (1, 1, 2, 128)), 255
    b.to_device()
    got = choose(cache, b, [298], [2], q, 8, 2, 3)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


def test_a_wide_selection_of_a_wide_step():
    """Sequences of 1 to 900 blocks, 64 and more of them, one with many tokens."""
    rng = np.random.default_rng(97)
    lengths = [int(n) for n in rng.integers(1, 3000, 80)]
    lengths[40] = 14400
    new = [int(n) for n in rng.integers(0, 2, 80)]
    new[3], new[40] = 30, 2
    cache = Cache(rng, "bf16", 1, 1, 64, [h + n for h, n in zip(lengths, new)]).to_device()
    b = Bounds(cache, 16).random(rng).to_device()
    check_choice(cache, b, lengths, new, normal_bits(rng, 1, sum(new), 2, 128), 12)


# --- attention --------------------------------------------------------------------------------------------------------------
def sparse(cache, lengths, new, q_bits, idx, count, block_rows, scale=SCALE, softcap=0.0, ragged=True, max_new=None, pads=(0, 0), stream=None):
    """dapq_paged_sparse_attention on the device; float64 [layers][tokens][n_q_heads][128]."""
    q, strides = strided(q_bits, *pads)
    step = make_step(lengths, new, ragged, n_q_heads=q_bits.shape[2], q_strides=strides, scale=scale, softcap=softcap, max_new=max_new)
    blocks = D.make_blocks(block_rows=block_rows, n_select=idx.shape[3])
    out = dev_bits(np.full(q_bits.shape, JUNK, dtype=np.uint16))
    work = torch.full((D.paged_sparse_attention_workspace_bytes(cache.pages, blocks, step),), 0xA5, dtype=torch.uint8, device="cuda")
    D.dapq_paged_sparse_attention(cache.pages, blocks, step, q, torch.from_numpy(idx).cuda(), torch.from_numpy(count).cuda(), out, work, stream=stream)
    torch.cuda.synchronize()
    return out.float().cpu().numpy().astype(np.float64)


def check_sparse(cache, lengths, new, q_bits, idx, count, block_rows, scale=SCALE, softcap=0.0, max_new=None, **kw):
    got = sparse(cache, lengths, new, q_bits, idx, count, block_rows, scale, softcap, max_new=max_new, **kw)
    out, weighted, size = BO.sparse_attention(cache.pool, cache.table, lengths, starts(new), max(new) if max_new is None else max_new,
                                              O.bf16_bits_to_f64(q_bits), idx, count, block_rows, float(np.float32(scale)), softcap)
    bound = attention_bound(out, weighted, size, 1)
    error = np.abs(got - out)
    tokens = [starts(new)[b] + t for b, n in enumerate(new) for t in range(n if max_new is None else min(n, max_new))]
    assert np.isfinite(got[:, tokens]).all() and (error <= bound)[:, tokens].all(), np.nanmax((error / bound)[:, tokens])
    return got


def random_choice(rng, layers, heads, lengths, new, block_rows, n_select, junk=True):
    """Blocks anywhere in what a token sees, its last one among them; entries past the count hold anything."""
    idx = rng.integers(-2 ** 31, 2 ** 31, (layers, sum(new), heads, n_select)).astype(np.int32) if junk else np.zeros((layers, sum(new), heads, n_select), np.int32)
    count = np.zeros((layers, sum(new), heads), np.int32)
    for b, n in enumerate(new):
        for t in range(n):
            blocks = -(-(lengths[b] + t + 1) // block_rows)
            for layer, head in np.ndindex(layers, heads):
                k = min(n_select, blocks)
                at = (layer, starts(new)[b] + t, head)
                idx[at][:k] = np.sort(np.append(rng.permutation(blocks - 1)[:k - 1], blocks - 1))
                count[at] = k
    return idx, count


SPARSE = [  # layers, kv heads, group, page_rows, block_rows, lengths, new, n_select
    (1, 1, 1, 16, 16, [0], [1], 1),
    (1, 8, 4, 64, 16, [982], [1], 8),
    (2, 3, 5, 32, 16, [170, 0, 9, 31], [1] * 4, 5),
    (1, 2, 8, 64, 32, [500, 64], [1, 1], 3),
    (1, 2, 16, 128, 64, [600], [2], 4),
    (1, 1, 17, 16, 16, [140], [3], 40),
    (1, 1, 40, 32, 32, [190], [2], 3),
    (1, 2, 70, 16, 16, [90, 30], [1, 2], 4),
    (1, 2, 4, 16, 16, [33, 0, 250], [4, 4, 4], 9),
    (2, 1, 3, 16, 16, [0, 5, 40], [37, 0, 20], 2),
    (1, 2, 2, 16, 16, [b for b in range(70)], [b % 3 for b in range(70)], 4),
    (1, 1, 4, 1024, 512, [3000], [1], 3),
    (1, 2, 4, 64, 16, [4000], [1], 200),
    (1, 8, 4, 16, 16, [70] * 40, [1] * 40, 3),
]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("case,softcap", [(i, 0.0) for i in range(len(SPARSE))] + [(i, c) for i in (1, 3, 4, 5, 7, 12) for c in (20.0, 100.0)])
def test_sparse_attention(fmt, case, softcap):
    layers, heads, group, page_rows, block_rows, lengths, new, n_select = SPARSE[case]
    rng = np.random.default_rng(700 + case)
    rows = [h + n for h, n in zip(lengths, new)]
    cache = Cache(rng, fmt, layers, heads, page_rows, rows).fill(rng, rows, gain=2.0).to_device()
    idx, count = random_choice(rng, layers, heads, lengths, new, block_rows, n_select)
    q = normal_bits(rng, layers, sum(new), heads * group, 128)
    check_sparse(cache, lengths, new, q, idx, count, block_rows, softcap=softcap, ragged=len(set(new)) > 1, pads=(8, 16) if case % 2 else (0, 0))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("group", [4, 12, 20])
def test_all_blocks_are_all_rows(fmt, group):
    """Every block chosen: what dapq_paged_attention gives, to the bounds of both."""
    rng = np.random.default_rng(71)
    lengths, new = [700, 40, 0], [2, 1, 1]
    rows = [h + n for h, n in zip(lengths, new)]
    cache = Cache(rng, fmt, 1, 2, 32, rows).fill(rng, rows).to_device()
    q = normal_bits(rng, 1, 4, 2 * group, 128)
    idx, count = random_choice(rng, 1, 2, lengths, new, 32, 30)
    got, dense = check_sparse(cache, lengths, new, q, idx, count, 32), attend(cache, lengths, new, q)
    out, weighted, size = PO.attention(cache.pool, cache.table, lengths, starts(new), O.bf16_bits_to_f64(q), SCALE)
    assert (np.abs(got - dense) <= 2 * attention_bound(out, weighted, size, 100)).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("wide", [False, True])
def test_entries_of_all_kinds(fmt, wide):
    """Blocks out of order, twice, past the token, past the table, negative; counts past n_select, of zero and below; pages that there are not."""
    rng = np.random.default_rng(72)
    lengths, new = [100, 200, 64, 300], [1, 2, 1, 1]
    rows = [h + n for h, n in zip(lengths, new)]
    cache = Cache(rng, fmt, 1, 2, 16, rows, extra_entries=3)
    cache.table[0, 1], cache.table[1, 3], cache.table[2, :], cache.table[3, 4] = -1, cache.n_pages, -5, 1 << 30
    cache.fill(rng, rows).to_device()
    n = 64 if wide else 9
    idx = np.full((1, 5, 2, n), 2 ** 31 - 1, np.int32)
    count = np.full((1, 5, 2), n, np.int32)
    idx[0, 0, 0, :9] = [6, 0, 0, 2, -1, 1, 7, 100, 5]
    idx[0, 0, 1, :9] = [3, 3, 3, 3, 3, 3, 3, 3, 3]
    idx[0, 1, 0, :9] = [12, 11, 10, 9, 8, 7, 6, 5, -2 ** 31]
    idx[0, 1, 1, :9] = [3, 1 << 26, 1 << 27, (1 << 28) - 1, 4, 20, 21, 12, 13]
    idx[0, 2, :, :9] = [0, 1, 2, 3, 4, 5, 6, 7, 12]
    count[0, 2] = [4, 1 << 30]
    idx[0, 3, :, :9] = np.arange(9)
    idx[0, 4, 0, :9], idx[0, 4, 1, :9] = 18, [4, 4, 19, -1, -1, 21, 22, -7, 30]
    count[0, 4, 0] = -3
    got = check_sparse(cache, lengths, new, normal_bits(rng, 1, 5, 8, 128), idx, count, 16)
    assert not got[0, 3].any() and not got[0, 4].any()


def test_a_block_named_twice_counts_twice():
    rng = np.random.default_rng(73)
    cache = Cache(rng, "bf16", 1, 1, 16, [48], extra_entries=0).fill(rng, [48]).to_device()
    q = np.zeros((1, 1, 1, 128), np.uint16)                                           # (all weights the same)
    idx, count = np.array([[[[0, 1, 1]]]], np.int32), np.full((1, 1, 1), 3, np.int32)
    got = sparse(cache, [47], [1], q, idx, count, 16)
    v = O.bf16_bits_to_f64(cache.pool["v"][0, cache.table[0], 0])
    want = (v[0].mean(0) + 2 * v[1].mean(0)) / 3
    assert (np.abs(got[0, 0, 0] - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -14 * np.abs(v).max()).all()


@pytest.mark.parametrize("n_select", [37, 38, 39, 77, 300, 4096])
def test_more_entries_than_the_table_has_blocks(n_select):
    """Blocks of a table of 38, in any order and more than once, or few of them where there is room for many."""
    rng = np.random.default_rng(74 + n_select)
    cache = Cache(rng, "bf16", 1, 2, 16, [600, 20], extra_entries=0).fill(rng, [600, 20]).to_device()
    idx = rng.integers(0, 38, (1, 2, 2, n_select)).astype(np.int32)
    count = np.array([[[n_select, min(n_select, 38)], [n_select, 5]]], np.int32)
    check_sparse(cache, [599, 19], [1, 1], normal_bits(rng, 1, 2, 8, 128), idx, count, 16)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("group,n_select", [(1, 6), (4, 6), (12, 6), (24, 6), (4, 70)])
def test_what_is_not_finite(fmt, group, n_select):
    """A NaN or an infinity in a row reaches the tokens whose blocks have the row, if they see it, and no others."""
    rng = np.random.default_rng(74)
    cache = Cache(rng, fmt, 1, 1, 32, [200]).fill(rng, [200])
    for name, row, value in (("v", 37, np.inf), ("v", 70, np.nan), ("k", 90, np.nan), ("v", 105, -np.inf), ("v", 170, np.nan)):
        page, slot = PO.place(cache.table, cache.n_pages, 32, 0, row)
        if fmt == "bf16":
            cache.pool[name][0, page, 0, slot, 3] = O.f64_to_bf16_bits(np.array([value]))[0]
        else:
            cache.pool[name + "_scales"][0, page, 0, slot, 0] = 255
    cache.to_device()
    new = 8
    idx, count = np.full((1, new, 1, n_select), -1, np.int32), np.full((1, new, 1), n_select, np.int32)
    idx[0, :, 0, :6] = [[0, 1, 3, -1, -1, -1], [0, 2, 3, -1, -1, -1], [0, 4, -1, -1, -1, -1], [1, 5, -1, -1, -1, -1], [0, 6, -1, -1, -1, -1], [0, 10, -1, -1, -1, -1],
                        [2, 4, 5, 6, 10, 11], [0, 1, 3, 7, 8, 9]]
    q = normal_bits(rng, 1, new, group, 128)
    got = sparse(cache, [102], [new], q, idx, count, 16)             # token 2 sees row 104, token 3 row 105
    with np.errstate(invalid="ignore"):
        want, weighted, size = BO.sparse_attention(cache.pool, cache.table, [102], [0, new], new, O.bf16_bits_to_f64(q), idx, count, 16, SCALE)
    finite = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and (got[np.isinf(want)] == want[np.isinf(want)]).all()
    with np.errstate(invalid="ignore"):
        assert (np.abs(got - want) <= attention_bound(want, weighted, size, 1))[finite].all()
    assert finite[0, [0, 5, 7]].all() and not finite[0, [1, 2, 3, 4, 6]].all(axis=(1, 2)).any()


@pytest.mark.parametrize("fmt", ["fp4", "e4m3"])
@pytest.mark.parametrize("group,n_select", [(1, 6), (4, 40), (12, 6), (24, 40)])
def test_values_past_the_largest_scales(fmt, group, n_select):
    """Groups of codes with infinite values among them: what the tokens see whose blocks have the row.  With queries of 0 every weight is 1, and a channel has one
    such value."""
    module = SCALES if fmt == "fp4" else E4M3
    rng = np.random.default_rng(76 + group)
    cache = Cache(rng, fmt, 1, 2, 32, [200]).fill(rng, [200])
    for g, (row, byte) in enumerate(((5, 253), (45, 254), (102, 254), (104, 253))):
        module.plant(rng, cache, "v", 1, row, g, byte, range(8) if fmt == "fp4" else range(0x70, 0x7f))
    cache.to_device()
    idx, count = np.full((1, 4, 2, n_select), -1, np.int32), np.full((1, 4, 2), n_select, np.int32)
    idx[0, :, :, :6] = np.array([[0, 2, 6, 1, 3, 4], [6, 1, 3, 4, 5, 12], [0, 1, 2, 3, 4, 5], [6, 5, 4, 3, 2, 1]])[:, None]
    q = np.zeros((1, 4, 2 * group, 128), np.uint16)
    got = sparse(cache, [101], [4], q, idx, count, 16)              # token 0 sees row 101
    with np.errstate(invalid="ignore", over="ignore"):
        want, weighted, size = BO.sparse_attention(module.as_bf16(cache), cache.table, [101], [0, 4], 4, O.bf16_bits_to_f64(q), idx, count, 16, SCALE)
        finite = np.isfinite(want)
        assert np.array_equal(np.isnan(got), np.isnan(want)) and (got[np.isinf(want)] == want[np.isinf(want)]).all()
        assert (np.abs(got - want) <= attention_bound(want, weighted, size, 1))[finite].all()
    inf = np.isinf(want[0, :, group:]).reshape(4, group, 4, 32).any((1, 3))
    assert inf.tolist() == [[True, True, False, False], [False, False, True, False], [True, True, False, False], [False, True, True, True]]


def test_extreme_scores():
    """One key far above all others, and keys of -inf."""
    rng = np.random.default_rng(75)
    cache = Cache(rng, "bf16", 1, 1, 16, [200]).fill(rng, [200], gain=4.0)
    q = normal_bits(rng, 1, 1, 4, 128)
    q[..., 0] = O.f64_to_bf16_bits(np.array([0.5]))
    idx, count = np.array([[[[1, 4, 7, 10, 12]]]], np.int32), np.full((1, 1, 1), 5, np.int32)
    page, slot = PO.place(cache.table, cache.n_pages, 16, 0, 170)
    cache.pool["k"][0, page, 0, slot] = O.f64_to_bf16_bits(O.bf16_bits_to_f64(q[0, 0, 0]) * 3)
    page, slot = PO.place(cache.table, cache.n_pages, 16, 0, 65)
    cache.pool["k"][0, page, :, slot] = O.f64_to_bf16_bits(np.full(128, 0.0))
    cache.pool["k"][0, page, :, slot, 0] = O.f64_to_bf16_bits(np.array([-np.inf]))
    cache.to_device()
    for softcap in (0.0, 5.0, 500.0):
        check_sparse(cache, [199], [1], q, idx, count, 16, scale=1.0, softcap=softcap)


def test_attention_of_tokens_past_max_new():
    rng = np.random.default_rng(76)
    cache = Cache(rng, "bf16", 2, 1, 16, [60, 90]).fill(rng, [60, 90]).to_device()
    idx, count = random_choice(rng, 2, 1, [40, 50], [2, 40], 16, 3)
    got = check_sparse(cache, [40, 50], [2, 40], normal_bits(rng, 2, 42, 2, 128), idx, count, 16, max_new=7)
    assert np.isnan(got[:, 9:]).all()                                # (what the buffer held)


@pytest.mark.parametrize("fmt", FORMATS)
def test_pools_of_more_than_four_gigabytes(fmt):
    """Blocks at the far end of pools whose rows, and of bounds whose bytes, pass 32 bits."""
    rng = np.random.default_rng(77)
    heads, page_rows, row = 8, 256, {"bf16": 256, "fp4": 64, "e4m3": 128}[fmt]
    n_pages = (5 << 30) // (heads * page_rows * row)
    if fmt == "fp4":
        n_pages *= 5                                                 # 26 GB of bounds (16 bytes a row)
    rows = 700
    small = Cache(rng, fmt, 1, heads, page_rows, [rows], spare=0, extra_entries=0).fill(rng, [rows])
    far = {n: torch.zeros((1, n_pages) + a.shape[2:], dtype=torch.uint8 if a.dtype == np.uint8 else torch.int16, device="cuda") for n, a in small.pool.items()}
    for n, a in small.pool.items():
        far[n][:, -small.n_pages:] = torch.from_numpy(a.view(np.int16 if a.dtype == np.uint16 else a.dtype)).cuda()
    table = dev_int((small.table[0] + n_pages - small.n_pages).tolist())
    small.pages = D.make_pages(n_layers=1, batch=1, n_kv_heads=heads, page_rows=page_rows, n_pages=n_pages, max_pages=small.max_pages, format=fmt,
                               k=far["k"], v=far["v"], k_scales=far.get("k_scales"), v_scales=far.get("v_scales"), table=table)
    b = Bounds(small, 16)
    b.dev = torch.zeros((1, n_pages, heads, 16, 2, 128), dtype=torch.int8, device="cuda")
    b.dev_scales = torch.zeros((1, n_pages, heads, 16), dtype=torch.uint8, device="cuda")
    assert fmt != "fp4" or b.dev.numel() > 1 << 32
    D.dapq_paged_bounds(small.pages, b.blocks(), None, dev_int([rows]), rows)
    b.bounds, b.scales = BO.bounds(small.pool, small.table, 16, None, [rows], rows, b.bounds * 0, b.scales * 0)
    assert np.array_equal(b.dev[:, -small.n_pages:].cpu().numpy(), b.bounds) and np.array_equal(b.dev_scales[:, -small.n_pages:].cpu().numpy(), b.scales)
    assert not b.dev_scales[:, :-small.n_pages].any()
    q = normal_bits(rng, 1, 2, heads * 4, 128)
    idx, count = check_choice(small, b, [rows - 2], [2], q, 9)
    check_sparse(small, [rows - 2], [2], q, idx, count, 16)


# --- together ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", FORMATS)
def test_evict_then_read_chosen_blocks(fmt):
    """A prompt is evicted into pages and its blocks get their bounds; steps of decoding append, note the bounds of completed blocks, choose and attend, each
    against its definition on the pools that the definitions of the steps before have left."""
    rng = np.random.default_rng(22)
    layers, heads, group, length, budget, page_rows, block_rows = 2, 2, 4, 400, 150, 32, 16
    k, v = normal_bits(rng, layers, length, heads, 128), normal_bits(rng, layers, length, heads, 128)
    prob = Problem(normal_bits(rng, layers, 1, heads * group, 16, 128), k, v, heads, None, "thd", SCALE)
    idx, count, _ = prob.pool_topk(prob.score(), 7, budget)
    cache = Cache(rng, fmt, layers, heads, page_rows, [budget + 60]).to_device()
    b = Bounds(cache, block_rows).to_device()
    lengths = dev_int([budget])
    D.dapq_paged_gather(prob.shape, cache.pages, prob.k, prob.v, idx, count, budget)
    D.dapq_paged_bounds(cache.pages, b.blocks(), None, lengths, budget)
    pool = PO.gather(cache.pool, cache.table, k, v, [0, length], idx.cpu().numpy(), count.cpu().numpy())
    ul, scales = BO.bounds(pool, cache.table, block_rows, None, [budget], budget, b.bounds, b.scales)
    rows, position = budget, length
    for new in (1, 3, 1, 20, 1, 1):
        kn, vn = normal_bits(rng, layers, new, heads, 128), normal_bits(rng, layers, new, heads, 128)
        (dk, ks), (dv, vs) = strided(kn), strided(vn)
        q = normal_bits(rng, layers, new, heads * group, 128)
        dq, qs = strided(q)
        step = D.make_step(n_q_heads=heads * group, total_new=new, max_new=new, lengths=lengths, k_strides=ks, v_strides=vs, q_strides=qs, scale=SCALE)
        blocks = b.blocks(n_select=5, n_first=1, n_last=2)
        positions = np.arange(position, position + new)
        chosen = torch.full((layers, new, heads, 5), -7, dtype=torch.int32, device="cuda")
        kept = torch.zeros((layers, new, heads), dtype=torch.int32, device="cuda")
        out = torch.empty((layers, new, heads * group, 128), dtype=torch.bfloat16, device="cuda")
        works = [torch.empty(f(cache.pages, blocks, step), dtype=torch.uint8, device="cuda") for f in (D.paged_select_workspace_bytes, D.paged_sparse_attention_workspace_bytes)]
        after = lengths + new
        D.dapq_paged_append(cache.pages, step, dk, dv, dev_int(positions), THETA)
        D.dapq_paged_bounds(cache.pages, blocks, lengths, after, new)
        D.dapq_paged_select(cache.pages, blocks, step, dq, chosen, kept, works[0])
        D.dapq_paged_sparse_attention(cache.pages, blocks, step, dq, chosen, kept, out, works[1])
        pool = PO.append(pool, cache.table, [rows], [0, new], new, kn, vn, positions, THETA)
        ul, scales = BO.bounds(pool, cache.table, block_rows, [rows], [rows + new], new, ul, scales)
        want = BO.select(cache.table, cache.n_pages, page_rows, ul, scales, block_rows, 5, 1, 2, [rows], [0, new], new, O.bf16_bits_to_f64(q))
        idx_h, count_h = chosen.cpu().numpy(), kept.cpu().numpy()
        for at, blocks_of in want.items():
            assert idx_h[at][:count_h[at]].tolist() == blocks_of
        exact, weighted, size = BO.sparse_attention(pool, cache.table, [rows], [0, new], new, O.bf16_bits_to_f64(q), idx_h, count_h, block_rows, SCALE)
        assert (np.abs(out.double().cpu().numpy() - exact) <= attention_bound(exact, weighted, size, 1)).all()
        lengths = after
        rows, position = rows + new, position + new
    same_pool(cache.from_device(), pool)
    assert np.array_equal(b.dev.cpu().numpy(), ul) and np.array_equal(b.dev_scales.cpu().numpy(), scales)


def test_the_block_of_a_needle_is_chosen():
    """A key along a query, in one of 300 blocks: its block is among the few that are read, and carries the output."""
    rng = np.random.default_rng(23)
    n = 4800
    cache = Cache(rng, "bf16", 1, 1, 64, [n]).fill(rng, [n])
    q = normal_bits(rng, 1, 1, 4, 128)
    page, slot = PO.place(cache.table, cache.n_pages, 64, 0, 2345)
    cache.pool["k"][0, page, 0, slot] = O.f64_to_bf16_bits(3 * O.bf16_bits_to_f64(q[0, 0, 2]))
    cache.to_device()
    b = Bounds(cache, 16).to_device()
    D.dapq_paged_bounds(cache.pages, b.blocks(), None, dev_int([n]), n)
    idx, count = choose(cache, b, [n - 1], [1], q, 8)
    assert 2345 // 16 in idx[0, 0, 0].tolist()
    got = sparse(cache, [n - 1], [1], q, idx, count, 16)
    v = O.bf16_bits_to_f64(cache.pool["v"][0, page, 0, slot])
    assert (np.abs(got[0, 0, 2] - v) <= 2.0 ** -8 * np.abs(v) + 1e-3).all()    # (its logit is some 30 above the others')


def test_steps_replayed_from_a_graph():
    """One step (append, bounds, selection, attention, then the lengths go on) recorded once and replayed; every replay is the eager step, bit for bit."""
    rng = np.random.default_rng(32)
    heads, group, page_rows, first, steps = 2, 4, 32, [140, 3, 900], 24

    def fresh():
        cache = Cache(np.random.default_rng(1), "e4m3", 1, heads, page_rows, [n + steps + 1 for n in first]).fill(np.random.default_rng(2), first).to_device()
        b = Bounds(cache, 16).to_device()
        lengths = dev_int(first)
        D.dapq_paged_bounds(cache.pages, b.blocks(), None, lengths, max(first))
        return cache, b, lengths, lengths + 1, dev_int([1000 + n for n in first])

    kn, vn = (torch.zeros((1, 3, heads, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q, out = (torch.zeros((1, 3, heads * group, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    idx, count = torch.zeros((1, 3, heads, 6), dtype=torch.int32, device="cuda"), torch.zeros((1, 3, heads), dtype=torch.int32, device="cuda")
    data = [[dev_bits(normal_bits(rng, *t.shape)) for t in (kn, vn, q)] for _ in range(steps)]

    def make(cache, b, lengths, after):
        step = D.make_step(n_q_heads=heads * group, total_new=3, max_new=1, lengths=lengths, k_strides=(0, heads * 128, 128),
                           v_strides=(0, heads * 128, 128), q_strides=(0, heads * group * 128, 128), scale=SCALE)
        blocks = b.blocks(n_select=6, n_first=1, n_last=1)
        works = [torch.full((f(cache.pages, blocks, step),), 0xA5, dtype=torch.uint8, device="cuda") for f in (D.paged_select_workspace_bytes, D.paged_sparse_attention_workspace_bytes)]

        def go(positions):
            D.dapq_paged_append(cache.pages, step, kn, vn, positions, THETA)
            D.dapq_paged_bounds(cache.pages, blocks, lengths, after, 1)
            D.dapq_paged_select(cache.pages, blocks, step, q, idx, count, works[0])
            D.dapq_paged_sparse_attention(cache.pages, blocks, step, q, idx, count, out, works[1])
            for t in (lengths, after, positions):
                t.add_(1)
        return go, works

    def load(i):
        for t, src in zip((kn, vn, q), data[i]):
            t.copy_(src)

    cache, b, lengths, after, positions = fresh()
    go, _ = make(cache, b, lengths, after)
    want = []
    for i in range(steps):
        load(i)
        go(positions)
        want.append((out.clone(), idx.clone(), count.clone()))
    eager = cache.from_device(), b.dev.clone(), b.dev_scales.clone()
    cache, b, lengths, after, positions = fresh()
    go, works = make(cache, b, lengths, after)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    load(0)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        go(positions)
    lengths.copy_(dev_int(first))
    after.copy_(dev_int([n + 1 for n in first]))
    positions.copy_(dev_int([1000 + n for n in first]))
    for i in range(steps):
        load(i)
        for w in works:
            w.fill_(0x5A)
        out.fill_(7.0)
        idx.copy_(want[i - 1][1] if i else torch.zeros_like(idx))
        graph.replay()
        if i % 3 == 0:
            torch.cuda.synchronize()
        assert torch.equal(out, want[i][0]) and torch.equal(idx, want[i][1]) and torch.equal(count, want[i][2]), i
    same_pool(cache.from_device(), eager[0])
    assert torch.equal(b.dev, eager[1]) and torch.equal(b.dev_scales, eager[2])


def test_two_steps_at_once():
    """On two streams, with a workspace each, over pages and bounds that two sequences share; the same bits every time."""
    rng = np.random.default_rng(43)
    cache = Cache(rng, "bf16", 1, 2, 16, [900, 900]).fill(rng, [900, 900])
    cache.table[1] = cache.table[0]
    cache.to_device()
    b = Bounds(cache, 16).to_device()
    D.dapq_paged_bounds(cache.pages, b.blocks(), None, dev_int([900, 900]), 900)
    calls, want = [], []
    for _ in range(2):
        q = normal_bits(rng, 1, 2, 8, 128)
        idx, count = choose(cache, b, [898, 400], [1, 1], q, 7)
        want.append((idx, sparse(cache, [898, 400], [1, 1], q, idx, count, 16)))
        dq, strides = strided(q)
        step = make_step([898, 400], [1, 1], False, n_q_heads=8, q_strides=strides)
        blocks = b.blocks(n_select=7, n_first=1, n_last=1)
        works = [torch.empty(f(cache.pages, blocks, step), dtype=torch.uint8, device="cuda") for f in (D.paged_select_workspace_bytes, D.paged_sparse_attention_workspace_bytes)]
        calls.append((torch.cuda.Stream(), dq, step, blocks, torch.zeros((1, 2, 2, 7), dtype=torch.int32, device="cuda"),
                      torch.zeros((1, 2, 2), dtype=torch.int32, device="cuda"), torch.zeros((1, 2, 8, 128), dtype=torch.bfloat16, device="cuda"), works))
    torch.cuda.synchronize()
    for _ in range(20):
        for stream, dq, step, blocks, idx, count, out, works in calls:
            D.dapq_paged_select(cache.pages, blocks, step, dq, idx, count, works[0], stream=stream)
            D.dapq_paged_sparse_attention(cache.pages, blocks, step, dq, idx, count, out, works[1], stream=stream)
    torch.cuda.synchronize()
    for call, (idx, out) in zip(calls, want):
        assert np.array_equal(call[4].cpu().numpy(), idx) and np.array_equal(call[6].double().cpu().numpy(), out)
