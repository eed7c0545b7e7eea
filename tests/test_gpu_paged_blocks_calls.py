"""Chosen blocks of a cache in pages as a serving program calls them: one workspace while sequences come and go, scores that tie at several levels."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2603_11564_amd as D  # noqa: E402
from oracle import blocks_oracle as BO  # noqa: E402
from oracle import dapq_oracle as O  # noqa: E402
from paged_harness import JUNK, SCALE, Cache, attention_bound, dev_bits, make_step, normal_bits, starts, strided  # noqa: E402
from test_gpu_paged_blocks import Bounds, check_choice  # noqa: E402

pytestmark = pytest.mark.gpu


def test_one_workspace_serves_steps_of_all_sizes():
    """Workspaces of the figure for 56 sequences, through a table of 2048 blocks: the largest step chooses in one kernel and has a workgroup to an item, smaller and ragged
    ones choose in two and share items out, in the same memory.  Nothing is written behind it."""
    rng = np.random.default_rng(61)
    heads, group, n_select, most = 8, 2, 64, 56
    lengths = [int(n) for n in rng.integers(0, 300, most)]
    lengths[0], lengths[7] = 1300, 0
    cache = Cache(rng, "bf16", 1, heads, 16, [n + 4 for n in lengths], extra_entries=0)
    wide = np.full((most, 2048), -1, np.int32)
    wide[:, :cache.max_pages] = cache.table
    cache.table, cache.max_pages = wide, 2048
    for name in ("k", "v"):
        cache.pool[name][:] = normal_bits(rng, *cache.pool[name].shape)
    cache.to_device()
    b = Bounds(cache, 16).random(rng).to_device()
    blocks = b.blocks(n_select=n_select, n_first=1, n_last=2)

    def pages_of(batch):
        return D.make_pages(n_layers=1, batch=batch, n_kv_heads=heads, page_rows=16, n_pages=cache.n_pages, max_pages=2048, format="bf16", k=cache.dev["k"], v=cache.dev["v"],
                            table=cache.dev_table[:batch])

    def step_of(batch, new, ragged, q_strides):
        return make_step(lengths[:batch], new, ragged, n_q_heads=heads * group, q_strides=q_strides, max_new=1 if max(new) <= 1 else 4)

    figures = (D.paged_select_workspace_bytes, D.paged_sparse_attention_workspace_bytes)
    _, strides = strided(normal_bits(rng, 1, most, heads * group, 128))
    room = [f(pages_of(most), blocks, step_of(most, [1] * most, False, strides)) for f in figures]
    works = [torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device="cuda") for n in room]
    for batch, new, ragged in ((56, [1] * 56, False), (30, [1] * 30, False), (13, [1] * 13, True), (56, [i % 2 for i in range(56)], True), (1, [1], False), (4, [4, 0, 3, 1], True)):
        q_bits = normal_bits(rng, 1, sum(new), heads * group, 128)
        q, strides = strided(q_bits)
        pages, step = pages_of(batch), step_of(batch, new, ragged, strides)
        idx = torch.full((1, sum(new), heads, n_select), -7, dtype=torch.int32, device="cuda")
        count = torch.full((1, sum(new), heads), -7, dtype=torch.int32, device="cuda")
        out = dev_bits(np.full(q_bits.shape, JUNK, dtype=np.uint16))
        D.dapq_paged_select(pages, blocks, step, q, idx, count, works[0][:room[0]])
        D.dapq_paged_sparse_attention(pages, blocks, step, q, idx, count, out, works[1][:room[1]])
        torch.cuda.synchronize()
        idx, count = idx.cpu().numpy(), count.cpu().numpy()
        queries = O.bf16_bits_to_f64(q_bits)
        want = BO.select(cache.table[:batch], cache.n_pages, 16, b.bounds, b.scales, 16, n_select, 1, 2, lengths[:batch], starts(new), 4, queries)
        for at, chosen in want.items():
            assert idx[at][:count[at]].tolist() == chosen, (batch, at)
        exact, weighted, size = BO.sparse_attention(cache.pool, cache.table[:batch], lengths[:batch], starts(new), 4, queries, idx, count, 16, float(np.float32(SCALE)))
        assert (np.abs(out.double().cpu().numpy() - exact) <= attention_bound(exact, weighted, size, 1)).all(), batch
        for work, n in zip(works, room):
            assert bool((work[n:] == 0xA5).all())


# --- scores that tie --------------------------------------------------------------------------------------------------------
LEVELS = [(150, 1), (150, 0), (120, 1), (120, 0)]     # scale byte, what the box of bounds is wider by: two pairs of close scores, the pairs far apart


def tied_levels(rng, cache, b, q_bits, seq, blocks, shares):
    """Bounds of a sequence's blocks 0 .. blocks - 1 that give its first token's queries one of four scores, wider boxes the higher ones: shares[i] blocks of level i, the last
    of them all that are left, anywhere.  Returns the level of every block."""
    level = np.full(blocks, len(LEVELS) - 1)
    level[:sum(shares)] = np.repeat(np.arange(len(shares)), shares)
    rng.shuffle(level)
    group = q_bits.shape[2] // cache.heads
    for head in range(cache.heads):
        mid, half = rng.integers(-40, 41, 128), rng.integers(5, 31, 128)
        step = np.ones(128, np.int64)
        if group == 1:      # as close as two scores can be: one channel, of the least whole number of the query that is not 0
            u, _ = BO.whole_query(O.bf16_bits_to_f64(q_bits[0, seq, head]))
            step[:] = 0
            step[np.argmin(np.where(u == 0, 1000, np.abs(u)))] = 1
        for block in range(blocks):
            page, row = divmod(block * b.block_rows, cache.page_rows)
            at = (0, cache.table[seq, page], head, row // b.block_rows)
            scale, wider = LEVELS[level[block]]
            b.bounds[at][0], b.bounds[at][1], b.scales[at] = mid + half + wider * step, mid - half - wider * step, scale
    return level


@pytest.mark.parametrize("blocks,heads,sequences,group,new", [
    (200, 2, 1, 1, 1), (256, 2, 3, 4, 1),           # one kernel of four waves
    (400, 1, 1, 1, 1), (430, 2, 2, 8, 2),           # of eight
    (2100, 8, 33, 1, 1),                            # of eight, four times four keys to a thread
    (1000, 2, 2, 4, 3), (1000, 1, 1, 1, 1),         # chosen by a second kernel: up to 1024 blocks
    (2000, 1, 1, 4, 1), (4000, 1, 1, 1, 1),         # 2048, 4096
    (8100, 1, 1, 1, 1), (16000, 1, 1, 2, 1),        # 8192, 16384
    (17000, 1, 1, 1, 1), (33000, 1, 2, 4, 1),       # any number, read from memory for every round
])
def test_ties_at_several_levels(blocks, heads, sequences, group, new):
    """Blocks of four scores, with the last chosen one inside a level that others lie above: of it the first blocks are chosen."""
    rng = np.random.default_rng(blocks)
    lengths = [16 * blocks - 5 - new] + [int(n) for n in rng.integers(1, 300, sequences - 1)]
    cache = Cache(rng, "bf16", 1, heads, 16, [n + new for n in lengths], extra_entries=0).to_device()
    b = Bounds(cache, 16).random(rng)
    q = normal_bits(rng, 1, sequences * new, heads * group, 128)
    level = tied_levels(rng, cache, b, q, 0, blocks, (7, 20, 60))
    b.to_device()
    n_first, n_last = 2, 1
    middle = level[n_first:blocks - n_last]
    for cut in range(4):
        above, of_cut = int((middle < cut).sum()), int((middle == cut).sum())
        n_select = min(n_first + n_last + above + (of_cut + 1) // 2, 4096)
        idx, count = check_choice(cache, b, lengths, [new] * sequences, q, n_select, n_first, n_last, ragged=False)
        for head in range(heads):
            assert count[0, new - 1, head] == n_select
            chosen = np.isin(np.arange(blocks), idx[0, new - 1, head])[n_first:blocks - n_last]
            assert chosen[middle < cut].all() and not chosen[middle > cut].any() and 0 < chosen[middle == cut].sum() < of_cut
            assert np.array_equal(chosen[middle == cut], np.arange(of_cut) < chosen[middle == cut].sum())
