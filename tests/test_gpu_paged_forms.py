"""The forms that the calls of the cache in pages take for large calls: runs of more heads in an append, loads and stores past the caches in a gather
and a read, and caps in every one of the attention's kernels."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2603_11564_amd as D  # noqa: E402
from dapq_harness import Problem  # noqa: E402
from oracle import dapq_oracle as O  # noqa: E402
from oracle import paged_oracle as PO  # noqa: E402
from paged_harness import JUNK, SCALE, THETA, Cache, dev_bits, dev_int, make_step, normal_bits, same_pool, starts, strided  # noqa: E402
from test_gpu_paged import ATTENTION, check_attention  # noqa: E402

pytestmark = pytest.mark.gpu
FORMATS = ("bf16", "fp4")


def put_rows(cache, name, bits, lengths, new):
    """bits [layers][tokens][heads][128] behind the rows that the sequences hold, on the host's pool."""
    cu = starts(new)
    page, slot = (np.concatenate([x[b] for b in range(len(new))]) for x in zip(*[
        (cache.table[b, (lengths[b] + np.arange(n)) // cache.page_rows], (lengths[b] + np.arange(n)) % cache.page_rows) for b, n in enumerate(new)]))
    assert len(page) == cu[-1] == bits.shape[1]
    for layer in range(cache.layers):
        for t in range(0, len(page), 1024):                       # (what the quantiser holds at once)
            p, s, x = page[t:t + 1024], slot[t:t + 1024], bits[layer, t:t + 1024]
            if cache.fmt == "fp4":
                cache.pool[name][layer, p, :, s], cache.pool[name + "_scales"][layer, p, :, s] = PO.fp4_quantise(O.bf16_bits_to_f64(x))
            else:
                cache.pool[name][layer, p, :, s] = x


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("layers,heads,lengths,new,pairing", [
    (1, 8, [3], [1100], 0),              # runs of 4 heads
    (2, 8, [0, 40], [700, 350], 1),      # 8
    (1, 5, [17], [1100], 1),             # 4 and 1
    (1, 5, [0, 9, 2], [2000, 0, 101], 0),  # 5, an odd number, of 8
    (1, 11, [5, 1], [1030, 20], 0),      # 8 and 3
    (1, 11, [0], [2100], 1),             # 11 of 16
    (1, 40, [2], [1100], 0),             # 32 and 8
    (1, 13, [8], [1200], None),          # 8 and 5, keys as they are
])
def test_appends_of_many_tokens(fmt, layers, heads, lengths, new, pairing):
    rng = np.random.default_rng(heads * 10 + layers)
    total = sum(new)
    k, v = normal_bits(rng, layers, total, heads, 128), normal_bits(rng, layers, total, heads, 128)
    positions = None if pairing is None else rng.integers(0, 1 << 20, total).astype(np.int32)
    cache = Cache(rng, fmt, layers, heads, 64, [h + n for h, n in zip(lengths, new)]).to_device()
    (dk, ks), (dv, vs) = strided(k, 8, 16), strided(v)
    D.dapq_paged_append(cache.pages, make_step(lengths, new, True, heads, k_strides=ks, v_strides=vs), dk, dv,
                        None if positions is None else dev_int(positions), THETA, pairing or 0)
    if positions is not None:
        k = np.stack([O.rope_apply(x, positions, THETA, "interleaved" if pairing else "half") for x in k])
    put_rows(cache, "k", k, lengths, new)
    put_rows(cache, "v", v, lengths, new)
    same_pool(cache.from_device(), cache.pool)


@pytest.mark.parametrize("heads", [65534, 65535])
def test_an_append_of_the_most_heads(heads):
    """One token: 32767 and 32768 pairs of heads of the keys and as many of the values, along one axis of a launch, which holds 65536."""
    g = torch.Generator(device="cuda").manual_seed(heads)
    new = [torch.empty((1, 1, heads, 128), dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(2)]
    pools = [torch.zeros((1, 2, heads, 16, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    pages = D.make_pages(n_layers=1, batch=1, n_kv_heads=heads, page_rows=16, n_pages=2, max_pages=1, format="bf16", k=pools[0], v=pools[1], table=dev_int([1]))
    strides = (heads * 128, heads * 128, 128)
    D.dapq_paged_append(pages, make_step([3], [1], False, heads, k_strides=strides, v_strides=strides), *new, None, THETA)
    for pool, x in zip(pools, new):
        assert torch.equal(pool[0, 1, :, 3], x[0, 0])
        pool[0, 1, :, 3] = 0
        assert not pool.any()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("layers,heads,lens,budget,page_rows,layout", [
    (2, 4, [50, 90], 900, 16, "thd"),       # a budget of 8 MB and more: stores past the caches
    (4, 8, [40, 7, 20], 3500, 32, "hnd"),   # of 192 MB and more: loads too
])
def test_gathers_of_large_budgets(fmt, layers, heads, lens, budget, page_rows, layout):
    """The form follows the budget; few of its rows are kept here."""
    rng = np.random.default_rng(budget)
    cu, keep = starts(lens), [n - n // 4 for n in lens]
    k, v = normal_bits(rng, layers, int(cu[-1]), heads, 128), normal_bits(rng, layers, int(cu[-1]), heads, 128)
    prob = Problem(normal_bits(rng, layers, len(lens), heads, 1, 128), k, v, heads, cu, layout, SCALE)
    idx = np.full((layers, len(lens), heads, budget), -7, dtype=np.int32)
    count = np.zeros((layers, len(lens), heads), dtype=np.int32)
    for layer, b, h in np.ndindex(count.shape):
        count[layer, b, h] = keep[b] - h % 2
        idx[layer, b, h, :keep[b]] = np.sort(rng.permutation(lens[b])[:keep[b]])
    cache = Cache(rng, fmt, layers, heads, page_rows, keep, extra_entries=budget // page_rows).to_device()
    D.dapq_paged_gather(prob.shape, cache.pages, prob.k, prob.v, torch.from_numpy(idx).cuda(), torch.from_numpy(count).cuda(), budget)
    same_pool(cache.from_device(), PO.gather(cache.pool, cache.table, k, v, cu, idx, count))


def test_a_gather_of_200_megabytes():
    """Every row of a full budget, against torch's indexing."""
    layers, batch, heads, length, budget, page_rows = 4, 2, 8, 4000, 3100, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.empty((layers, batch * length, heads, 128), dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(2))
    cache = Cache(np.random.default_rng(3), "bf16", layers, heads, page_rows, [budget] * batch).to_device()
    idx = torch.rand((layers, batch, heads, length), generator=g, device="cuda").topk(budget, -1).indices.to(torch.int32)
    count = torch.full((layers, batch, heads), budget, dtype=torch.int32, device="cuda")
    strides = (batch * length * heads * 128, 0, 128, heads * 128)
    shape = D.make_shape(n_layers=layers, batch=batch, n_q_heads=heads, n_kv_heads=heads, n_pseudo=1, total_tokens=batch * length,
                         cu_seqlens=dev_int([0, length, 2 * length]), k_strides=strides, v_strides=strides, scale=SCALE)
    D.dapq_paged_gather(shape, cache.pages, k, v, idx, count, budget)
    row = torch.arange(budget, device="cuda")
    layer, head = torch.arange(layers, device="cuda")[:, None, None], torch.arange(heads, device="cuda")[:, None]
    for b in range(batch):
        page = cache.dev_table[b].long()[row // page_rows]
        for name, x in (("k", k), ("v", v)):
            got = cache.dev[name][:, page, :, row % page_rows]   # [row][layer][head][d]
            want = x[layer, idx[:, b].long() + b * length, head].permute(2, 0, 1, 3)
            assert torch.equal(got, want.view(torch.int16))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("layers,heads,page_rows,lengths,max_rows", [(2, 4, 64, [600, 37, 0], 620), (1, 3, 16, [1601, 1600, 5, 33], 1601)])
def test_reads_of_many_rows(fmt, layers, heads, page_rows, lengths, max_rows):
    rng = np.random.default_rng(max_rows)
    cache = Cache(rng, fmt, layers, heads, page_rows, [max(lengths)] * len(lengths)).fill(rng, lengths)
    cache.table[0, 3] = -1
    cache.to_device()
    outs = [dev_bits(np.full((layers, len(lengths), heads, max_rows, 128), JUNK, np.uint16)) for _ in range(2)]
    D.dapq_paged_read(cache.pages, dev_int(lengths), max_rows, *outs)
    for got, ref in zip(outs, PO.read(cache.pool, cache.table, lengths, max_rows, JUNK)):
        assert np.array_equal(got.view(torch.int16).cpu().numpy().view(np.uint16), ref)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("softcap", [20.0, 300.0])
@pytest.mark.parametrize("case", range(len(ATTENTION)))
def test_capped_attention_through_a_wide_table(fmt, softcap, case):
    """Parts of an item whose references come from capped scores, in the kernels of 8, 16 and 32 columns and of turns."""
    layers, heads, group, page_rows, lengths, new = ATTENTION[case]
    rng = np.random.default_rng(700 + case)
    rows = [h + n for h, n in zip(lengths, new)]
    cache = Cache(rng, fmt, layers, heads, page_rows, rows, extra_entries=20000 // page_rows).fill(rng, rows, gain=2.0).to_device()
    check_attention(cache, lengths, new, normal_bits(rng, layers, sum(new), heads * group, 128), softcap, ragged=len(set(new)) > 1)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("softcap", [1.0, 64.0, 65.0, 300.0, 1e6])
@pytest.mark.parametrize("new", [1, 3, 6, 9, 40])
@pytest.mark.parametrize("wide", [False, True])
def test_caps_in_all_kernels(fmt, softcap, new, wide):
    """4, 12, 24, 36 and 160 query rows of a KV head; scores far above the cap, around it and far below it."""
    rng = np.random.default_rng(73 + new)
    cache = Cache(rng, fmt, 1, 1, 32, [150 + new], extra_entries=600 if wide else 1).fill(rng, [150 + new], gain=3.0).to_device()
    check_attention(cache, [150], [new], normal_bits(rng, 1, new, 4, 128), softcap, scale=0.5)
