"""Calls of the cache in pages that a program may make and the other tests do not: rows of a head one after the other, dense batches, more sequences
than a launch's axis, turns replayed from a graph."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2603_11564_amd as D  # noqa: E402
from oracle import dapq_oracle as O  # noqa: E402
from oracle import paged_oracle as PO  # noqa: E402
from paged_harness import JUNK, SCALE, THETA, Cache, attend, attention_bound, dev_bits, dev_int, normal_bits, same_pool, starts  # noqa: E402

pytestmark = pytest.mark.gpu
FORMATS = ("bf16", "fp4")


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("new", [[1, 1], [5, 2], [30, 0]])
def test_rows_of_a_head_one_after_the_other(fmt, new):
    """k_new, v_new and q as [layer][head][token][d]."""
    rng = np.random.default_rng(sum(new))
    layers, heads, group, lengths, total = 2, 3, 4, [40, 17], sum(new)
    k, v = normal_bits(rng, layers, total, heads, 128), normal_bits(rng, layers, total, heads, 128)
    q = normal_bits(rng, layers, total, heads * group, 128)
    cache = Cache(rng, fmt, layers, heads, 16, [n + m for n, m in zip(lengths, new)]).fill(rng, lengths).to_device()
    kv = (heads * total * 128, 128, total * 128)
    step = D.make_step(n_q_heads=heads * group, total_new=total, max_new=max(new), cu_new=dev_int(starts(new)), lengths=dev_int(lengths), k_strides=kv,
                       v_strides=kv, q_strides=(heads * group * total * 128, 128, total * 128), scale=SCALE)
    dk, dv, dq = (dev_bits(x.transpose(0, 2, 1, 3)) for x in (k, v, q))
    positions = rng.integers(0, 1 << 17, total).astype(np.int32)
    out = dev_bits(np.full(q.shape, JUNK, np.uint16))
    work = torch.empty(D.paged_attention_workspace_bytes(cache.pages, step), dtype=torch.uint8, device="cuda")
    D.dapq_paged_append(cache.pages, step, dk, dv, dev_int(positions), THETA)
    D.dapq_paged_attention(cache.pages, step, dq, out, work)
    expect = PO.append(cache.pool, cache.table, lengths, starts(new), max(new), k, v, positions, THETA)
    same_pool(cache.from_device(), expect)
    want, weighted, size = PO.attention(expect, cache.table, lengths, starts(new), O.bf16_bits_to_f64(q), SCALE)
    assert (np.abs(out.double().cpu().numpy() - want) <= attention_bound(want, weighted, size, group * max(new))).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("packed", [True, False])
def test_gather_of_a_dense_batch(fmt, packed):
    """No cu_seqlens: sequences of one length, one behind the other, or each a constant apart from where that would be."""
    rng = np.random.default_rng(11)
    layers, batch, heads, length, budget = 2, 3, 2, 50, 20
    k, v = normal_bits(rng, layers, batch * length, heads, 128), normal_bits(rng, layers, batch * length, heads, 128)
    gap = 0 if packed else 64
    seq = length * heads * 128
    def device(x):
        buf = np.full((layers, batch, seq + gap), JUNK, np.uint16)
        buf[:, :, :seq] = x.reshape(layers, batch, seq)
        return dev_bits(buf)
    strides = (batch * (seq + gap), gap, 128, heads * 128)
    shape = D.make_shape(n_layers=layers, batch=batch, n_q_heads=heads, n_kv_heads=heads, n_pseudo=1, total_tokens=batch * length, k_strides=strides,
                         v_strides=strides, scale=SCALE)
    idx = np.sort(np.stack([rng.permutation(length)[:budget] for _ in range(layers * batch * heads)]), -1).astype(np.int32).reshape(layers, batch, heads, budget)
    count = np.full((layers, batch, heads), budget, np.int32)
    cache = Cache(rng, fmt, layers, heads, 16, [budget] * batch).to_device()
    D.dapq_paged_gather(shape, cache.pages, device(k), device(v), torch.from_numpy(idx).cuda(), torch.from_numpy(count).cuda(), budget)
    same_pool(cache.from_device(), PO.gather(cache.pool, cache.table, k, v, np.arange(batch + 1) * length, idx, count))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("most", [1, 2, 40])
def test_more_sequences_than_an_axis_holds(fmt, most):
    """70000 sequences of up to 16 rows, most of them with one new token: each as in a call of a few sequences."""
    rng = np.random.default_rng(70 + most)
    batch, some = 70000, [0, 1, 63, 64, 4095, 4096, 65535, 65536, 69998, 69999]
    new = np.ones(batch, np.int64)
    new[rng.permutation(batch)[:5000]] = 0
    new[some[3::2]] = most
    lengths = np.minimum(rng.integers(0, 16, batch), 16 - np.minimum(new, 16))
    total = int(new.sum())
    g = torch.Generator(device="cuda").manual_seed(most)
    row = 128 if fmt == "bf16" else 64
    pool = {}
    for name in ("k", "v"):
        x = torch.empty((1, batch, 1, 16, 128), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        pool[name] = x.view(torch.int16) if fmt == "bf16" else torch.randint(0, 256, (1, batch, 1, 16, row), generator=g, device="cuda", dtype=torch.uint8)
        if fmt == "fp4":
            pool[name + "_scales"] = torch.randint(123, 129, (1, batch, 1, 16, 4), generator=g, device="cuda", dtype=torch.uint8)
    table = torch.randperm(batch, generator=g, device="cuda", dtype=torch.int32)[:, None].contiguous()
    pages = D.make_pages(n_layers=1, batch=batch, n_kv_heads=1, page_rows=16, n_pages=batch, max_pages=1, format=fmt, table=table, **pool)
    q = torch.empty((1, total, 4, 128), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    kn, vn = (torch.empty((1, total, 1, 128), dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(2))
    cu = starts(new)
    step = D.make_step(n_q_heads=4, total_new=total, max_new=most, cu_new=dev_int(cu), lengths=dev_int(lengths), k_strides=(0, 128, 128),
                       v_strides=(0, 128, 128), q_strides=(0, 512, 128), scale=SCALE)
    out = torch.full_like(q, float("nan"))
    work = torch.empty(D.paged_attention_workspace_bytes(pages, step), dtype=torch.uint8, device="cuda")
    before = {n: t.clone() for n, t in pool.items()}
    D.dapq_paged_append(pages, step, kn, vn, None, THETA)
    D.dapq_paged_attention(pages, step, q, out, work)
    assert not torch.isnan(out).any()
    picked = [int(b) for b in some]
    at = table[picked, 0].long().cpu()
    host = {n: t[:, at.to(t.device)].cpu().numpy().view(np.uint16 if fmt == "bf16" else np.uint8) for n, t in before.items()}
    small = np.arange(len(picked), dtype=np.int32)[:, None]
    rows = np.concatenate([np.arange(cu[b], cu[b + 1]) for b in picked])
    bits = [t[:, rows].contiguous().view(torch.int16).cpu().numpy().view(np.uint16) for t in (kn, vn, q)]
    expect = PO.append(host, small, lengths[picked], starts(new[picked]), most, bits[0], bits[1], None, THETA)
    for n, a in expect.items():
        assert np.array_equal(pool[n][:, at.to(table.device)].cpu().numpy().view(a.dtype), a)
    # (what changed is as many rows as there are tokens that have a place)
    placed = int(np.minimum(new, np.maximum(0, 16 - lengths)).sum())
    changed = ((pool["v"] != before["v"]).any(-1)).sum()
    assert placed * 0.99 <= int(changed) <= placed
    want, weighted, size = PO.attention(expect, small, lengths[picked], starts(new[picked]), O.bf16_bits_to_f64(bits[2]), SCALE)
    got = out[:, rows].double().cpu().numpy()
    assert (np.abs(got - want) <= attention_bound(want, weighted, size, 4 * most)).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("extra", [1, 500])
def test_turns_replayed_from_a_graph(fmt, extra):
    """An append and an attention of up to 40 tokens a sequence, recorded once; lengths, tokens, positions and the table change between replays, through a table
    in which rows are shared out and one in which they are not."""
    rng = np.random.default_rng(51)
    heads, group, batch, total = 2, 4, 3, 90
    cache = Cache(rng, fmt, 1, heads, 16, [400] * batch, extra_entries=extra).fill(rng, [400] * batch).to_device()
    lengths, cu, positions = dev_int([0] * batch), dev_int([0] * batch + [total]), dev_int([0] * total)
    kn, vn = (torch.zeros((1, total, heads, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros((1, total, heads * group, 128), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(q)
    kv = (0, heads * 128, 128)
    step = D.make_step(n_q_heads=heads * group, total_new=total, max_new=40, cu_new=cu, lengths=lengths, k_strides=kv, v_strides=kv,
                       q_strides=(0, heads * group * 128, 128), scale=SCALE)
    work = torch.empty(D.paged_attention_workspace_bytes(cache.pages, step), dtype=torch.uint8, device="cuda")

    def go():
        D.dapq_paged_append(cache.pages, step, kn, vn, positions, THETA)
        D.dapq_paged_attention(cache.pages, step, q, out, work)

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        go()
    expect = cache.pool
    for held, new in (([0, 7, 350], [30, 40, 20]), ([200, 0, 100], [40, 10, 40]), ([360, 360, 5], [40, 33, 17]), ([15, 16, 17], [30, 30, 30])):
        bits = [normal_bits(rng, *t.shape) for t in (kn, vn, q)]
        for t, b in zip((kn, vn, q), bits):
            t.copy_(dev_bits(b))
        at = rng.integers(0, 1 << 17, total).astype(np.int32)
        order = rng.permutation(cache.batch)
        cache.table = cache.table[order]
        for t, x in ((lengths, held), (cu, starts(new)), (positions, at)):
            t.copy_(dev_int(x))
        cache.dev_table.copy_(torch.from_numpy(cache.table).cuda())
        work.fill_(0x5A)
        out.fill_(7.0)
        graph.replay()
        got = out.clone()
        expect = PO.append(expect, cache.table, held, starts(new), 40, bits[0], bits[1], at, THETA)
        same_pool(cache.from_device(), expect)
        want, weighted, size = PO.attention(expect, cache.table, held, starts(new), O.bf16_bits_to_f64(bits[2]), SCALE)
        assert (np.abs(got.double().cpu().numpy() - want) <= attention_bound(want, weighted, size, 160)).all()
        go()                                                     # (eager, the same rows again)
        assert torch.equal(out, got)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("group,new", [(4, 1), (4, 4), (8, 4), (4, 30)])
@pytest.mark.parametrize("extra", [1, 1000])
def test_calls_repeat_themselves(fmt, group, new, extra):
    """The same call again gives the same bits, whatever the workspace held and the output was."""
    rng = np.random.default_rng(new)
    lengths = [900, 5, 0, 333]
    rows = [n + new for n in lengths]
    cache = Cache(rng, fmt, 1, 2, 16, rows, extra_entries=extra).fill(rng, rows, gain=2.0).to_device()
    q = normal_bits(rng, 1, 4 * new, 2 * group, 128)
    first = attend(cache, lengths, [new] * 4, q)
    for _ in range(5):
        assert np.array_equal(attend(cache, lengths, [new] * 4, q), first)
