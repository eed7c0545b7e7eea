"""The calls of chosen blocks without a GPU: what they refuse before anything is enqueued, and their float64 definition against values worked
out by hand."""
import ctypes as C

import numpy as np
import pytest

import paper_2603_11564_amd as D
from oracle import blocks_oracle as BO
from oracle import dapq_oracle as O
from paper_2603_11564_amd import binding
from test_paged_host import A, ERR_INVALID, ERR_UNSUPPORTED, ERR_WORKSPACE, At, BAD_PAGES, attention, fp4, pages, step

N = None


def blocks(**kw):
    a = dict(block_rows=16, n_select=8, n_first=1, n_last=1, bounds=A, scales=A)
    a.update(kw)
    return D.make_blocks(**a)


def bounds(p=None, b=None, first=A, lengths=A, rows=16):
    D.dapq_paged_bounds(p or pages(), b or blocks(), first, lengths, rows, 0)


def select(p=None, b=None, s=None, q=A, idx=A, count=A, work=A):
    D.dapq_paged_select(p or pages(), b or blocks(), s or step(), q, idx, count, work, 0)


def sparse(p=None, b=None, s=None, q=A, idx=A, count=A, out=A, work=A):
    D.dapq_paged_sparse_attention(p or pages(), b or blocks(), s or step(), q, idx, count, out, work, 0)


CALLS = (bounds, select, sparse)


@pytest.mark.parametrize("bad,code,message", BAD_PAGES, ids=[str(i) for i in range(len(BAD_PAGES))])
def test_bad_pages_are_refused_by_every_call(bad, code, message):
    for call in CALLS:
        with pytest.raises(D.DapqError, match=message) as e:
            call(p=pages(**bad))
        assert e.value.code == code
    for figure in (D.paged_select_workspace_bytes, D.paged_sparse_attention_workspace_bytes):
        assert figure(pages(**bad), blocks(), step()) == 0


BAD_BLOCKS = [
    (dict(block_rows=0), ERR_UNSUPPORTED, r"block_rows \(0\)"), (dict(block_rows=8), ERR_UNSUPPORTED, r"block_rows \(8\)"),
    (dict(block_rows=24), ERR_UNSUPPORTED, r"block_rows \(24\)"), (dict(block_rows=32), ERR_UNSUPPORTED, r"page_rows \(16\)"),
    (dict(block_rows=-16), ERR_UNSUPPORTED, r"block_rows \(-16\)"), (dict(n_select=0), ERR_UNSUPPORTED, r"n_select \(0\)"),
    (dict(n_select=4097), ERR_UNSUPPORTED, r"n_select \(4097\)"), (dict(n_first=-1), ERR_INVALID, r"n_first \(-1\)"),
    (dict(n_last=0), ERR_INVALID, r"n_last \(0\)"), (dict(n_first=5, n_last=4), ERR_INVALID, "no more than n_select"),
    (dict(n_first=2 ** 31 - 1, n_last=2 ** 31 - 1), ERR_INVALID, "no more than n_select"),
]


@pytest.mark.parametrize("bad,code,message", BAD_BLOCKS, ids=[str(i) for i in range(len(BAD_BLOCKS))])
def test_bad_blocks_are_refused_by_every_call(bad, code, message):
    for call in CALLS:
        with pytest.raises(D.DapqError, match=message) as e:
            call(b=blocks(**bad))
        assert e.value.code == code
    for figure in (D.paged_select_workspace_bytes, D.paged_sparse_attention_workspace_bytes):
        assert figure(pages(), blocks(**bad), step()) == 0


REFUSED = [
    (lambda: bounds(b=blocks(bounds=N)), ERR_INVALID, "bounds and scales"), (lambda: bounds(b=blocks(scales=N)), ERR_INVALID, "bounds and scales"),
    (lambda: select(b=blocks(bounds=N)), ERR_INVALID, "bounds and scales"), (lambda: select(b=blocks(bounds=At(8))), ERR_UNSUPPORTED, "16-byte"),
    (lambda: bounds(b=blocks(bounds=At(4))), ERR_UNSUPPORTED, "16-byte"), (lambda: bounds(lengths=N), ERR_INVALID, "lengths"),
    (lambda: bounds(rows=-1), ERR_INVALID, r"max_rows \(-1\)"), (lambda: bounds(p=pages(batch=70000)), ERR_UNSUPPORTED, "65535"),
    (lambda: bounds(p=pages(max_pages=(1 << 26) - 1), rows=2 ** 31 - 1), ERR_UNSUPPORTED, "too large"),
    (lambda: select(q=N), ERR_INVALID, "q, idx and count"), (lambda: select(idx=N), ERR_INVALID, "q, idx and count"),
    (lambda: select(count=N), ERR_INVALID, "q, idx and count"), (lambda: select(q=At(8)), ERR_UNSUPPORTED, "q must be 16-byte"),
    (lambda: select(work=N), ERR_INVALID, "workspace is NULL"), (lambda: select(work=At(16)), ERR_UNSUPPORTED, "256-byte"),
    (lambda: select(work=At(0, 128)), ERR_WORKSPACE, "workspace has 128 bytes"), (lambda: select(s=step(q_strides=(0, 64, 128))), ERR_UNSUPPORTED, "q strides"),
    (lambda: select(s=step(q_strides=(0, 1024, 4))), ERR_UNSUPPORTED, "q strides"), (lambda: select(s=step(lengths=N)), ERR_INVALID, "lengths"),
    (lambda: select(s=step(n_q_heads=6)), ERR_INVALID, r"n_q_heads \(6\)"), (lambda: select(s=step(total_new=3)), ERR_INVALID, "multiple of batch"),
    (lambda: select(s=step(n_q_heads=65536)), ERR_UNSUPPORTED, "65535"), (lambda: select(s=step(total_new=1 << 20, max_new=1 << 20)), ERR_UNSUPPORTED, "2\\^22"),
    (lambda: select(s=step(total_new=-2)), ERR_INVALID, "negative"), (lambda: select(s=step(max_new=-1)), ERR_INVALID, "negative"),
    (lambda: sparse(q=N), ERR_INVALID, "q and out"), (lambda: sparse(out=N), ERR_INVALID, "q and out"), (lambda: sparse(idx=N), ERR_INVALID, "idx and count"),
    (lambda: sparse(count=N), ERR_INVALID, "idx and count"), (lambda: sparse(out=At(8)), ERR_UNSUPPORTED, "16-byte"),
    (lambda: sparse(work=N), ERR_INVALID, "workspace is NULL"), (lambda: sparse(work=At(16)), ERR_UNSUPPORTED, "256-byte"),
    (lambda: sparse(work=At(0, 128)), ERR_WORKSPACE, "workspace has 128 bytes"), (lambda: sparse(s=step(scale=0.0)), ERR_INVALID, "scale"),
    (lambda: sparse(s=step(softcap=-1.0)), ERR_INVALID, "softcap"), (lambda: sparse(s=step(scale=0.1, softcap=1e36)), ERR_UNSUPPORTED, "must be from"),
    (lambda: sparse(s=step(q_strides=(4, 1024, 128))), ERR_UNSUPPORTED, "q strides"), (lambda: sparse(s=step(total_new=1 << 21, max_new=1 << 21)), ERR_UNSUPPORTED, "2\\^23"),
    (lambda: sparse(s=step(lengths=N)), ERR_INVALID, "lengths"), (lambda: sparse(p=fp4(v_scales=N)), ERR_INVALID, "k_scales and v_scales"),
]


@pytest.mark.parametrize("call,code,message", REFUSED, ids=[str(i) for i in range(len(REFUSED))])
def test_refusals(call, code, message):
    with pytest.raises(D.DapqError, match=message) as e:
        call()
    assert e.value.code == code


@pytest.mark.parametrize("call,figure", [(lambda s: attention(s=s), lambda s: D.paged_attention_workspace_bytes(pages(), s)),
                                         (lambda s: sparse(s=s), lambda s: D.paged_sparse_attention_workspace_bytes(pages(), blocks(), s))], ids=["attention", "sparse"])
def test_more_query_heads_than_a_launch_has_are_refused(call, figure):
    for heads in (65536, 1 << 30):
        with pytest.raises(D.DapqError, match="exceeds 65535") as e:
            call(step(n_q_heads=heads))
        assert e.value.code == ERR_UNSUPPORTED and figure(step(n_q_heads=heads)) == 0
    assert figure(step(n_q_heads=65532)) > 0


def test_nothing_to_do_is_no_error():
    """No new tokens or rows: nothing is enqueued (there is no GPU here), whatever the buffers."""
    bounds(rows=0)
    bounds(first=N, rows=0)
    for s in (step(total_new=0), step(max_new=0), step(total_new=0, cu_new=A)):
        select(s=s)
        sparse(s=s)
        sparse(b=blocks(bounds=N, scales=N), s=s)


def test_descriptors_have_the_header_s_layout():
    assert C.sizeof(binding.Blocks) == 4 * 4 + 2 * 8
    for bad in (lambda: D.dapq_paged_bounds(pages(), step(), A, A, 8, 0), lambda: D.dapq_paged_select(pages(), step(), step(), A, A, A, A, 0),
                lambda: D.dapq_paged_select(pages(), blocks(), pages(), A, A, A, A, 0),
                lambda: D.dapq_paged_sparse_attention(blocks(), blocks(), step(), A, A, A, A, A, 0)):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(D.DapqError, match=r"max_rows \(-8\)"):   # (a number that only ctypes converts)
        D.dapq_paged_bounds(pages(), blocks(), A, A, C.c_int32(-8), 0)


def test_workspace_bytes_depend_on_no_device_data():
    """The figures are the same whatever table, lengths and cu_new hold: their addresses are not followed (here they are no memory)."""
    for p in (pages(), fp4(), pages(batch=64, max_pages=1 << 16), fp4(n_layers=8, n_kv_heads=8, page_rows=64)):
        for b in (blocks(), blocks(n_select=4096), blocks(block_rows=p.page_rows)):
            for s in (step(total_new=p.batch, n_q_heads=64), step(total_new=64 * p.batch, max_new=64), step(total_new=5, max_new=5, cu_new=A)):
                s.lengths = 1 << 60
                p.table = 1 << 60
                for figure in (D.paged_select_workspace_bytes, D.paged_sparse_attention_workspace_bytes):
                    n = figure(p, b, s)
                    assert n > 0 and n % 256 == 0
    # a row of scores for every token and KV head, as wide as the table, where a second kernel reads them
    assert D.paged_select_workspace_bytes(pages(max_pages=100), blocks(), step(total_new=8, max_new=4)) >= 8 * 4 * 100 * 4
    assert D.paged_select_workspace_bytes(pages(max_pages=100), blocks(), step()) == 256


def test_the_largest_descriptors():
    """At the limits, products of descriptors stay in their types (the sanitized library runs this too)."""
    for p in (pages(batch=(1 << 24) - 1, n_kv_heads=1, max_pages=(1 << 26) - 1), pages(n_kv_heads=65535, batch=255, page_rows=1024, max_pages=(1 << 20) - 1)):
        s = step(total_new=63, max_new=63, cu_new=A, n_q_heads=p.n_kv_heads)
        assert D.paged_select_workspace_bytes(p, blocks(n_select=4096), s) >= 63 * p.n_kv_heads * 4 * (p.max_pages * p.page_rows // 16)
        assert D.paged_sparse_attention_workspace_bytes(p, blocks(n_select=4096), s) > 0


# --- the definition ---------------------------------------------------------------------------------------------------------
def test_bounds_by_hand():
    keys = np.zeros((16, 128))
    keys[3, 0], keys[7, 0], keys[2, 1], keys[4, 2] = 1.0, -0.25, 0.001, -3.0
    upper, lower, s = BO.block_bounds(keys)
    assert s == 127 - 5 and upper[:4].tolist() == [32, 1, 0, 0] and lower[:4].tolist() == [-8, 0, -96, 0]      # 3 <= 127 / 32 = 3.97, 3 > 127 / 64
    assert BO.block_bounds(np.full((16, 128), 127.0))[2] == 127 and BO.block_bounds(np.full((16, 128), 127.5))[2] == 128
    assert BO.block_bounds(np.zeros((16, 128)))[2] == 77 and BO.block_bounds(np.full((16, 128), 1e30))[0].tolist() == [127] * 128
    keys[5, 5] = np.inf
    upper, lower, s = BO.block_bounds(keys)
    assert s == 255 and not upper.any() and not lower.any()


def test_bounds_hold_every_key():
    rng = np.random.default_rng(0)
    for _ in range(50):
        keys = O.bf16_bits_to_f64(O.f64_to_bf16_bits(rng.standard_normal((32, 128)) * np.exp(rng.uniform(-9, 9)) * np.exp(rng.uniform(-3, 3, 128))))
        upper, lower, s = BO.block_bounds(keys)
        u = 2.0 ** (s - 127.0)
        assert (keys <= upper * u).all() and (keys >= lower * u).all() and (upper * u - keys.max(0) < u).all() and (keys.min(0) - lower * u < u).all()
        q, f = BO.whole_query(rng.standard_normal(128))
        assert (np.maximum(q * upper, q * lower).sum() * u >= (keys @ q).max()).all()


def test_selection_by_hand():
    """Six blocks of one head; query (1, -1, 0, ...): scores upper[0] - lower[1] in units of their scales."""
    ul = np.zeros((1, 2, 1, 4, 2, 128), np.int8)
    scales = np.full((1, 2, 1, 4), 127, np.uint8)
    score = {0: (1, 0, 127), 1: (9, -4, 127), 2: (6, -7, 127), 3: (13, 0, 126), 4: (5, 0, 128), 5: (99, 0, 127)}
    for b, (up, down, s) in score.items():
        ul[0, b // 4, 0, b % 4, 0, 0], ul[0, b // 4, 0, b % 4, 1, 1], scales[0, b // 4, 0, b % 4] = up, down, s
    q = np.zeros((1, 1, 1, 128))
    q[0, 0, 0, :2] = 1.0, -1.0
    table = np.array([[0, 1]], np.int32)

    def chosen(n, first, last, rows=96, table=table):
        return BO.select(table, 2, 64, ul, scales, 16, n, first, last, [rows - 1], [0, 1], 1, q)[0, 0, 0]

    assert chosen(6, 0, 1) == [0, 1, 2, 3, 4, 5] and chosen(2, 0, 1) == [1, 5]     # 1 and 2 both score 13: the first
    assert chosen(3, 0, 1) == [1, 2, 5] and chosen(4, 0, 1) == [1, 2, 4, 5]       # 4: 5 * 2 = 10 > 13 / 2
    assert chosen(3, 1, 1) == [0, 1, 5] and chosen(3, 1, 2) == [0, 4, 5] and chosen(2, 0, 1, 80) == [1, 4]
    scales[0, 0, 0, 3] = 255
    assert chosen(2, 0, 1) == [3, 5]
    assert chosen(2, 0, 1, table=np.array([[-1, 1]], np.int32)) == [4, 5] and chosen(2, 0, 1, table=np.array([[0, 9]], np.int32)) == [1, 3]
