"""What the calls of the cache in pages refuse at the ends of their descriptors' integers, before anything is enqueued."""
import pytest

import paper_2603_11564_amd as D
from test_paged_host import A, ERR_INVALID, ERR_UNSUPPORTED, append, attention, fp4, gather, pages, read, step

MOST, LEAST = 2 ** 31 - 1, -2 ** 31
PAGES = [
    (dict(n_layers=MOST, batch=MOST, n_kv_heads=MOST), ERR_UNSUPPORTED, "exceeds 65535"),
    (dict(n_layers=1 << 22, batch=1 << 21, n_kv_heads=1 << 21), ERR_UNSUPPORTED, "exceeds 65535"),  # (2^64 together)
    (dict(n_layers=MOST, batch=MOST, n_kv_heads=1), ERR_UNSUPPORTED, "exceeds 65535"),
    (dict(n_layers=1, batch=MOST, n_kv_heads=65535), ERR_UNSUPPORTED, "2\\^24"),
    (dict(n_layers=1, batch=MOST, n_kv_heads=1), ERR_UNSUPPORTED, "2\\^24"),
    (dict(n_layers=LEAST, batch=LEAST, n_kv_heads=LEAST), ERR_INVALID, "must be >= 1"),
    (dict(n_layers=5, n_kv_heads=13107, n_pages=MOST, page_rows=1024), ERR_UNSUPPORTED, "2\\^36 rows"),
    (dict(n_pages=LEAST), ERR_INVALID, "must be >= 1"), (dict(max_pages=MOST, page_rows=1024), ERR_UNSUPPORTED, "2\\^30"),
    (dict(raw=dict(page_rows=LEAST)), ERR_UNSUPPORTED, "page_rows"), (dict(raw=dict(page_rows=MOST)), ERR_UNSUPPORTED, "page_rows"),
    (dict(raw=dict(head_dim=MOST)), ERR_UNSUPPORTED, "head_dim"), (dict(raw=dict(format=LEAST)), ERR_INVALID, "format"),
]


@pytest.mark.parametrize("make", [pages, fp4])
@pytest.mark.parametrize("bad,code,message", PAGES, ids=[str(i) for i in range(len(PAGES))])
def test_pages_at_the_ends_of_their_range(make, bad, code, message):
    for call in (append, read, attention, lambda p: gather(p=p)):
        with pytest.raises(D.DapqError, match=message) as e:
            call(make(**bad))
        assert e.value.code == code
    assert D.paged_attention_workspace_bytes(make(**bad), step()) == 0


STEPS = [
    (dict(total_new=2 ** 63 - 1, max_new=MOST), ERR_UNSUPPORTED, "2\\^25"), (dict(total_new=-2 ** 63), ERR_INVALID, "negative"),
    (dict(max_new=LEAST), ERR_INVALID, "negative"), (dict(n_q_heads=MOST), ERR_INVALID, "n_q_heads"), (dict(n_q_heads=LEAST), ERR_INVALID, "n_q_heads"),
    (dict(n_q_heads=MOST - 3, total_new=1 << 25, max_new=MOST), ERR_UNSUPPORTED, "65535"),
    (dict(n_q_heads=65532, total_new=1 << 25, max_new=MOST), ERR_UNSUPPORTED, "2\\^31"),
    (dict(q_strides=(2 ** 63 - 1, 1024, 128)), ERR_UNSUPPORTED, "q strides"), (dict(q_strides=(0, -2 ** 63, 128)), ERR_UNSUPPORTED, "q strides"),
]


@pytest.mark.parametrize("bad,code,message", STEPS, ids=[str(i) for i in range(len(STEPS))])
def test_steps_at_the_ends_of_their_range(bad, code, message):
    with pytest.raises(D.DapqError, match=message) as e:
        attention(s=step(**bad))
    assert e.value.code == code
    assert D.paged_attention_workspace_bytes(pages(), step(**bad)) == 0


def test_workspaces_of_the_largest_calls():
    """Nothing overflows on the way to the figure: the most sequences, heads, rows and tokens that are taken."""
    for p in (pages(batch=256, n_layers=1, n_kv_heads=65535), fp4(batch=(1 << 24) - 1, n_layers=1, n_kv_heads=1, max_pages=(1 << 26) - 1),
              pages(batch=1, n_layers=65535, n_kv_heads=1, max_pages=(1 << 20) - 1, page_rows=1024, n_pages=1)):
        for s in (step(n_q_heads=p.n_kv_heads, total_new=0), step(n_q_heads=p.n_kv_heads, total_new=(1 << 31) // 65536, max_new=MOST, cu_new=A),
                  step(n_q_heads=p.n_kv_heads, total_new=p.batch, max_new=1)):
            n = D.paged_attention_workspace_bytes(p, s)
            assert 0 < n < 1 << 60 and n % 256 == 0
