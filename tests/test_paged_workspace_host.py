"""The workspace of a step that reads chosen blocks, without a GPU: one that is large enough for a step is so for all smaller ones."""
import itertools

import pytest

import paper_2603_11564_amd as D
from test_paged_blocks_host import blocks
from test_paged_host import A, N, pages, step

FIGURES = [D.paged_select_workspace_bytes, D.paged_sparse_attention_workspace_bytes]


def figure_of(figure, batch, new, *, heads=8, group=4, layers=1, max_pages=256, page_rows=16, block_rows=16, n_select=128, max_new=None, cu=N):
    """Of a step of `new` tokens in all."""
    n = figure(pages(batch=batch, n_layers=layers, n_kv_heads=heads, max_pages=max_pages, n_pages=max_pages, page_rows=page_rows),
               blocks(n_select=n_select, n_first=0, block_rows=block_rows),
               step(n_q_heads=heads * group, total_new=new, max_new=new if max_new is None else max_new, cu_new=cu))
    assert n > 0 and n % 256 == 0
    return n


@pytest.mark.parametrize("figure", FIGURES)
@pytest.mark.parametrize("group", [1, 2, 4, 7, 8, 16, 32])
@pytest.mark.parametrize("max_pages", [4, 27, 64, 256, 2048, 8192, 20000])
def test_figures_do_not_fall_as_steps_grow(figure, group, max_pages):
    """In the sequences, their tokens, the layers, the width of the table and the chosen blocks."""
    def grows(values, of):
        got = [of(v) for v in values]
        assert got == sorted(got), list(zip(values, got))

    kw = dict(group=group, max_pages=max_pages)
    batches = [1, 2, 3, 8, 16, 31, 32, 33, 48, 64, 96, 97, 128, 200, 1024]
    for new in (1, 2, 4, 9):
        grows(batches, lambda b: figure_of(figure, b, new * b, max_new=new, **kw))
        grows(batches, lambda b: figure_of(figure, b, new * b, max_new=new, cu=A, **kw))
    for batch in (1, 8, 64):
        for cu in (N, A):
            grows([batch * t for t in (1, 2, 3, 4, 5, 8, 9, 16, 17, 33, 100)], lambda n: figure_of(figure, batch, n, cu=cu, **kw))
            grows([1, 2, 3, 4, 5, 8, 9, 17, 64], lambda most: figure_of(figure, batch, 8 * batch, max_new=most, cu=cu, **kw))
        grows([1, 2, 3, 8, 32], lambda layers: figure_of(figure, batch, batch, layers=layers, **kw))
        grows([1, 2, 3, 8, 32], lambda heads: figure_of(figure, batch, batch, heads=heads, **kw))
        grows([1, 16, 17, 32, 64, 128, 1000, 4096], lambda n: figure_of(figure, batch, batch, n_select=n, **kw))
        grows([1, 2, 7, 27, 28, 29, 100, 512, 513, 4096, 8192, 8193, 60000], lambda wide: figure_of(figure, batch, batch, group=group, max_pages=wide))


@pytest.mark.parametrize("figure", FIGURES)
def test_figures_do_not_depend_on_how_tokens_are_packed(figure):
    for batch, new, most, group, wide in itertools.product((1, 3, 64), (1, 2, 8), (1, 2, 8, 1000), (1, 4, 8), (8, 256, 2048)):
        kw = dict(max_new=most, group=group, max_pages=wide)
        assert figure_of(figure, batch, new * batch, **kw) == figure_of(figure, batch, new * batch, cu=A, **kw)


@pytest.mark.parametrize("figure", FIGURES)
def test_a_workspace_of_the_largest_step_serves_as_sequences_end(figure):
    """Sequences of a batch end one after the other, and a uniform step becomes a ragged one: through a table of 2048 pages, and of 256 with tokens drafted."""
    room = figure_of(figure, 64, 64, max_pages=2048)
    assert all(figure_of(figure, b, b, max_pages=2048, cu=cu) <= room for b in range(1, 65) for cu in (N, A))
    room = figure_of(figure, 64, 512, max_new=8)
    assert all(figure_of(figure, b, n, max_new=8, cu=A) <= room for b in range(1, 65) for n in (1, b, 2 * b, 8 * b - 1, 8 * b))
