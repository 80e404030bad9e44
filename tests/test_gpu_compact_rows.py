"""Compaction of pools whose tables have more rows than there are sequences: the other rows hold no entries afterwards."""
import random

import pytest

import trees
from test_gpu_cache import m  # noqa: F401
from test_gpu_pages import _pool, _same_pool
from paged import PAGE

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("pages,rows,batch,blocks", [(9, 5, 3, 4), (40, 7, 0, 6), (1000, 30, 11, 40), (4096, 16, 15, 128), (5000, 300, 20, 130), (300, 4096, 17, 2)])
def test_fewer_sequences_than_rows(m, pages, rows, batch, blocks, apart):  # noqa: F811
    """The first `batch` rows hold the entries that are counted; what the others hold (numbers of pages that are free or another's by then) is not kept."""
    rng = random.Random(pages + rows)
    lens = [min(blocks * PAGE, int(rng.random() * 2 * 0.7 * pages / max(batch, 1) * PAGE)) for _ in range(batch)]
    free = rng.sample(range(pages), pages)
    table, refs = [[rng.randrange(-1, pages) for _ in range(blocks)] for _ in range(rows)], [0] * pages
    for b, n in enumerate(lens):
        for j in range(trees.Pool.blocks(n)):
            table[b][j] = free.pop() if free else -1
            if table[b][j] >= 0:
                refs[table[b][j]] += 1
    more = 6 if apart else 0                # rows of `out` beyond those of the pool
    want = trees.Pool(refs, table)
    pool = _pool(m, refs, table, blocks + 5)
    out = _pool(m, [7] * pages, [[55] * blocks for _ in range(rows + more)], blocks + 2) if apart else None
    pairs, live = want.compact(lens)
    moves, n = m.pages_compact(pool, lens, out)
    want.table = want.table[:batch] + [[-1] * blocks for _ in range(rows + more - batch)]
    assert n.tolist() == [live, len(pairs)] and moves.tolist() == pairs + [[-1, -1]] * (pages // 2 - len(pairs))
    if apart:
        assert pool.refs.tolist() == refs and pool.page_table.tolist() == table
    got = out or pool
    assert _same_pool(got, want)
    assert bool((got.page_table._base[:, blocks:] == 77).all())             # (the wider table around it)
