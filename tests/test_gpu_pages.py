"""Page tables, copies of pages and accepted paths: each against its definition, equal to the last bit."""
import random

import pytest
import torch

import paged
import trees
from paged import PAGE
from test_gpu_cache import _cache, _gen, _params, _same, m  # noqa: F401

pytestmark = pytest.mark.gpu


def _pool(m, refs, table, stride=None):  # noqa: F811
    t = torch.tensor(table, dtype=torch.int32, device="cuda")
    if stride:                              # part of a wider table
        wide = torch.full((t.shape[0], stride), 77, dtype=torch.int32, device="cuda")
        wide[:, :t.shape[1]] = t
        t = wide[:, :t.shape[1]]
    return m.PagePool(torch.tensor(refs, dtype=torch.int32, device="cuda"), t)


def _same_pool(pool, want):
    return pool.refs.tolist() == want.refs and pool.page_table.tolist() == want.table


@pytest.mark.parametrize("pages,rows,blocks,stride", [(1, 1, 1, None), (7, 3, 4, 9), (300, 20, 20, None), (9000, 64, 100, None), (40000, 9, 3000, 3001), (600, 4096, 2, None)])
def test_resize(m, pages, rows, blocks, stride):  # noqa: F811
    """Sequences grow, shrink and go in any order, into pools with too few pages as well; pages that are shared are free when the last one lets go."""
    rng = random.Random(pages)
    lens = [0] * rows
    want = trees.Pool([0] * pages, [[-1] * blocks for _ in range(rows)])
    pool = _pool(m, want.refs, want.table, stride)
    for step in range(6):
        fill = [0.3, 1.2, 0.5, 2.0, 0.0, 0.8][step]
        new = [min(blocks * PAGE, int(rng.random() * 2 * fill * pages / rows * PAGE)) if rng.random() < 0.8 else x for x in lens]
        short = want.resize(lens, new)
        got = m.pages_resize(pool, lens, new)
        assert _same_pool(pool, want), step
        assert int(got) == short
        lens = new
    assert stride is None or bool((pool.page_table._base[:, blocks:] == 77).all())
    m.pages_resize(pool, lens, [0] * rows)
    assert int(pool.refs.abs().sum()) == 0 and bool((pool.page_table == -1).all())


@pytest.mark.parametrize("pages,rows,blocks", [(5, 2, 3), (400, 40, 12), (20000, 300, 600)])
def test_fork(m, pages, rows, blocks):  # noqa: F811
    """Continuations of whole and partial last blocks, of prefixes, several of one source, in the place of others; sources with pages that are not there; pools
    that run out; rows freed one by one afterwards."""
    rng = random.Random(rows)
    want = trees.Pool([0] * pages, [[-1] * blocks for _ in range(rows)])
    lens = [0] * rows
    pool = _pool(m, want.refs, want.table)
    first = [rng.randint(1, blocks * PAGE) if b < rows // 3 + 1 else 0 for b in range(rows)]
    want.resize(lens, first)
    m.pages_resize(pool, lens, first)
    lens = first
    for step in range(5):
        order = list(range(rows))
        rng.shuffle(order)
        src, dst = order[:rows // 3 + 1], order[rows // 3 + 1:]
        dst = dst[:rng.randint(1, len(dst))]
        of = [rng.choice(src) for _ in dst]
        tokens = [rng.choice([lens[s], lens[s] // PAGE * PAGE, rng.randint(0, lens[s])]) for s in of]
        old = [lens[d] for d in dst]
        copies, short = want.fork(of, dst, tokens, old)
        got, lacking = m.pages_fork(pool, m.Forks(of, dst, tokens, old))
        assert _same_pool(pool, want), step
        assert got.tolist() == copies and int(lacking) == short
        for d, n in zip(dst, tokens):
            lens[d] = n
        if step == 2:                       # a page that is not there
            b = src[0]
            if lens[b]:
                want.give(b, 0)
                page = int(pool.page_table[b, 0])
                if 0 <= page < pages:
                    pool.refs[page] -= 1
                pool.page_table[b, 0] = -1
    for b in rng.sample(range(rows), rows):
        new = list(lens)
        new[b] = 0
        if b % 7 == 0 or rows < 50:
            want.resize(lens, new)
            m.pages_resize(pool, lens, new)
            lens = new
    assert _same_pool(pool, want)


def test_nothing_to_do(m):  # noqa: F811
    """No sequences, no forks, lengths that stay, prefixes of no tokens: nothing changes, nothing is wanting."""
    pool = _pool(m, [1, 0, 1], [[0, 2], [-1, -1]])
    assert int(m.pages_resize(pool, [], [])) == 0 and int(m.pages_resize(pool, [100, 0], [128, 0])) == 0
    copies, short = m.pages_fork(pool, m.Forks([], [], [], []))
    assert copies.shape == (0, 2) and int(short) == 0
    copies, short = m.pages_fork(pool, m.Forks([0], [1], [0]))
    assert copies.tolist() == [[-1, -1]] and int(short) == 0
    moves, live = m.pages_compact(pool, [128, 0])
    assert pool.refs.tolist() == [1, 1, 0] and pool.page_table.tolist() == [[0, 1], [-1, -1]] and moves.tolist() == [[2, 1]] and live.tolist() == [2, 1]


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("pages,rows,blocks", [(1, 1, 1), (2, 1, 2), (9, 3, 4), (1000, 30, 40), (4096, 16, 128), (4097, 16, 128), (4096, 683, 3), (50000, 40, 1500)])
def test_compact(m, pages, rows, blocks, apart):  # noqa: F811
    rng = random.Random(pages + 1)
    for fill in (0.0, 0.4, 0.9, 1.0):
        lens = [min(blocks * PAGE, int(rng.random() * 2 * fill * pages / rows * PAGE)) for _ in range(rows)]
        free = rng.sample(range(pages), pages)
        table, refs = [[-1] * blocks for _ in range(rows)], [0] * pages
        for b, n in enumerate(lens):
            for j in range(trees.Pool.blocks(n)):
                page = table[b - 1][j] if b and j < 3 and table[b - 1][j] >= 0 and b % 2 else free.pop() if free else -1         # (some are shared)
                table[b][j] = page
                if page >= 0:
                    refs[page] += 1
        want = trees.Pool(refs, table)
        pool = _pool(m, refs, table)
        out = _pool(m, [7] * pages, [[55] * (blocks + 3) for _ in range(rows)]) if apart else None
        pairs, live = want.compact(lens)
        moves, n = m.pages_compact(pool, lens, out)
        assert n.tolist() == [live, len(pairs)] and moves.tolist() == pairs + [[-1, -1]] * (pages // 2 - len(pairs))
        if apart:
            assert pool.refs.tolist() == refs and pool.page_table.tolist() == table
            want.table = [r + [-1] * 3 for r in want.table]
        assert _same_pool(out or pool, want)


def _random_cache(m, p, lens, kv, seed, layout="heads"):  # noqa: F811
    """pages full of rows of any magnitude, some not finite"""
    c = _cache(m, p, lens, kv, seed, layout)
    gen = _gen(seed)
    for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)):
        if kv == "e4m3":
            x.view(torch.uint8).copy_(torch.randint(0, 256, x.shape, generator=gen, device="cuda", dtype=torch.uint8))
            s.copy_(torch.exp2(torch.randint(-6, 7, s.shape, generator=gen, device="cuda").float()))
        else:
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
            x.masked_fill_(torch.rand(x.shape, generator=gen, device="cuda") < 0.01, float("inf"))
    return c


def _state(c):
    return [c.k.clone(), c.v.clone()] + ([c.k_scale.clone(), c.v_scale.clone()] if c.k_scale is not None else [None, None])


CACHES = [("bf16", 2, 128, "heads", "e4m3"), ("bf16", 3, 64, "tokens", "native"), ("fp32", 1, 64, "heads", "e4m3"), ("fp32", 2, 128, "tokens", "native"),
          ("bf16", 1, 128, "heads", "native")]


@pytest.mark.parametrize("dtype,hkv,d,layout,kv", CACHES)
def test_copies(m, dtype, hkv, d, layout, kv):  # noqa: F811
    p = _params(m, dtype, hkv, hkv, d)
    c = _random_cache(m, p, [64 * 40], kv, 3, layout)
    pages = c.k.shape[0]
    k, v, ks, vs = _state(c)
    pairs = [[0, 1], [5, 2], [-1, -1], [3, pages], [pages, 4], [6, -5], [0, 7], [9, 9], [5, pages - 1], [-(1 << 31), 3], [(1 << 31) - 1, 3]]
    m.cache_copy_pages(p, c, torch.tensor(pairs, dtype=torch.int32, device="cuda"))
    for a, b in pairs:
        if 0 <= a < pages and 0 <= b < pages:
            for x in (k, v) if kv == "native" else (k.view(torch.uint8), v.view(torch.uint8), ks, vs):
                x[b] = x[a]
    assert _same(c.k, k) and _same(c.v, v)
    assert ks is None or (torch.equal(c.k_scale, ks) and torch.equal(c.v_scale, vs))
    m.cache_copy_pages(p, c, torch.empty((0, 2), dtype=torch.int32, device="cuda"))


PATHS = [[], [0], [1], [0, 1, 2], [0, 2, 3, 7], [5, 6, 7], [2, 2, 3], [3, 1], [0, -1, 5], [0, 1, 40], list(range(1, 30, 2)), [0, 4, 9, 10, 20, 33, 39]]


@pytest.mark.parametrize("dtype,hkv,d,layout,kv", CACHES)
@pytest.mark.parametrize("front", [0, 1, 60, 64, 127, 300])
def test_accepted_paths(m, dtype, hkv, d, layout, kv, front):  # noqa: F811
    """Paths of one sequence each (none, the first tokens, gaps, ones that end early, over page ends); NaN and infinities among the rows, scales that grow."""
    p = _params(m, dtype, hkv, hkv, d)
    news, steps = [40] * len(PATHS), max(map(len, PATHS)) + 1
    ctxs = [front + 40] * len(PATHS)
    c = _random_cache(m, p, ctxs, kv, front + 1, layout)
    k, v, ks, vs = _state(c)
    want = trees.accept(k, v, None if ks is None else (ks, vs), c.page_table, news, ctxs, PATHS)
    path = torch.tensor([x + [-1] * (steps - len(x)) for x in PATHS], dtype=torch.int32, device="cuda")
    cu = [40 * i for i in range(len(PATHS) + 1)]
    got = m.cache_accept(p, c, cu, ctxs, path)
    assert got.tolist() == want
    assert _same(c.k, k) and _same(c.v, v)
    assert ks is None or (torch.equal(c.k_scale, ks) and torch.equal(c.v_scale, vs))


@pytest.mark.parametrize("dtype,hkv,d,layout,kv", CACHES)
def test_long_paths(m, dtype, hkv, d, layout, kv):  # noqa: F811
    """Paths over several pages (each page's rows come from its own and later ones), a path without room for its end, sequences without drafted tokens, pages
    that are not there."""
    p = _params(m, dtype, hkv, hkv, d)
    rng = random.Random(d + hkv)
    news, fronts = [700, 0, 333, 1, 900, 64], [30, 77, 0, 64, 500, 63]
    paths = [sorted(rng.sample(range(n), n * 2 // 3)) for n in news]
    paths[4] = list(range(5, 300))
    paths[5] = list(range(64))
    ctxs = [a + b for a, b in zip(news, fronts)]
    c = _random_cache(m, p, ctxs, kv, 8, layout)
    c.page_table[0, 3], c.page_table[4, 8], c.page_table[2, 5] = -1, c.k.shape[0], -(1 << 31)
    k, v, ks, vs = _state(c)
    steps = 400
    want = trees.accept(k, v, None if ks is None else (ks, vs), c.page_table, news, ctxs, [x[:steps] for x in paths])
    path = torch.tensor([(x + [-1] * steps)[:steps] for x in paths], dtype=torch.int32, device="cuda")
    cu = [sum(news[:i]) for i in range(len(news) + 1)]
    got = m.cache_accept(p, c, cu, ctxs, path)
    assert got.tolist() == want
    assert _same(c.k, k) and _same(c.v, v)
    assert ks is None or (torch.equal(c.k_scale, ks) and torch.equal(c.v_scale, vs))


def test_paths_of_sequences_without_drafted_tokens(m):  # noqa: F811
    """Lengths stay as they are, and so does the cache."""
    p = m.Params.make("bf16", 8, 2, 64)
    ctxs = [100, 0, 64]
    c = _random_cache(m, p, ctxs, "e4m3", 5)
    k, v, ks, vs = _state(c)
    path = torch.zeros((3, 4), dtype=torch.int32, device="cuda")
    assert m.cache_accept(p, c, [0, 0, 0, 0], ctxs, path).tolist() == ctxs
    assert _same(c.k, k) and _same(c.v, v) and torch.equal(c.k_scale, ks) and torch.equal(c.v_scale, vs)
