"""Trees of drafted tokens over the paged cache: ancestors and positions, attention against a plain form in 64 bits, a step from the draft to the accepted path."""
import math

import pytest
import torch

import paged
import trees
from paged import PAGE
from test_gpu_cache import SHAPES, _filled, _gen, _params, m  # noqa: F401

pytestmark = pytest.mark.gpu


def _cu(news):
    return [sum(news[:i]) for i in range(len(news) + 1)]


# ------------------------------------------------------------------------------------------------ masks
@pytest.mark.parametrize("order", [None, "any"])
@pytest.mark.parametrize("news", [[1], [26], [32, 33, 0, 64, 65], [5] * 100, [1024], [509, 3, 200, 1000], [700, 0, 1]])
def test_masks(m, news, order):  # noqa: F811
    gen = torch.Generator().manual_seed(sum(news))
    per = [trees.random_parents(n, gen, order=order) for n in news]
    ctxs = [n + 13 * b for b, n in enumerate(news)]
    parents = torch.tensor([x for p in per for x in p], dtype=torch.int32, device="cuda")
    mask, pos = m.tree_masks(parents, _cu(news), ctxs)
    words = (max(news) + 31) // 32
    sets = [trees.ancestors(p) for p in per]
    assert mask.shape == (sum(news), words) and torch.equal(mask.cpu(), trees.to_words([s for x in sets for s in x], words))
    assert pos.tolist() == [L - n + len(s) - 1 for x, L, n in zip(sets, ctxs, news) for s in x]
    wide = torch.full((sum(news), words + 3), -1, dtype=torch.int32, device="cuda")          # a mask with room for more
    m.tree_masks(parents, _cu(news), ctxs, mask=wide)
    assert torch.equal(wide[:, :words], mask) and bool((wide[:, words:] == 0).all())


def test_masks_of_chains_stars_and_what_is_no_tree(m):  # noqa: F811
    n = 1000
    per = [list(range(-1, n - 1)), [-1] * n, [n - 1] + list(range(n - 1)), [i + 1 for i in range(n)], [7 if i == 7 else -(1 << 31) for i in range(n)],
           [(1 << 31) - 1] * n]             # a chain, a star, a circle, a chain from behind, a token that is its own parent, numbers far outside
    mask, pos = m.tree_masks(torch.tensor(sum(per, []), dtype=torch.int32, device="cuda"), _cu([n] * 6), [n + 5] * 6)
    sets = [s for p in per for s in trees.ancestors(p)]
    assert torch.equal(mask.cpu(), trees.to_words(sets, 32))
    assert pos.tolist() == [5 + len(s) - 1 for s in sets]


# ------------------------------------------------------------------------------------------------ attention
def _check(m, p, c, q, news, ctxs, mask, lists=None, **kw):  # noqa: F811
    blocks = None
    if lists is not None:
        blocks = torch.tensor([[h + [-1] * (p.topk_total - len(h)) for h in b] for b in lists], dtype=torch.int32, device="cuda")
    out, lse = m.cache_tree_attn(p, c, q, _cu(news), ctxs, mask, blocks, **kw)
    sc = None if c.k_scale is None else (c.k_scale, c.v_scale)
    sets, t = [], 0
    words = mask.cpu()
    for n in news:
        sets += trees.to_sets(words[t:t + n], n)
        t += n
    want, want_lse, mass = trees.attention(q, c.k, c.v, sc, c.page_table, news, ctxs, sets, p.softmax_scale, lists, p.dense_threshold)
    # as for cache_attn: the result's own rounding; weights of 16 bits and more, logits in 32: 2^-12 (bf16) and 1e-4 (fp32) of |v| <= 6
    tol = 2.0 ** -8 * want.abs() + 6 * 2.0 ** -12 if q.dtype == torch.bfloat16 else torch.full_like(want, 1e-4)
    if q.dtype == torch.bfloat16 and max(news) > 8:
        # trees of more than 8 tokens: weights may be rounded to bf16 in front of the second product, p (1 + e) with |e| <= 2^-8
        many = torch.tensor([n > 8 for n in news for _ in range(n)], device="cuda")
        tol = tol + 2.0 ** -8 * mass * many[:, None, None]
    bad = ~((out.double() - want).abs() <= tol)
    assert not bool(bad.any()), (torch.nonzero(bad)[:4].tolist(), float((out.double() - want).abs().max()))
    none = torch.isinf(want_lse)
    assert torch.equal(none, torch.isinf(lse)) and bool((out[none] == 0).all())
    assert float((lse.double() - want_lse)[~none].abs().max() if bool((~none).any()) else 0) <= 1e-4
    return out, lse


def _masks(m, news, ctxs, seed):  # noqa: F811
    gen = torch.Generator().manual_seed(seed)
    parents = [x for n in news for x in trees.random_parents(n, gen)]
    return m.tree_masks(torch.tensor(parents, dtype=torch.int32, device="cuda"), _cu(news), ctxs)[0]


def _q(p, news, seed):
    return torch.randn((sum(news), p.num_q_heads, p.head_dim), generator=_gen(seed), device="cuda").to(p.torch_dtype)


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
def test_trees_over_contexts(m, kv, dtype, hq, hkv, d):  # noqa: F811
    """One token to large trees for each sequence, contexts of no tokens and around page ends, sequences without drafted tokens."""
    p = _params(m, dtype, hq, hkv, d)
    news, ctxs = [1, 1, 2, 0, 7, 8, 9, 26, 33, 64, 90, 5], [1, 64, 66, 50, 7, 72, 300, 26, 97, 1000, 200, 2000]
    c, _, _ = _filled(m, p, ctxs, kv, 21, "tokens" if d == 64 else "heads")
    _check(m, p, c, _q(p, news, 5), news, ctxs, _masks(m, news, ctxs, 3))


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
def test_any_mask(m, kv, dtype, hq, hkv, d):  # noqa: F811
    """Masks that are no tree's: rows of random bits, without the token itself, of later tokens, empty ones; bits behind the tree; contexts of no tokens, so that rows
    have no key at all; pages that are not there."""
    p = _params(m, dtype, hq, hkv, d)
    news, ctxs = [3, 40, 70, 12, 4], [3, 40, 500, 140, 260]
    c, _, _ = _filled(m, p, ctxs, kv, 22)
    gen = _gen(9)
    mask = torch.randint(-(1 << 31), 1 << 31, (sum(news), 4), generator=gen, device="cuda", dtype=torch.int64).to(torch.int32)
    mask[::5] = 0
    mask[1::7] = -1
    _check(m, p, c, _q(p, news, 6), news, ctxs, mask)
    c.page_table[2, 6], c.page_table[2, 1], c.page_table[3, 1], c.page_table[4, :] = -1, c.k.shape[0], -(1 << 31), -1
    _check(m, p, c, _q(p, news, 7), news, ctxs, mask)


def _lists(p, news, ctxs, seed):
    gen = torch.Generator().manual_seed(seed)
    out = []
    for n, L in zip(news, ctxs):
        per = []
        for _ in range(p.num_kv_heads):
            k = int(torch.randint(0, p.topk_total + 1, (1,), generator=gen))            # empty lists among them
            per.append(torch.randperm((L - n + PAGE - 1) // PAGE, generator=gen)[:k].tolist())
        out.append(per)
    return out


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
def test_trees_over_lists(m, kv, dtype, hq, hkv, d):  # noqa: F811
    """Listed blocks of the context, with and without the one that drafted rows begin in, in any order, empty lists, lists longer than the context; a dense sequence
    among them; entries outside; pages that are not there."""
    p = _params(m, dtype, hq, hkv, d, topk_total=12, dense_threshold=100)
    news, ctxs = [9, 1, 26, 64, 40, 5, 33, 8], [1500, 99, 720, 264, 41, 300, 97, 3000]
    c, _, _ = _filled(m, p, ctxs, kv, 31)
    lists = _lists(p, news, ctxs, 3)
    lists[0][0] = [23, 2, -7, 24, 1 << 30, 0, 9]
    lists[3] = [[3, 0] if h % 2 == 0 else [0] for h in range(hkv)]               # rows 0 .. 199 are the context: block 3 is shared with the tree
    mask = _masks(m, news, ctxs, 4)
    q = _q(p, news, 8)
    blocks = [[[j for j in h if 0 <= j * PAGE < L - n] for h in b] for b, n, L in zip(lists, news, ctxs)]
    _check(m, p, c, q, news, ctxs, mask, blocks)
    raw = torch.tensor([[h + [-1] * (p.topk_total - len(h)) for h in b] for b in lists], dtype=torch.int32, device="cuda")
    last = torch.tensor([(L - n + PAGE - 1) // PAGE for n, L in zip(news, ctxs)], dtype=torch.int32, device="cuda")[:, None, None]
    skipped = torch.where(raw >= last, -1, raw)         # (in the same places: what a split goes through depends on them)
    assert torch.equal(m.cache_tree_attn(p, c, q, _cu(news), ctxs, mask, raw)[0], m.cache_tree_attn(p, c, q, _cu(news), ctxs, mask, skipped)[0])
    c.page_table[0, 2], c.page_table[2, 0], c.page_table[7, 46] = -1, c.k.shape[0], -(1 << 31)
    _check(m, p, c, q, news, ctxs, mask, blocks)


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("dtype,hq,hkv,d,n,ctx", [
    ("bf16", 32, 2, 128, 64, 9000), ("bf16", 32, 2, 128, 8, 20000), ("bf16", 32, 2, 128, 5, 33001), ("bf16", 8, 2, 64, 100, 7003), ("bf16", 8, 2, 64, 8, 30000),
    ("bf16", 4, 1, 64, 300, 5000), ("bf16", 12, 4, 128, 130, 3100), ("fp32", 8, 2, 64, 21, 5000), ("fp32", 6, 2, 128, 3, 9001)])
@pytest.mark.parametrize("listed", [False, True])
def test_long_contexts(m, kv, dtype, hq, hkv, d, n, ctx, listed):  # noqa: F811
    """Contexts that are split over workgroups, in both kernels and both tile sizes, with all pages and with lists."""
    p = _params(m, dtype, hq, hkv, d, topk_total=40)
    c, _, _ = _filled(m, p, [ctx, 77], kv, 41)
    news, ctxs = [n, 2], [ctx, 77]
    _check(m, p, c, _q(p, news, 9), news, ctxs, _masks(m, news, ctxs, 5), _lists(p, news, ctxs, 6) if listed else None)


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
def test_a_chain_is_proposed_tokens(m, kv, dtype, hq, hkv, d):  # noqa: F811
    """Every token the child of the one before it: what cache_attn gives, within both calls' roundings."""
    p = _params(m, dtype, hq, hkv, d)
    news, ctxs = [5, 1, 40, 8], [700, 130, 2000, 8]
    c, _, _ = _filled(m, p, ctxs, kv, 51)
    q = _q(p, news, 10)
    parents = torch.tensor([i - 1 for n in news for i in range(n)], dtype=torch.int32, device="cuda")
    mask, pos = m.tree_masks(parents, _cu(news), ctxs)
    assert pos.tolist() == [L - n + i for n, L in zip(news, ctxs) for i in range(n)]
    got, got_lse = m.cache_tree_attn(p, c, q, _cu(news), ctxs, mask)
    want, want_lse = m.cache_attn(p, c, q, _cu(news), ctxs)
    # each is off by its weights' rounding (2^-8 of |v| <= 6 on average over a few hundred keys, never above it) and its own
    tol = 2 * (2.0 ** -8 * want.double().abs() + 2.0 ** -8 * 6) if dtype == "bf16" else 2e-4
    assert bool(((got.double() - want.double()).abs() <= tol).all()) and float((got_lse - want_lse).abs().max()) <= 2e-4


@pytest.mark.parametrize("dtype,hq,hkv,d,n,ctx", [("bf16", 32, 2, 128, 5, 300), ("bf16", 32, 2, 128, 40, 2000), ("bf16", 8, 2, 64, 100, 9000), ("bf16", 5, 5, 64, 9, 90),
                                                  ("fp32", 4, 1, 64, 9, 300), ("bf16", 32, 2, 128, 8, 20000), ("bf16", 16, 16, 64, 1, 65)])
@pytest.mark.parametrize("kv", ["e4m3", "native"])
def test_rows_that_are_not_finite(m, kv, dtype, hq, hkv, d, n, ctx):  # noqa: F811
    """Values (and keys) of drafted rows that are infinite or NaN: outputs of the tokens that do not see them, and rows behind the sequence, are as without; the others
    are not finite in those channels."""
    p = _params(m, dtype, hq, hkv, d, topk_total=4)
    news, ctxs = [n], [ctx]
    c, _, _ = _filled(m, p, [ctx], kv, 61)
    q = _q(p, news, 11)
    mask = _masks(m, news, ctxs, 7)
    lists = torch.tensor([[[0, 2, -1, -1]] * hkv], dtype=torch.int32, device="cuda") if ctx - n > 192 else None
    for blocks in (None, lists):
        clean, _ = m.cache_tree_attn(p, c, q, [0, n], ctxs, mask, blocks)
        for j in sorted({0, n // 2, n - 1}):
            t = ctx - n + j
            page, row = int(c.page_table[0, t // PAGE]), t % PAGE
            was = c.v.view(torch.uint8 if kv == "e4m3" else p.torch_dtype)[page, :, row, 3].clone()
            if kv == "e4m3":
                c.v.view(torch.uint8)[page, :, row, 3] = 0x7f
            else:
                c.v[page, :, row, 3] = -float("inf")
            got, _ = m.cache_tree_attn(p, c, q, [0, n], ctxs, mask, blocks)
            c.v.view(torch.uint8 if kv == "e4m3" else p.torch_dtype)[page, :, row, 3] = was
            sees = torch.tensor([j in s for s in trees.to_sets(mask.cpu(), n)], device="cuda")
            bad = got[sees][..., 3]
            assert bool((torch.isnan(bad) if kv == "e4m3" else bad == -float("inf")).all())
            rest = [x for x in range(d) if x != 3]
            assert torch.equal(got[..., rest], clean[..., rest]) and torch.equal(got[~sees], clean[~sees])
    # a key of NaN: tokens that do not see it
    t = ctx - n + n // 2
    page, row = int(c.page_table[0, t // PAGE]), t % PAGE
    clean, _ = m.cache_tree_attn(p, c, q, [0, n], ctxs, mask)
    if kv == "e4m3":
        c.k.view(torch.uint8)[page, :, row, :] = 0x7f
    else:
        c.k[page, :, row, :] = float("nan")
    got, _ = m.cache_tree_attn(p, c, q, [0, n], ctxs, mask)
    sees = torch.tensor([n // 2 in s for s in trees.to_sets(mask.cpu(), n)], device="cuda")
    assert torch.equal(got[~sees], clean[~sees])


@pytest.mark.parametrize("dtype,hq,hkv,d,n,ctx", [("bf16", 32, 2, 128, 3, 300), ("bf16", 32, 2, 128, 2, 9001), ("bf16", 8, 2, 64, 6, 9001), ("fp32", 4, 1, 64, 9, 9001), ("fp32", 6, 2, 128, 70, 330),
                                                  ("bf16", 32, 2, 128, 40, 9001), ("bf16", 8, 2, 64, 70, 3001), ("bf16", 12, 4, 128, 8, 30001)])
@pytest.mark.parametrize("kv", ["e4m3", "native"])
def test_rows_beside_the_tree_that_are_not_finite(m, kv, dtype, hq, hkv, d, n, ctx):  # noqa: F811
    """An infinite (e4m3: NaN) value in a row of the context, in the block that drafted rows begin in, of a drafted row, and behind the sequence: each token gets those
    that it sees, in calls of one and of several splits, with the block listed and not."""
    p = _params(m, dtype, hq, hkv, d, topk_total=70, dense_threshold=0)
    c, _, _ = _filled(m, p, [ctx], kv, 65)
    q, mask = _q(p, [n], 17), _masks(m, [n], [ctx], 18)
    front = (ctx - n) // PAGE
    assert (ctx - n) % PAGE > 0 and ctx % PAGE > 0
    clean = {}
    blocks = {"all": None, "listed": [front, 0, 1], "not listed": [0, 1]}
    give = lambda x: None if x is None else torch.tensor([[x + [-1] * (70 - len(x))] * hkv], dtype=torch.int32, device="cuda")  # noqa: E731
    for name, x in blocks.items():
        clean[name] = m.cache_tree_attn(p, c, q, [0, n], [ctx], mask, give(x))[0]
    raw = c.v.view(torch.uint8) if kv == "e4m3" else c.v
    bad = 0x7f if kv == "e4m3" else float("inf")
    sees = torch.tensor([n - 1 in s for s in trees.to_sets(mask.cpu(), n)], device="cuda")
    rows = [(ctx - n - 1, 5, None), (ctx - 1, 6, sees)] + [(t, 7, torch.zeros(n, dtype=torch.bool, device="cuda")) for t in range(ctx, front * PAGE + PAGE)]
    for t, ch, _ in rows:
        raw[int(c.page_table[0, t // PAGE]), :, t % PAGE, ch] = bad
    for name, x in blocks.items():
        got = m.cache_tree_attn(p, c, q, [0, n], [ctx], mask, give(x))[0]
        want = clean[name].clone()
        for t, ch, who in rows:
            who = torch.full((n,), name != "not listed", device="cuda") if who is None else who
            want[who, :, ch] = float("nan") if kv == "e4m3" else bad
        assert bool(((got == want) | (got.isnan() & want.isnan())).all()), name


def test_context_rows_that_are_not_listed(m):  # noqa: F811
    """The block that drafted rows begin in, not listed: its context rows are as if they were not there, whatever they hold."""
    for n, ctx, hq, hkv, d in ((5, 300, 32, 2, 128), (40, 2020, 32, 2, 128), (40, 2020, 8, 2, 64)):
        p = _params(m, "bf16", hq, hkv, d, topk_total=4)
        c, _, _ = _filled(m, p, [ctx], "native", 62)
        mask, q = _masks(m, [n], [ctx], 8), _q(p, [n], 12)
        blocks = torch.tensor([[[1, 3, -1, -1]] * hkv], dtype=torch.int32, device="cuda")
        want = _check(m, p, c, q, [n], [ctx], mask, [[[1, 3]] * hkv])[0]
        front = (ctx - n) % PAGE
        page = int(c.page_table[0, (ctx - n) // PAGE])
        c.v[page, :, :front], c.k[page, :, :front] = float("inf"), float("nan")
        assert torch.equal(m.cache_tree_attn(p, c, q, [0, n], [ctx], mask, blocks)[0], want)


def test_outputs_of_sequences_without_drafted_tokens_and_scratch(m):  # noqa: F811
    """Output rows are those of the drafted tokens and no others; scratch of the size that was asked for, full of NaN before the call."""
    p = _params(m, "bf16", 32, 2, 128)
    news, ctxs = [0, 40, 0, 3, 0], [100, 9000, 64, 3000, 1]
    c, _, _ = _filled(m, p, ctxs, "e4m3", 71)
    mask, q = _masks(m, news, ctxs, 9), _q(p, news, 13)
    out = torch.full((50, 32, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((50, 32), 7.0, device="cuda")
    ws = torch.full((m.workspace_bytes(m.OP_CACHE_TREE_ATTN, p, 5, 43, 9000),), 0xff, dtype=torch.uint8, device="cuda")
    _check(m, p, c, q, news, ctxs, mask, out=out[:43], lse=lse[:43], workspace=ws)
    assert bool((out[43:] == 7).all()) and bool((lse[43:] == 7).all())


def test_a_step_from_the_draft_to_the_accepted_path(m):  # noqa: F811
    """Masks, append at the tree's positions, block lists of the newest token, attention, accepted paths, pages that the rest had, compressed keys: the cache is then that
    of the accepted tokens appended one after the other, and a decode step over it gives the same."""
    p = _params(m, "bf16", 32, 2, 128, topk_total=16, dense_threshold=512)
    rot = m.Rotary(m.rotary_turns(128), 128)
    rows, blocks, pages = 3, 60, 140
    pool = m.PagePool.empty(pages, rows, blocks)
    prev, n = [1000, 63, 2900], [40, 26, 64]
    both = [a + b for a, b in zip(prev, n)]
    assert int(m.pages_resize(pool, [0] * rows, prev)) == 0
    c = m.PagedCache.empty(p, pages, pool.page_table, "native")
    gen = _gen(90)
    k, v = (torch.randn((2, sum(prev), 128), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    m.cache_append(p, c, k, v, _cu(prev), [0] * rows, rot)
    kc = torch.zeros((rows, 2, m.num_cmp(p, max(both)), 128), device="cuda")
    m.cache_compress_k(p, c, kc, [0] * rows, prev)
    for step in range(2):
        # the draft
        assert int(m.pages_resize(pool, prev, both)) == 0
        host = torch.Generator().manual_seed(step)
        per = [trees.random_parents(x, host) for x in n]
        parents = torch.tensor(sum(per, []), dtype=torch.int32, device="cuda")
        mask, pos = m.tree_masks(parents, _cu(n), both)
        dk, dv = (torch.randn((2, sum(n), 128), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
        m.cache_append(p, c, dk, dv, _cu(n), prev, rot, pos)
        newest = torch.randn((rows, 32, 128), generator=gen, device="cuda").to(torch.bfloat16)
        lists = m.decode_blocks(p, newest, kc, prev)
        q = torch.randn((sum(n), 32, 128), generator=gen, device="cuda").to(torch.bfloat16)
        _check(m, p, c, q, n, both, mask, [[[j for j in h if j >= 0] for h in b] for b in lists.tolist()])
        # the path to the last token of each tree
        paths = [sorted(trees.ancestors(x)[-1]) for x in per]
        most = max(map(len, paths)) + 1
        path = torch.tensor([x + [-1] * (most - len(x)) for x in paths], dtype=torch.int32, device="cuda")
        lens = m.cache_accept(p, c, _cu(n), both, path).tolist()
        assert lens == [a + len(x) for a, x in zip(prev, paths)]
        m.pages_resize(pool, both, lens)
        m.cache_compress_k(p, c, kc, prev, lens)
        # the same, one after the other
        plain = m.PagedCache(p, c.k.clone(), c.v.clone(), pool.page_table)
        at = [[_cu(n)[b] + j for j in x] for b, x in enumerate(paths)]
        flat = torch.tensor(sum(at, []), device="cuda")
        m.cache_append(p, plain, dk[:, flat].contiguous(), dv[:, flat].contiguous(), _cu([len(x) for x in paths]), prev, rot)
        for b, L in enumerate(lens):
            for h in range(2):
                for x, y in ((c.k, plain.k), (c.v, plain.v)):
                    assert torch.equal(paged.rows_of(x, None, pool.page_table, b, L, h)[0], paged.rows_of(y, None, pool.page_table, b, L, h)[0])
        want_kc = torch.zeros_like(kc)
        m.cache_compress_k(p, plain, want_kc, [0] * rows, lens)
        for b, L in enumerate(lens):
            assert torch.equal(kc[b, :, :m.num_cmp(p, L)], want_kc[b, :, :m.num_cmp(p, L)])
        prev, both = lens, [a + b for a, b in zip(lens, n)]


def test_continuations_of_a_prompt(m):  # noqa: F811
    """Three continuations of one prompt share its pages, go on by themselves, one takes another's place, the pool is compacted: each attends to its own tokens."""
    p = _params(m, "bf16", 8, 2, 64)
    pool = m.PagePool.empty(64, 4, 20)
    c = m.PagedCache.empty(p, 64, pool.page_table, "e4m3")
    gen = _gen(91)
    new = lambda t: [torch.randn((2, t, 64), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2)]  # noqa: E731
    lens = [0, 0, 0, 0]

    def fork(src, dst, tokens):
        copies, short = m.pages_fork(pool, m.Forks(src, dst, tokens, [lens[d] for d in dst]))
        assert int(short) == 0
        m.cache_copy_pages(p, c, copies)
        for d, t in zip(dst, tokens):
            lens[d] = t

    def grow(more):
        nonlocal lens
        to = [a + b for a, b in zip(lens, more)]
        assert int(m.pages_resize(pool, lens, to)) == 0
        k, v = new(sum(more))
        m.cache_append(p, c, k, v, _cu(more), lens)
        lens = to

    def outputs():
        q = torch.randn((4, 8, 64), generator=_gen(92), device="cuda").to(torch.bfloat16)
        return m.cache_attn(p, c, q, [0, 1, 2, 3, 4], lens)[0]

    def rows(b, t):
        return [paged.rows_of(x, s, pool.page_table, b, t, h)[0] for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)) for h in range(2)]

    grow([500, 0, 0, 0])
    before = rows(0, 500)
    fork([0, 0, 0], [1, 2, 3], [500, 448, 300])
    assert int(pool.refs.max()) == 4
    for b, t in ((1, 500), (2, 448), (3, 300)):
        assert all(torch.equal(x, y[:t]) for x, y in zip(rows(b, t), before))
    grow([30, 100, 7, 64])
    assert all(torch.equal(x, y) for x, y in zip(rows(0, 448), [y[:448] for y in before]))
    fork([1], [2], [lens[1]])
    assert all(torch.equal(x, y) for x, y in zip(rows(1, lens[1]), rows(2, lens[1])))
    grow([1, 1, 1, 1])
    want, was = outputs(), [rows(b, lens[b]) for b in range(4)]
    drop = list(lens)
    drop[0] = 0
    m.pages_resize(pool, lens, drop)
    lens = drop
    moves, live = m.pages_compact(pool, lens)
    m.cache_copy_pages(p, c, moves)
    used = int((pool.refs > 0).sum())
    assert live.tolist()[0] == used and bool((pool.refs[:used] > 0).all()) and int(pool.page_table.max()) == used - 1
    lens[0] = lens[1]
    assert all(torch.equal(x, y) for b in range(1, 4) for x, y in zip(rows(b, lens[b]), was[b]))
    q = torch.randn((4, 8, 64), generator=_gen(92), device="cuda").to(torch.bfloat16)
    got = m.cache_attn(p, c, q[1:].contiguous(), [0, 0, 1, 2, 3], lens)[0]
    assert float((got.double() - want[1:].double()).abs().max()) <= 2.0 ** -7 * float(want.abs().max())          # (a bf16 rounding each)


def test_captured(m):  # noqa: F811
    """A speculative step and a fork in a captured graph, replayed with other inputs beside eager calls on another stream: the same bits."""
    p = _params(m, "bf16", 32, 2, 128, topk_total=16)
    n, prev = [26, 40], [3000, 500]
    both = [a + b for a, b in zip(n, prev)]
    pool = m.PagePool.empty(80, 4, 60)
    m.pages_resize(pool, [0] * 4, both + [0, 0])
    c = m.PagedCache.empty(p, 80, pool.page_table, "e4m3")
    k, v = (torch.randn((2, sum(prev), 128), generator=_gen(95), device="cuda").to(torch.bfloat16) for _ in range(2))
    m.cache_append(p, c, k, v, _cu(prev), [0, 0])
    cu, cx, pv = m.SeqInfo(_cu(n)), m.DecodeInfo(both), m.DecodeInfo(prev)
    parents = torch.empty(66, dtype=torch.int32, device="cuda")
    dk, dv = (torch.empty((2, 66, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q, out = (torch.empty((66, 32, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lse, path = torch.empty((66, 32), device="cuda"), torch.empty((2, 8), dtype=torch.int32, device="cuda")
    mask, pos, lens = torch.empty((66, 2), dtype=torch.int32, device="cuda"), torch.empty(66, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    ws = torch.empty(m.workspace_bytes(m.OP_CACHE_TREE_ATTN, p, 2, 66, max(both)), dtype=torch.uint8, device="cuda")
    forks = m.Forks([0, 1], [2, 3], [3000, 510], [3000, 510])
    copies, short = torch.empty((2, 2), dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    state = [x.view(torch.uint8) for x in (c.k, c.v)] + [c.k_scale, c.v_scale, pool.refs, pool.page_table]
    before = [x.clone() for x in state]

    def call():
        m.tree_masks(parents, cu, cx, mask, pos)
        m.cache_append(p, c, dk, dv, cu, pv, None)
        m.cache_tree_attn(p, c, q, cu, cx, mask, out=out, lse=lse, workspace=ws)
        m.cache_accept(p, c, cu, cx, path, lens)
        m.pages_fork(pool, forks, copies, short)
        m.cache_copy_pages(p, c, copies)

    def inputs(seed):
        host = torch.Generator().manual_seed(seed)
        per = [trees.random_parents(x, host) for x in n]
        parents.copy_(torch.tensor(sum(per, []), dtype=torch.int32))
        path.copy_(torch.tensor([(sorted(trees.ancestors(x)[-1 - seed]) + [-1] * 8)[:8] for x in per], dtype=torch.int32))
        gen = _gen(seed)
        for x in (dk, dv, q):
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        for x, y in zip(state, before):
            x.copy_(y)
        out.zero_()

    results = [out, lse, mask, pos, lens, copies, short] + state
    inputs(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for seed in (2, 3, 4):
        inputs(seed)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            call()
        side.synchronize()
        want = [x.clone() for x in results]
        inputs(seed)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(results, want)), seed


@pytest.mark.parametrize("dtype,hq,hkv,d,n,ctx", [("bf16", 32, 2, 128, 5, 300), ("bf16", 32, 2, 128, 40, 9000), ("bf16", 8, 2, 64, 100, 9000), ("fp32", 4, 1, 64, 9, 3000),
                                                  ("bf16", 32, 2, 128, 8, 20000)])
@pytest.mark.parametrize("kv", ["e4m3", "native"])
def test_large_values(m, kv, dtype, hq, hkv, d, n, ctx):  # noqa: F811
    """A mean of values next to the largest float is one of them, however many keys (drafted ones and the context's), and other channels are as without."""
    p = _params(m, dtype, hq, hkv, d, softmax_scale=1.0)
    c, _, _ = _filled(m, p, [ctx], kv, 63)
    mask = _masks(m, [n], [ctx], 14)
    q = torch.zeros((n, hq, d), device="cuda", dtype=p.torch_dtype)
    q[..., 0] = 1.0
    gen = _gen(15)
    k = torch.zeros((hkv, ctx, d), device="cuda")
    k[..., 0] = torch.randn(ctx, generator=gen, device="cuda") * 0.25
    v = torch.randn((hkv, ctx, d), generator=gen, device="cuda")
    v[..., :8] = 0
    write = lambda x: m.cache_append(p, c, k.to(p.torch_dtype), x.to(p.torch_dtype), [0, ctx], [0])  # noqa: E731
    write(v)
    clean, clean_lse = m.cache_tree_attn(p, c, q, [0, n], [ctx], mask)
    big = 3.3895313892515355e38 if dtype == "bf16" else 3.4028234663852886e38
    if kv == "e4m3":
        big = 448 * 2.0 ** 119
    large = v.clone()
    large[..., 0], large[..., 1] = big, -big
    write(large)
    got, lse = m.cache_tree_attn(p, c, q, [0, n], [ctx], mask)
    assert torch.equal(lse, clean_lse)
    # sums of up to 9000 weights in 32 bits, each rounded; 2^-8 for bf16 outputs and weights
    tol = 2.0 ** -7 if dtype == "bf16" else 1e-4
    near = lambda x, to: (x.double() / to - 1).abs() <= tol  # noqa: E731
    up, down = near(got[..., 0], big), near(got[..., 1], -big)
    if dtype == "fp32" and kv == "native":
        # A mean of N values that are the largest float, N products and sums in 32 bits: off by up to (N + 3) 2^-24 of it, and what is above the largest float
        # by half a step is infinity.  At 3e38, 12 % below it, there is room for that.
        up, down = up | (got[..., 0] == float("inf")), down | (got[..., 1] == -float("inf"))
        lower = large.clone()
        lower[..., :2] *= 3.0e38 / big
        write(lower)
        less, _ = m.cache_tree_attn(p, c, q, [0, n], [ctx], mask)
        assert bool(near(less[..., 0], 3.0e38).all()) and bool(near(less[..., 1], -3.0e38).all())
    assert bool(up.all()) and bool(down.all())
    if kv == "native":                      # (a page's scale serves all its channels)
        assert torch.equal(got[..., 8:], clean[..., 8:])


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 32, 2, 128), ("fp32", 4, 1, 64), ("bf16", 8, 2, 64)])
def test_masks_of_many_tokens(m, dtype, hq, hkv, d):  # noqa: F811
    """More drafted tokens than infllmv2_tree_masks takes, by a mask of the caller's own that is wider than they need: a window of 300 tokens and every 97th."""
    p = _params(m, dtype, hq, hkv, d)
    news, ctxs = [1500, 3], [1711, 70]
    c, _, _ = _filled(m, p, ctxs, "native", 64)
    sets = [{j for j in range(i + 1) if i - j < 300 or j % 97 == 5} for i in range(1500)] + [{0}, {0, 1}, {2}]
    mask = trees.to_words(sets, 50).cuda()
    _check(m, p, c, _q(p, news, 16), news, ctxs, mask)


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("hq,hkv,d", [(32, 2, 128), (4, 1, 64), (5, 5, 64)])
def test_all_bits_of_fp32_queries_and_weights(m, kv, hq, hkv, d):  # noqa: F811
    """Results that are what the last bits of a query or of a weight leave: where those are dropped, nothing or something else is left."""
    p = _params(m, "fp32", hq, hkv, d, softmax_scale=1.0)
    B = 40
    gen = _gen(91)
    # one key (1, 1, 0, ..): a logit of x - y, y being x without its last 8 bits
    x = torch.randn((B, hq), generator=gen, device="cuda") * 4
    y = (x.view(torch.int32) & ~0xff).view(torch.float32)
    c, _, _ = _filled(m, p, [1] * B, kv, 5)
    k = torch.zeros((hkv, B, d), device="cuda")
    k[..., 0] = k[..., d - 1] = 1.0
    m.cache_append(p, c, k, k, list(range(B + 1)), [0] * B)
    q = torch.zeros((B, hq, d), device="cuda")
    q[..., 0], q[..., d - 1] = x, -y
    mask = torch.ones((B, 1), dtype=torch.int32, device="cuda")
    _, lse = m.cache_tree_attn(p, c, q, list(range(B + 1)), [1] * B, mask)
    # (the sum is exact; times log2 e, by ln 2 back, each rounded: four roundings of 2^-24)
    want = x.double() - y.double()
    assert bool(((lse.double() - want).abs() <= 2.0 ** -21 * want.abs()).all())
    # two keys, the second's weight w = exp(-q) close to 1 / 8, their values 1 and -8: (1 - 8 w) / (1 + w)
    c, _, _ = _filled(m, p, [2] * B, kv, 6)
    k, v = (torch.zeros((hkv, 2 * B, d), device="cuda") for _ in range(2))
    k[:, 0::2, 0] = 1.0
    v[:, 0::2], v[:, 1::2] = 1.0, -8.0
    m.cache_append(p, c, k, v, list(range(0, 2 * B + 1, 2)), [0] * B)
    q = torch.zeros((B, hq, d), device="cuda")
    q[..., 0] = math.log(8) + 2.0 ** -10 * torch.rand((B, hq), generator=gen, device="cuda")
    got, _ = m.cache_tree_attn(p, c, q, list(range(B + 1)), [2] * B, mask)
    w = torch.exp(-q[..., 0].double())
    # 8 w = 1 + less than 2^-9: a logit of 3 in units of log2, rounded three times (3 x 3 x 2^-24 ln 2), its power by 2 steps (2^-22), three sums and a
    # quotient; a weight without its last 8 bits would be off by up to 2^-17
    assert bool(((got.double() - ((1 - 8 * w) / (1 + w))[..., None]).abs() <= 2.0 ** -20).all())


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("dtype,hq,hkv,d", [("fp32", 8, 2, 128), ("fp32", 4, 1, 64), ("bf16", 32, 2, 128)])
def test_queries_that_are_not_finite(m, kv, dtype, hq, hkv, d):  # noqa: F811
    """They give NaN (of keys seen) and leave other rows and heads as they are."""
    p = _params(m, dtype, hq, hkv, d)
    n, ctx = 12, 700
    c, _, _ = _filled(m, p, [ctx], kv, 7)
    mask, q = _masks(m, [n], [ctx], 15), _q(p, [n], 16)
    want, want_lse = m.cache_tree_attn(p, c, q, [0, n], [ctx], mask)
    odd = q.clone()
    bad = torch.zeros((n, hq), dtype=torch.bool)
    for t, h, ch, x in ((0, 1, 3, float("inf")), (4, 0, d - 1, -float("inf")), (5, hq - 1, 17, float("nan")), (11, 2, 40, float("inf"))):
        odd[t, h, ch] = x
        bad[t, h] = True
    if dtype == "fp32":
        odd.view(torch.int32)[7, 3, 9] = 0x7f800001          # a NaN of low bits only
        bad[7, 3] = True
    got, lse = m.cache_tree_attn(p, c, odd, [0, n], [ctx], mask)
    bad = bad.cuda()
    assert bool(got[bad].isnan().all())
    assert torch.equal(got[~bad], want[~bad]) and torch.equal(lse[~bad], want_lse[~bad])
