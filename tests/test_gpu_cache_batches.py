"""Batches of the paged cache with more sequences than a search looks at in one step (64), ragged ones, pages that are not there, and steps in flight together."""
import pytest
import torch

import paged
from test_gpu_cache import _cache, _filled, _gen, _params, _same, m  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("batch,long", [(66, 0), (128, 65), (150, 149), (150, 63)])
@pytest.mark.parametrize("dtype,hkv,d", [("bf16", 2, 128), ("fp32", 1, 64)])
def test_compressed_keys_of_ragged_batches(m, kv, batch, long, dtype, hkv, d):  # noqa: F811
    """One long prompt among sequences that have grown by a row, by several, by none: what each of them alone gives, bit for bit."""
    p = _params(m, dtype, hkv, hkv, d)
    ctxs = [9001 if b == long else 40 + b % 300 for b in range(batch)]
    prevs = [0 if b == long else max(0, c - (1, 17, 300)[b % 3]) for b, c in enumerate(ctxs)]
    c, _, _ = _filled(m, p, ctxs, kv, 3)
    rows = m.num_cmp(p, 9001)
    kc = torch.full((batch, hkv, rows, d), 9.0, device="cuda")
    m.cache_compress_k(p, c, kc, prevs, ctxs)
    for b in sorted({0, 1, 62, 63, 64, 65, batch - 2, batch - 1, long}):
        one = torch.full((1, hkv, rows, d), 9.0, device="cuda")
        sc = (c.k_scale, c.v_scale) if kv == "e4m3" else (None, None)
        m.cache_compress_k(p, m.PagedCache(p, c.k, c.v, c.page_table[b:b + 1], *sc), one, [prevs[b]], [ctxs[b]])
        assert torch.equal(one[0], kc[b]), b
        x, _ = paged.rows_of(c.k, c.k_scale, c.page_table, b, ctxs[b], 0)
        for i in range(m.num_cmp(p, prevs[b]), m.num_cmp(p, ctxs[b])):      # (a sum of 32 values of at most 6, rounded 32 times)
            assert float((kc[b, 0, i].double() - x[i * 16:i * 16 + 32].mean(0)).abs().max()) <= 32 * 6 * 2.0 ** -24 + 2.0 ** -22
    fresh = sum(m.num_cmp(p, a) - m.num_cmp(p, b) for a, b in zip(ctxs, prevs))
    assert int((kc[..., 0] != 9.0).sum()) == fresh * hkv    # nothing else is written


def test_compressed_keys_of_more_heads_than_a_grid_is_wide(m):  # noqa: F811
    """70000 sequences of 8 heads that share a page."""
    p = _params(m, "bf16", 8, 8, 64)
    c, _, _ = _filled(m, p, [32], "e4m3", 3)
    c = m.PagedCache(p, c.k, c.v, c.page_table[:, :1].repeat(70000, 1), c.k_scale, c.v_scale)
    kc = torch.zeros((70000, 8, 1, 64), device="cuda")
    m.cache_compress_k(p, c, kc, [0] * 70000, [32] * 70000)
    want = torch.zeros((1, 8, 1, 64), device="cuda")
    m.cache_compress_k(p, m.PagedCache(p, c.k, c.v, c.page_table[:1], c.k_scale, c.v_scale), want, [0], [32])
    assert bool((want != 0).all()) and torch.equal(kc, want.expand_as(kc))


def _cu(news):
    cu = [0]
    for n in news:
        cu.append(cu[-1] + n)
    return cu


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("batch", [65, 128, 150])
def test_append_to_many_sequences(m, kv, batch):  # noqa: F811
    """Ragged appends over several pages each, sequences without new tokens in between."""
    p = _params(m, "bf16", 2, 2, 64)
    news = [(0, 1, 70, 64, 200, 3)[b % 6] for b in range(batch)]
    prevs = [(b * 37) % 190 for b in range(batch)]
    c = _cache(m, p, [a + b for a, b in zip(news, prevs)], kv, 5)
    if kv == "e4m3":                    # what continued pages hold: zeros in a small scale
        for x in (c.k, c.v):
            x.view(torch.uint8).zero_()
        c.k_scale.fill_(2.0 ** -100), c.v_scale.fill_(2.0 ** -100)
    k, v = c.k.clone(), c.v.clone()
    sc = (c.k_scale.clone(), c.v_scale.clone()) if kv == "e4m3" else None
    gen = _gen(batch)
    nk, nv = (torch.randn((2, sum(news), 64), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    paged.append(k, v, sc, nk.double(), nv.double(), c.page_table, news, prevs)
    m.cache_append(p, c, nk, nv, _cu(news), prevs)
    assert _same(c.k, k) and _same(c.v, v)
    if sc is not None:
        assert torch.equal(c.k_scale, sc[0]) and torch.equal(c.v_scale, sc[1])


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 32, 2, 128), ("fp32", 4, 1, 64)])
@pytest.mark.parametrize("batch,form", [(65, "one"), (65, "few"), (130, "few"), (150, "few"), (130, "lists"), (150, "chunk")])
def test_attention_of_many_sequences(m, kv, dtype, hq, hkv, d, batch, form):  # noqa: F811
    """Ragged batches whose workgroups, splits and tiles belong to sequences behind the first 64: what each sequence gives alone, up to the order of its sums, and
    (some of them) the definition's."""
    p = _params(m, dtype, hq, hkv, d, topk_total=40, dense_threshold=0)
    ctxs = [100 + (b * 911) % 1500 for b in range(batch)]
    for b in (batch - 1, batch - 2, 63, 64):
        ctxs[b] = 9000 + b             # several splits
    news = {"one": [1] * batch, "lists": [1] * batch, "few": [(1, 3, 0, 2)[b % 4] for b in range(batch)], "chunk": [(1, 0, 2)[b % 3] for b in range(batch)]}[form]
    if form == "chunk":
        news[batch - 1], news[64] = 150, 200
    c, _, _ = _filled(m, p, ctxs, kv, 7)
    q = torch.randn((sum(news), hq, d), generator=_gen(8), device="cuda").to(p.torch_dtype)
    cu = _cu(news)
    blocks = None
    if form == "lists":
        blocks = torch.full((batch, hkv, 40), -1, dtype=torch.int32)
        gen = torch.Generator().manual_seed(3)
        for b, n in enumerate(ctxs):
            for h in range(hkv):
                x = torch.randperm((n + 63) // 64, generator=gen)[:40].sort().values
                blocks[b, h, :len(x)] = x.to(torch.int32)
        blocks = blocks.cuda()
    out, lse = m.cache_attn(p, c, q, cu, ctxs, blocks)
    sc = None if kv == "native" else (c.k_scale, c.v_scale)
    tiles = dtype == "bf16" and form == "chunk"
    for b in sorted({0, 1, 62, 63, 64, 65, 66, batch - 2, batch - 1}):
        if b >= batch or news[b] == 0:
            continue
        rows, one = slice(cu[b], cu[b + 1]), (lambda x: None if x is None else x[cu[b]:cu[b + 1]])
        alone = m.PagedCache(p, c.k, c.v, c.page_table[b:b + 1], *(sc or (None, None)))
        o, s = m.cache_attn(p, alone, q[rows], [0, news[b]], [ctxs[b]], one(blocks))
        want, want_lse, mass = paged.attention(q[rows][-3:], c.k, c.v, sc, c.page_table[b:b + 1], [min(3, news[b])], [ctxs[b]], p.softmax_scale, one(blocks))
        # as in test_gpu_cache.py: the result's own rounding; weights of 16 bits and logits and sums in 32 2^-12 of |v| <= 6; chunks' weights of 8 bits 2^-8 of the sum of
        # p |v|.  The two results are each within that of the definition's.
        rough = 2.0 ** -8 if tiles and news[b] > 8 else 0.0
        tol = 2.0 ** -8 * want.abs() + 6 * 2.0 ** -12 + rough * mass if dtype == "bf16" else torch.full_like(want, 1e-4)
        assert bool(((out[rows][-3:].double() - want).abs() <= tol).all()), b
        assert float((lse[rows][-3:].double() - want_lse).abs().max()) <= 1e-4
        both = 2.0 ** -7 * o.double().abs() + 13 * 2.0 ** -12 + 2 * rough * 6 if dtype == "bf16" else torch.full_like(o.double(), 2e-4)
        assert bool(((out[rows].double() - o.double()).abs() <= both).all()), b
        assert float((lse[rows] - s).abs().max()) <= 2e-4


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("window", [(32, 16), (150, 40)])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp32", 64)])
def test_compressed_keys_with_pages_that_are_not_there(m, kv, window, dtype, d):  # noqa: F811
    """Entries outside the pages at the front, in the middle and at the end of windows: their tokens count as 0.  Page 0, whose address stands in for them, holds NaN."""
    p = _params(m, dtype, 2, 2, d, cmp_len=window[0], cmp_stride=window[1])
    ctxs = [1000, 640, 333]
    c, _, _ = _filled(m, p, ctxs, kv, 9)
    pages = c.k.shape[0]
    spare = torch.where(c.page_table == 0, pages - 1, c.page_table)          # (page 0 is nobody's)
    c.k[pages - 1].copy_(c.k[0]) if kv == "native" else c.k.view(torch.uint8)[pages - 1].copy_(c.k.view(torch.uint8)[0])
    if kv == "e4m3":
        c.k_scale[pages - 1] = c.k_scale[0]
        c.k.view(torch.uint8)[0] = 0x7f
        c.k_scale[0] = float("nan")
    else:
        c.k[0] = float("nan")
    c.page_table.copy_(spare)
    for b, j, e in ((0, 0, -1), (0, 3, pages), (0, 4, -(1 << 31)), (0, 15, 1 << 30), (1, 1, -1), (1, 2, -1), (1, 9, pages + 7), (2, 5, -1)):
        c.page_table[b, j] = e
    rows = m.num_cmp(p, 1000)
    kc = torch.full((3, 2, rows, d), 9.0, device="cuda")
    m.cache_compress_k(p, c, kc, [0, 0, 0], ctxs)
    for b, n in enumerate(ctxs):
        for h in range(2):
            x, _ = paged.rows_of(c.k, c.k_scale, c.page_table, b, n, h)
            for i in range(m.num_cmp(p, n)):
                want = x[i * window[1]:i * window[1] + window[0]].mean(0)
                assert float((kc[b, h, i].double() - want).abs().max()) <= window[0] * 6 * 2.0 ** -24 + 2.0 ** -22
            assert bool((kc[b, h, m.num_cmp(p, n):] == 9.0).all())


def test_steps_in_flight_together(m):  # noqa: F811
    """Two captured steps replayed on two streams and an eager step on a third, all at once, each with its own cache, outputs and scratch: what they give one after the
    other.  Long contexts and a chunk, so that splits and tiles of different calls share the chip."""
    p = _params(m, "bf16", 32, 2, 128)
    ctxs, prevs, news = [30000, 9000, 500], [29850, 8999, 498], [150, 1, 2]
    rot = m.Rotary(m.rotary_turns(128), 128)
    cu, pv, cx = m.SeqInfo(_cu(news)), m.DecodeInfo(prevs), m.DecodeInfo(ctxs)
    T = sum(news)

    def make(seed):
        c, _, _ = _filled(m, p, ctxs, "e4m3", seed)
        gen = _gen(seed)
        s = dict(c=c, k=torch.randn((2, T, 128), generator=gen, device="cuda").to(torch.bfloat16), q=torch.randn((T, 32, 128), generator=gen, device="cuda").to(torch.bfloat16),
                 out=torch.zeros((T, 32, 128), dtype=torch.bfloat16, device="cuda"), lse=torch.zeros((T, 32), device="cuda"),
                 kc=torch.zeros((3, 2, m.num_cmp(p, 30000), 128), device="cuda"),
                 ws=torch.empty(m.workspace_bytes(m.OP_CACHE_ATTN, p, 3, T, 30000), dtype=torch.uint8, device="cuda"))
        s["pages"] = [s["c"].k.view(torch.uint8), s["c"].v.view(torch.uint8), s["c"].k_scale, s["c"].v_scale]
        s["start"] = [x.clone() for x in s["pages"]]
        return s

    def step(s):
        m.cache_append(p, s["c"], s["k"], s["k"], cu, pv, rot)
        m.cache_compress_k(p, s["c"], s["kc"], pv, cx)
        m.cache_attn(p, s["c"], s["q"], cu, cx, out=s["out"], lse=s["lse"], workspace=s["ws"])

    def reset(s):
        for x, y in zip(s["pages"], s["start"]):
            x.copy_(y)
        for x in ("out", "lse", "kc"):
            s[x].zero_()

    steps = [make(seed) for seed in (1, 2, 3)]
    want = []
    for s in steps:
        step(s)
        torch.cuda.synchronize()
        want.append([s[x].clone() for x in ("out", "lse", "kc")] + [x.clone() for x in s["pages"]])
        reset(s)
    streams, graphs = [torch.cuda.Stream() for _ in steps], []
    torch.cuda.synchronize()
    for s in steps[:2]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(s)
        graphs.append(g)
    for _ in range(4):
        for s in steps:
            reset(s)
        torch.cuda.synchronize()
        for g, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                g.replay()
        with torch.cuda.stream(streams[2]):
            step(steps[2])
        torch.cuda.synchronize()
        for s, w in zip(steps, want):
            assert all(torch.equal(x, y) for x, y in zip([s["out"], s["lse"], s["kc"]] + s["pages"], w))
