"""The paged cache: appends (rotated keys, two stores), compressed keys, attention over the pages, each against a plain form in 64 bits."""
import math

import pytest
import torch

import paged
from paged import PAGE

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def m():
    import paper_2509_24663_amd as m
    m.lib()
    return m


def _params(m, dtype, hq, hkv, d, **over):
    kw = dict(n_init=1, n_local=2, topk_total=8)
    kw.update(over)
    return m.Params.make(dtype, hq, hkv, d, **kw)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _cache(m, p, lens, kv, seed=0, layout="heads", spare=3):
    """an empty cache over junk: what nobody wrote must not matter"""
    table, pages = paged.pages_for(lens, spare, seed)
    shape = (pages, p.num_kv_heads, PAGE, p.head_dim)
    dtype = torch.float8_e4m3fn if kv == "e4m3" else p.torch_dtype
    if layout == "tokens":
        make = lambda: torch.empty((pages, PAGE, p.num_kv_heads, p.head_dim), dtype=dtype, device="cuda").transpose(1, 2)  # noqa: E731
    else:
        make = lambda: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    k, v = make(), make()
    for x in (k, v):
        x.view(torch.uint8 if kv == "e4m3" else dtype).fill_(0x7f if kv == "e4m3" else float("nan"))       # NaN
    sc = [torch.full((pages, p.num_kv_heads), 2.0 ** 100, device="cuda") for _ in range(2)] if kv == "e4m3" else [None, None]
    return m.PagedCache(p, k, v, table, *sc)


def _same(a, b):
    """equal bits, any NaN equal to any NaN"""
    if a.dtype == torch.float8_e4m3fn:
        a, b = a.float(), b.float()
    return bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all())


# ------------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("dtype,hkv,d,layout", [("bf16", 2, 128, "heads"), ("bf16", 3, 64, "tokens"), ("fp32", 1, 64, "heads"), ("fp32", 2, 128, "tokens")])
def test_append_steps(m, kv, dtype, hkv, d, layout):
    """Three appends: prompts, one token each, ragged continuations; magnitudes grow, so scales of continued pages do too."""
    p = _params(m, dtype, hkv, hkv, d)
    steps = [[130, 0, 1, 64, 63, 200], [1, 1, 1, 1, 1, 1], [7, 66, 0, 129, 1, 3]]
    lens = [sum(s[b] for s in steps) for b in range(6)]
    c = _cache(m, p, lens, kv, 5, layout)
    k, v = c.k.clone(), c.v.clone()
    sc = (c.k_scale.clone(), c.v_scale.clone()) if kv == "e4m3" else None
    prevs, gen = [0] * 6, _gen(11)
    for i, news in enumerate(steps):
        T = sum(news)
        size = 4.0 ** i * torch.exp2(torch.randint(-3, 4, (hkv, T, 1), generator=gen, device="cuda").float())
        nk, nv = ((torch.randn((hkv, T, d), generator=gen, device="cuda") * size).to(p.torch_dtype) for _ in range(2))
        if layout == "tokens":         # token-major new rows as well
            nk, nv = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (nk, nv))
        cu = [0]
        for n in news:
            cu.append(cu[-1] + n)
        paged.append(k, v, sc, nk.double(), nv.double(), c.page_table, news, prevs)
        m.cache_append(p, c, nk, nv, cu, prevs)
        assert _same(c.k, k) and _same(c.v, v), f"step {i}"
        if sc is not None:
            assert torch.equal(c.k_scale, sc[0]) and torch.equal(c.v_scale, sc[1])
        prevs = [a + b for a, b in zip(prevs, news)]


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("dtype,d,rot_dim,interleaved,given", [
    ("bf16", 128, 128, False, False), ("bf16", 128, 104, True, True), ("bf16", 64, 50, False, False), ("fp32", 64, 32, True, False),
    ("fp32", 128, 20, False, True)])
def test_append_turns_keys(m, kv, dtype, d, rot_dim, interleaved, given):
    hkv, news, prevs = 2, [100, 1, 70], [0, 64, 30]
    p = _params(m, dtype, hkv, hkv, d)
    layout = "interleaved" if interleaved else "half"
    rot = m.Rotary(m.rotary_turns(rot_dim, 5000.0), rot_dim, layout, 1.1)
    c = _cache(m, p, [a + b for a, b in zip(news, prevs)], kv, 1)
    T, gen = sum(news), _gen(2)
    nk, nv = (torch.randn((hkv, T, d), generator=gen, device="cuda").to(p.torch_dtype) for _ in range(2))
    own = torch.cat([torch.arange(a, a + n) for n, a in zip(news, prevs)]).to(torch.int32).cuda()
    pos = torch.randint(0, 1 << 20, (T,), generator=gen, device="cuda", dtype=torch.int32) if given else own
    if kv == "e4m3":          # what the continued page holds: zeros, in a small scale
        c.k.view(torch.uint8).zero_(), c.v.view(torch.uint8).zero_(), c.k_scale.fill_(2.0 ** -100), c.v_scale.fill_(2.0 ** -100)
    m.cache_append(p, c, nk, nv, [0, 100, 101, 171], prevs, rot, pos if given else None)
    want = paged.turned(nk.transpose(0, 1), pos, paged.frequencies(rot_dim, 5000.0), layout, 1.1).transpose(0, 1)
    t = 0
    for b, (n, a) in enumerate(zip(news, prevs)):
        for h in range(hkv):
            got, there = paged.rows_of(c.k, c.k_scale, c.page_table, b, a + n, h)
            x = want[h, t:t + n]
            if kv == "native":
                tol = 2.0 ** -8 * x.abs() + 6e-6 if dtype == "bf16" else torch.full_like(x, 6e-6)
            else:             # half a step of a 3-bit mantissa; among subnormals half of 2^-9 scales; and the turned key's own 6e-6
                s = torch.stack([c.k_scale[c.page_table[b, u // PAGE], h] for u in range(a, a + n)]).double()[:, None]
                tol = torch.maximum(2.0 ** -4 * x.abs(), 2.0 ** -10 * s) + 6e-6
            assert bool(((got[a:] - x).abs() <= tol).all())
            vals, _ = paged.rows_of(c.v, c.v_scale, c.page_table, b, a + n, h)
            if kv == "native":
                assert torch.equal(vals[a:], nv[h, t:t + n].double())
        t += n


def test_append_odd_values(m):
    """zeros, infinities and NaN, the largest and the smallest numbers"""
    p = _params(m, "fp32", 1, 1, 64)
    c = _cache(m, p, [4 * 64], "e4m3")
    x = torch.zeros((1, 256, 64), device="cuda")
    x[0, 64:128] = torch.randn((64, 64), generator=_gen(1), device="cuda")
    x[0, 70, 3], x[0, 71, 5], x[0, 72, 7] = float("nan"), float("inf"), -float("inf")
    x[0, 128:192, :] = 3.4e38
    x[0, 192:, :] = 1e-37
    x[0, 192, 0] = 1e-30
    k, v, sc = c.k.clone(), c.v.clone(), (c.k_scale.clone(), c.v_scale.clone())
    m.cache_append(p, c, x, x, [0, 256], [0])
    paged.append(k, v, sc, x.double(), x.double(), c.page_table, [256], [0])
    assert torch.equal(c.k_scale, sc[0]) and _same(c.k, k) and _same(c.v, v)
    rows, _ = paged.rows_of(c.k, c.k_scale, c.page_table, 0, 256, 0)
    assert bool((rows[:64] == 0).all()) and bool(torch.isnan(rows[70, 3] + rows[71, 5] + rows[72, 7]))
    assert int(torch.isnan(rows).sum()) == 3 and float(rows[130, 0]) == 448 * 2.0 ** 119


def test_append_leaves_the_rest(m):
    """Pages that are not there, rows of other tokens, spare pages; a sequence without new tokens."""
    p = _params(m, "bf16", 2, 2, 64)
    c = _cache(m, p, [200, 100, 64], "native", 9)
    c.page_table[0, 1], c.page_table[0, 2] = -1, 1 << 20
    before = c.k.clone()
    x = torch.ones((2, 215, 64), dtype=torch.bfloat16, device="cuda")
    m.cache_append(p, c, x, x, [0, 200, 215, 215], [0, 70, 64])
    touched = torch.zeros(c.k.shape[0], dtype=torch.bool, device="cuda")
    touched[c.page_table[0, 0].long()] = touched[c.page_table[0, 3].long()] = touched[c.page_table[1, 1].long()] = True
    assert _same(c.k[~touched], before[~touched])
    a, b, d = int(c.page_table[0, 0]), int(c.page_table[0, 3]), int(c.page_table[1, 1])
    assert bool((c.k[a] == 1).all()) and bool((c.k[b, :, :8] == 1).all()) and bool(torch.isnan(c.k[b, :, 8:]).all())
    assert bool((c.k[d, :, 6:21] == 1).all()) and bool(torch.isnan(c.k[d, :, :6]).all()) and bool(torch.isnan(c.k[d, :, 21:]).all())


# ------------------------------------------------------------------------------------------------ compressed keys
def _filled(m, p, lens, kv, seed=0, layout="heads"):
    c = _cache(m, p, lens, kv, seed, layout)
    gen = _gen(seed + 100)
    T = sum(lens)
    k, v = (torch.randn((p.num_kv_heads, T, p.head_dim), generator=gen, device="cuda").to(p.torch_dtype) for _ in range(2))
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    m.cache_append(p, c, k, v, cu, [0] * len(lens))
    return c, k, v


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("dtype,hkv,d,window", [("bf16", 2, 128, (32, 16)), ("fp32", 1, 64, (32, 16)), ("bf16", 2, 64, (7, 3)), ("fp32", 2, 128, (150, 40))])
def test_compressed_keys(m, kv, dtype, hkv, d, window):
    p = _params(m, dtype, hkv, hkv, d, cmp_len=window[0], cmp_stride=window[1])
    ctxs, prevs = [700, 33, 31, 64, 500], [0, 17, 0, 63, 480]
    c, k, _ = _filled(m, p, ctxs, kv, 3, "tokens")
    rows = max(max(m.num_cmp(p, n) for n in ctxs), 1)
    kc = torch.full((5, hkv, rows, d), 9.0, device="cuda")
    m.cache_compress_k(p, c, kc, prevs, ctxs)
    for b, (n, a) in enumerate(zip(ctxs, prevs)):
        for h in range(hkv):
            x, _ = paged.rows_of(c.k, c.k_scale, c.page_table, b, n, h)
            want = torch.full((rows, d), 9.0, dtype=torch.float64, device="cuda")
            for i in range(m.num_cmp(p, a), m.num_cmp(p, n)):
                want[i] = x[i * window[1]:i * window[1] + window[0]].mean(0)
            # a sum of l values of at most 6, rounded l times
            assert float((kc[b, h].double() - want).abs().max()) <= window[0] * 6 * 2.0 ** -24 + 2.0 ** -22
    if kv == "native":        # the same bits as from planes
        plane = torch.zeros((5, hkv, 700, d), dtype=p.torch_dtype, device="cuda")
        t = 0
        for b, n in enumerate(ctxs):
            plane[b, :, :n] = k[:, t:t + n]
            t += n
        ref = torch.full_like(kc, 9.0)
        m.compress_k_append(p, plane, ref, prevs, ctxs)
        assert torch.equal(ref, kc)


# ------------------------------------------------------------------------------------------------ attention
def _check_attn(m, p, c, q, news, ctxs, blocks=None, **kw):
    cu = [0]
    for n in news:
        cu.append(cu[-1] + n)
    out, lse = m.cache_attn(p, c, q, cu, ctxs, blocks, **kw)
    sc = None if c.k_scale is None else (c.k_scale, c.v_scale)
    want, want_lse, mass = paged.attention(q, c.k, c.v, sc, c.page_table, news, ctxs, p.softmax_scale, blocks, p.dense_threshold)
    # the result's own rounding; weights of 16 bits and more, logits in 32: 2^-12 (bf16) and 1e-4 (fp32, as elsewhere) of |v| <= 6
    tol = 2.0 ** -8 * want.abs() + 6 * 2.0 ** -12 if q.dtype == torch.bfloat16 else torch.full_like(want, 1e-4)
    if q.dtype == torch.bfloat16 and max(news) > 8:
        # chunks of prompts: weights p rounded to bf16 in front of the second product, p (1 + e) with |e| <= 2^-8, so the sum of p v is off by at most
        # 2^-8 times the sum of p |v|
        many = torch.tensor([n > 8 for n in news for _ in range(n)], device="cuda")
        tol = tol + 2.0 ** -8 * mass * many[:, None, None]
    bad = ~((out.double() - want).abs() <= tol)
    assert not bool(bad.any()), (torch.nonzero(bad)[:4].tolist(), float((out.double() - want).abs().max()))
    none = torch.isinf(want_lse)
    assert torch.equal(none, torch.isinf(lse)) and bool((out[none] == 0).all())
    assert float((lse.double() - want_lse)[~none].abs().max() if bool((~none).any()) else 0) <= 1e-4
    return out, lse


SHAPES = [("bf16", 32, 2, 128), ("bf16", 8, 2, 64), ("bf16", 12, 4, 128), ("bf16", 5, 5, 64), ("fp32", 4, 1, 64), ("fp32", 6, 2, 128), ("bf16", 16, 1, 64)]


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
def test_attention_lengths(m, kv, dtype, hq, hkv, d):
    """One token to a chunk for each sequence, contexts around page ends, sequences without queries."""
    p = _params(m, dtype, hq, hkv, d)
    news, ctxs = [1, 1, 1, 1, 3, 0, 17, 64, 5], [1, 63, 64, 65, 130, 50, 17, 200, 1000]
    c, _, _ = _filled(m, p, ctxs, kv, 21, "tokens" if d == 64 else "heads")
    q = torch.randn((sum(news), hq, d), generator=_gen(5), device="cuda").to(p.torch_dtype)
    _check_attn(m, p, c, q, news, ctxs)
    one = [0 if n == 0 else 1 for n in news]
    _check_attn(m, p, c, q[:sum(one)].contiguous(), one, ctxs)


def _lists(p, news, ctxs, seed, topk):
    gen = torch.Generator().manual_seed(seed)
    rows = []
    for n, L in zip(news, ctxs):
        for i in range(n):
            bt = (L - n + i) // PAGE
            per = []
            for _ in range(p.num_kv_heads):
                k = int(torch.randint(0, topk + 1, (1,), generator=gen))            # empty lists among them
                x = torch.randperm(bt + 1, generator=gen)[:k].sort().values.tolist()
                per.append(x + [-1] * (topk - len(x)))
            rows.append(per)
    return torch.tensor(rows, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
def test_attention_over_lists(m, kv, dtype, hq, hkv, d):
    """Listed blocks, empty lists, a dense sequence among them, entries that no token may see, pages that are not there."""
    p = _params(m, dtype, hq, hkv, d, topk_total=8, dense_threshold=100)
    news, ctxs = [1, 1, 4, 1, 2], [1500, 99, 700, 100, 64]
    c, _, _ = _filled(m, p, ctxs, kv, 31)
    blocks = _lists(p, news, ctxs, 3, 8)
    blocks[0, 0, :] = torch.tensor([23, 2, -7, 24, 1 << 30, 0, 9, -1], dtype=torch.int32)      # any order, some outside
    blocks[3, :, :] = -1
    c.page_table[0, 2], c.page_table[2, 0], c.page_table[1, 1] = -1, c.k.shape[0], -(1 << 31)
    q = torch.randn((sum(news), hq, d), generator=_gen(6), device="cuda").to(p.torch_dtype)
    _check_attn(m, p, c, q, news, ctxs, blocks)
    _check_attn(m, p, c, q, news, ctxs)


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 32, 2, 128), ("fp32", 4, 1, 64)])
@pytest.mark.parametrize("topk,ctxs", [(24, [130, 64, 1, 900]), (600, [700, 1, 5000, 20000])])
def test_lists_longer_than_the_pages(m, kv, dtype, hq, hkv, d, topk, ctxs):
    """A list's blocks may stand anywhere in it, also where it has more entries than the sequence has blocks."""
    p = _params(m, dtype, hq, hkv, d, topk_total=topk)
    c, _, _ = _filled(m, p, ctxs, kv, 33)
    gen = torch.Generator().manual_seed(topk)
    for news in ([1] * 4, [1, 1, 0, 7]):
        blocks = torch.full((sum(news), hkv, topk), -1, dtype=torch.int32)
        row = 0
        for n, L in zip(news, ctxs):
            for i in range(n):
                own = (L - n + i) // PAGE
                for h in range(hkv):
                    here = torch.randperm(own + 1, generator=gen)[:topk - 3].to(torch.int32)
                    here = torch.cat([here[:len(here) - len(here) // 3], torch.tensor([own + 1, 1 << 30, -5], dtype=torch.int32)])
                    blocks[row, h, torch.randperm(topk, generator=gen)[:len(here)]] = here
                    blocks[row, h, topk - 1], last = here[0], blocks[row, h, topk - 1].clone()       # (one of them last of all)
                    blocks[row, h, :topk - 1][blocks[row, h, :topk - 1] == here[0]] = last
                row += 1
        q = torch.randn((sum(news), hq, d), generator=_gen(16), device="cuda").to(p.torch_dtype)
        _check_attn(m, p, c, q, news, ctxs, blocks.cuda())


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("dtype,hq,hkv,d,news,ctxs", [
    ("bf16", 32, 2, 128, [1], [9001]), ("bf16", 8, 2, 64, [1, 2], [5000, 20000]), ("fp32", 4, 1, 64, [1, 1], [6000, 130]),
    ("bf16", 32, 2, 128, [150], [3000]), ("bf16", 16, 2, 128, [40, 1, 333, 1], [40, 2000, 700, 1]), ("bf16", 8, 2, 64, [700], [1100])])
def test_attention_long(m, kv, dtype, hq, hkv, d, news, ctxs):
    """Splits along the keys, chunks of prompts beside single tokens."""
    p = _params(m, dtype, hq, hkv, d)
    c, _, _ = _filled(m, p, ctxs, kv, 41)
    q = torch.randn((sum(news), hq, d), generator=_gen(8), device="cuda").to(p.torch_dtype) * 2
    _check_attn(m, p, c, q, news, ctxs)


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 32, 2, 128), ("bf16", 8, 2, 64), ("fp32", 4, 2, 64)])
@pytest.mark.parametrize("n", [9, 150])
def test_values_that_are_not_finite(m, kv, dtype, hq, hkv, d, n):
    """Rows of later tokens and of no token at all hold infinities and NaN: tokens that do not see them are as if they did not."""
    p = _params(m, dtype, hq, hkv, d)
    ctxs, news = [300 + n, 70 + n, n], [n] * 3
    c, _, _ = _filled(m, p, ctxs, kv, 51)
    q = torch.randn((3 * n, hq, d), generator=_gen(9), device="cuda").to(p.torch_dtype)
    clean, clean_lse = _check_attn(m, p, c, q, news, ctxs)
    for b, L in enumerate(ctxs):         # the last three tokens' rows
        for t in range(L - 3, L):
            page = int(c.page_table[b, t // PAGE])
            for x in (c.k, c.v):
                if kv == "e4m3":
                    x.view(torch.uint8)[page, :, t % PAGE] = 0xff
                else:
                    x[page, :, t % PAGE] = float("inf") if t % 2 else float("nan")
    out, lse = m.cache_attn(p, c, q, [0, n, 2 * n, 3 * n], ctxs)
    for b in range(3):
        a = slice(b * n, (b + 1) * n - 3)
        assert torch.equal(out[a], clean[a]) and torch.equal(lse[a], clean_lse[a])
        assert bool(torch.isnan(out[(b + 1) * n - 1]).all())
    # queries that are not finite: their own rows alone
    q2 = q.clone()
    q2[n - 5] = float("inf")
    out2, _ = m.cache_attn(p, c, q2, [0, n, 2 * n, 3 * n], ctxs)
    keep = [i for i in range(3 * n) if i != n - 5]
    assert bool(torch.isnan(out2[n - 5]).all()) and _same(out2[keep], out[keep])


def test_only_logits_of_minus_infinity(m):
    """A softmax over them is 0 / 0; that is not the same as a token without keys."""
    p = _params(m, "bf16", 2, 2, 64)
    c, _, _ = _filled(m, p, [100], "native", 1)
    c.k.fill_(1.0)
    q = torch.full((1, 2, 64), -float("inf"), dtype=torch.bfloat16, device="cuda")
    out, _ = m.cache_attn(p, c, q, [0, 1], [100])
    assert bool(torch.isnan(out).all())


def test_rows_of_far_pages(m):
    """Pages whose byte offsets pass 32 bits, in the cache and in the strides; scales far apart from page to page."""
    p = _params(m, "bf16", 32, 2, 128)
    pages = (1 << 32) // (2 * PAGE * 128) + 5
    table = torch.tensor([[pages - 1, 2, pages - 3, 0]], dtype=torch.int32, device="cuda")
    c = m.PagedCache.empty(p, pages, table)
    gen = _gen(3)
    k = torch.randn((2, 250, 128), generator=gen, device="cuda").to(torch.bfloat16)
    v = k.flip(1).contiguous()
    v[:, 64:128] *= 2.0 ** -60
    m.cache_append(p, c, k, v, [0, 250], [0])
    q = torch.randn((1, 32, 128), generator=gen, device="cuda").to(torch.bfloat16)
    _check_attn(m, p, c, q, [1], [250])


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 32, 2, 128), ("bf16", 8, 2, 64), ("fp32", 4, 1, 64)])
def test_steps_as_with_planes(m, dtype, hq, hkv, d):
    """Prompts and five decode steps over pages in the data's type: turned keys, compressed keys and block lists are those of the planes, bit for
    bit, and the attention is that of infllmv2_sparse_decode up to rounding; over codes it is that of the codes' values."""
    p = _params(m, dtype, hq, hkv, d, topk_total=6, dense_threshold=150)
    prompts, steps = [1000, 100, 640, 149], 5
    B, room = len(prompts), max(prompts) + steps
    lens = [n + steps for n in prompts]
    gen = _gen(77)
    rot = m.Rotary(m.rotary_turns(d // 2), d // 2)
    caches = {kv: _cache(m, p, lens, kv, 61) for kv in ("native", "e4m3")}
    kp, vp = (torch.zeros((B, hkv, room, d), dtype=p.torch_dtype, device="cuda") for _ in range(2))
    nc = max(m.num_cmp(p, room), 1)
    kcs = {name: torch.zeros((B, hkv, nc, d), device="cuda") for name in ("planes", "native", "e4m3")}
    prev = [0] * B
    for step in range(steps + 1):
        news = prompts if step == 0 else [1] * B
        ctx = [a + b for a, b in zip(prev, news)]
        cu = [0]
        for n in news:
            cu.append(cu[-1] + n)
        T = cu[-1]
        k, v = (torch.randn((hkv, T, d), generator=gen, device="cuda").to(p.torch_dtype) for _ in range(2))
        pos = torch.cat([torch.arange(a, a + n) for a, n in zip(prev, news)]).to(torch.int32).cuda()
        kr = m.rotary_fwd(p, rot, k.transpose(0, 1), pos).transpose(0, 1)
        for b in range(B):
            kp[b, :, prev[b]:ctx[b]], vp[b, :, prev[b]:ctx[b]] = kr[:, cu[b]:cu[b + 1]], v[:, cu[b]:cu[b + 1]]
        m.compress_k_append(p, kp, kcs["planes"], prev, ctx)
        for kv, c in caches.items():
            m.cache_append(p, c, k, v, cu, prev, rot)
            m.cache_compress_k(p, c, kcs[kv], prev, ctx)
        for b in range(B):
            rows, _ = paged.rows_of(caches["native"].k, None, caches["native"].page_table, b, ctx[b], 0)
            assert torch.equal(rows.to(p.torch_dtype), kp[b, 0, :ctx[b]])
        assert torch.equal(kcs["planes"], kcs["native"])
        q = m.rotary_fwd(p, rot, torch.randn((B, hq, d), generator=gen, device="cuda").to(p.torch_dtype),
                         torch.tensor([x - 1 for x in ctx], dtype=torch.int32, device="cuda"))
        want, want_lse, want_idx = m.sparse_decode(p, q, kp, vp, kcs["planes"], ctx)
        idx = m.decode_blocks(p, q, kcs["native"], ctx)
        assert torch.equal(idx, want_idx)
        out, lse = _check_attn(m, p, caches["native"], q, [1] * B, ctx, idx)
        # both are within one rounding of the exact value (weights of 8 bits in the planes' bf16 form: 2^-8 of |v| <= 6 each)
        assert float((out.double() - want.double()).abs().max()) <= (6 * 2.0 ** -8 if dtype == "bf16" else 2e-4)
        assert float((lse - want_lse).abs().max()) <= 2e-3
        idx = m.decode_blocks(p, q, kcs["e4m3"], ctx)
        _check_attn(m, p, caches["e4m3"], q, [1] * B, ctx, idx)
        prev = ctx


@pytest.mark.parametrize("lse_mode", [0, 1])
@pytest.mark.parametrize("dtype,hq,hkv,d,ctxs", [("bf16", 32, 2, 128, [30000, 77, 5000]), ("bf16", 32, 2, 128, [140000]), ("fp32", 4, 1, 64, [3000, 31])])
def test_decode_blocks_are_those_of_the_step(m, lse_mode, dtype, hq, hkv, d, ctxs):
    p = _params(m, dtype, hq, hkv, d, topk_total=16, dense_threshold=40, lse_mode=lse_mode)
    gen = _gen(13)
    B, nc = len(ctxs), m.num_cmp(p, max(ctxs))
    kc = torch.randn((B, hkv, nc, d), generator=gen, device="cuda") * 0.3
    q = torch.randn((B, hq, d), generator=gen, device="cuda").to(p.torch_dtype)
    k = torch.zeros((1, 1, 1, 1), dtype=p.torch_dtype, device="cuda").expand(1, 1, 1, 1)
    k = torch.zeros((B, hkv, max(ctxs), d), dtype=p.torch_dtype, device="cuda")
    _, _, want = m.sparse_decode(p, q, k, k, kc, ctxs)
    assert torch.equal(m.decode_blocks(p, q, kc, ctxs), want)


def test_captured_and_on_other_streams(m):
    """A step captured in a graph and replayed with new inputs, beside eager calls; two captured steps with scratch of their own."""
    p = _params(m, "bf16", 32, 2, 128)
    ctxs = [3000, 500]
    rot = m.Rotary(m.rotary_turns(128), 128)
    side = torch.cuda.Stream()
    gen = _gen(5)
    steps = []
    for i in range(2):
        c, _, _ = _filled(m, p, [n - 1 for n in ctxs], "e4m3", 70 + i)
        c.page_table, _ = paged.pages_for(ctxs, 3, 70 + i)         # (room for the step)
        c2 = m.PagedCache.empty(p, int(c.page_table.max()) + 4, c.page_table)
        k, v = (torch.randn((2, sum(ctxs), 128), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
        m.cache_append(p, c2, k, v, [0, 3000, 3500], [0, 0])
        s = dict(c=c2, cu=m.SeqInfo([0, 1, 2]), prev=m.DecodeInfo([2999, 499]), ctx=m.DecodeInfo(ctxs), one=m.SeqInfo([0, 1, 2]),
                 k=torch.empty((2, 2, 128), dtype=torch.bfloat16, device="cuda"), q=torch.empty((2, 32, 128), dtype=torch.bfloat16, device="cuda"),
                 pos=torch.tensor([2999, 499], dtype=torch.int32, device="cuda"), kc=torch.zeros((2, 2, m.num_cmp(p, 3000), 128), device="cuda"),
                 blocks=torch.empty((2, 2, 8), dtype=torch.int32, device="cuda"), out=torch.empty((2, 32, 128), dtype=torch.bfloat16, device="cuda"),
                 lse=torch.empty((2, 32), device="cuda"), qr=torch.empty((2, 32, 128), dtype=torch.bfloat16, device="cuda"),
                 wa=torch.empty(m.workspace_bytes(m.OP_CACHE_ATTN, p, 2, 2, 3000), dtype=torch.uint8, device="cuda"),
                 wb=torch.empty(m.workspace_bytes(m.OP_DECODE_BLOCKS, p, 2, 0, 3000), dtype=torch.uint8, device="cuda"))
        m.cache_compress_k(p, c2, s["kc"], [0, 0], [2999, 499])
        steps.append(s)

    def step(s):
        m.cache_append(p, s["c"], s["k"], s["k"], s["cu"], s["prev"], rot)
        m.cache_compress_k(p, s["c"], s["kc"], s["prev"], s["ctx"])
        m.rotary_fwd(p, rot, s["q"], s["pos"], out=s["qr"])
        m.decode_blocks(p, s["qr"], s["kc"], s["ctx"], out=s["blocks"], workspace=s["wb"])
        m.cache_attn(p, s["c"], s["qr"], s["one"], s["ctx"], s["blocks"], out=s["out"], lse=s["lse"], workspace=s["wa"])

    def inputs(s, seed):
        gen = _gen(seed)
        s["k"].copy_(torch.randn((2, 2, 128), generator=gen, device="cuda"))
        s["q"].copy_(torch.randn((2, 32, 128), generator=gen, device="cuda"))

    graphs = []
    for s in steps:
        inputs(s, 1)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            step(s)
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(s)
        graphs.append(g)
    for seed in (2, 3, 4):
        want = []
        for s in steps:
            inputs(s, seed)
            state = [s["c"].k.view(torch.uint8).clone(), s["c"].v.view(torch.uint8).clone(), s["c"].k_scale.clone(), s["c"].v_scale.clone()]
            step(s)
            torch.cuda.synchronize()
            want.append([s["out"].clone(), s["lse"].clone(), s["blocks"].clone()])
            for x, y in zip((s["c"].k.view(torch.uint8), s["c"].v.view(torch.uint8), s["c"].k_scale, s["c"].v_scale), state):
                x.copy_(y)
            s["out"].zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for s, w in zip(steps, want):
            assert torch.equal(s["out"], w[0]) and torch.equal(s["lse"], w[1]) and torch.equal(s["blocks"], w[2])


def test_chunks_captured(m):
    """A chunk of a prompt for the tiles of 8 wavefronts and a few proposed tokens, appended and attended to in one captured graph."""
    p = _params(m, "bf16", 32, 2, 128)
    rot = m.Rotary(m.rotary_turns(128), 128)
    news, prev = [200, 3], [5000, 700]
    ctxs = [5200, 703]
    c, _, _ = _filled(m, p, prev, "e4m3", 81)
    table = torch.full((2, 82), -1, dtype=torch.int32, device="cuda")
    table[:, :c.page_table.shape[1]] = c.page_table
    pages = c.k.shape[0]
    c = m.PagedCache(p, *(torch.cat([x.view(torch.uint8), x.view(torch.uint8)[:8]]).view(torch.float8_e4m3fn) for x in (c.k, c.v)), table,
                     *(torch.cat([x, x[:8]]) for x in (c.k_scale, c.v_scale)))
    table[0, 79:82] = torch.tensor([pages, pages + 1, pages + 2], dtype=torch.int32)
    cu, pv, cx = m.SeqInfo([0, 200, 203]), m.DecodeInfo(prev), m.DecodeInfo(ctxs)
    k, v = (torch.empty((2, 203, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q, out = (torch.empty((203, 32, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lse = torch.empty((203, 32), device="cuda")
    ws = torch.empty(m.workspace_bytes(m.OP_CACHE_ATTN, p, 2, 203, 5200), dtype=torch.uint8, device="cuda")
    pages = [x.view(torch.uint8) for x in (c.k, c.v)] + [c.k_scale, c.v_scale]
    before = [x.clone() for x in pages]

    def call():
        m.cache_append(p, c, k, v, cu, pv, rot)
        m.cache_attn(p, c, q, cu, cx, out=out, lse=lse, workspace=ws)

    def inputs(seed):
        gen = _gen(seed)
        for x in (k, v, q):
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        for x, y in zip(pages, before):
            x.copy_(y)
        out.zero_()

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
        call()
        torch.cuda.synchronize()
        want = [x.clone() for x in [out, lse] + pages]
        inputs(seed)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip([out, lse] + pages, want))
    sc = (c.k_scale, c.v_scale)
    exact, exact_lse, mass = paged.attention(q, c.k, c.v, sc, table, news, ctxs, p.softmax_scale)
    assert bool(((out.double() - exact).abs() <= 2.0 ** -8 * exact.abs() + 6 * 2.0 ** -12 + 2.0 ** -8 * mass).all())
    assert float((lse.double() - exact_lse).abs().max()) <= 1e-4


def test_arguments_that_do_not_fit(m):
    """Refused before a call: another dtype or number of heads than the cache's, a table without room, wrong shapes."""
    p = _params(m, "bf16", 8, 2, 64)
    c, k, v = _filled(m, p, [100, 300], "native", 91)
    q = torch.zeros((2, 8, 64), dtype=torch.bfloat16, device="cuda")
    kc = torch.zeros((2, 2, 20, 64), device="cuda")
    new = torch.zeros((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    wide = torch.full((2, 100), 0, dtype=torch.int32, device="cuda")
    part = m.PagedCache(p, c.k, c.v, wide[:, :5])              # room for 320 tokens each
    other = _params(m, "bf16", 16, 4, 64)
    fp32 = _params(m, "fp32", 8, 2, 64)
    for call in (lambda: m.cache_attn(other, c, torch.zeros((2, 16, 64), dtype=torch.bfloat16, device="cuda"), [0, 1, 2], [100, 300]),
                 lambda: m.cache_attn(fp32, c, q.float(), [0, 1, 2], [100, 300]),
                 lambda: m.cache_attn(p, part, q, [0, 1, 2], [100, 321]),
                 lambda: m.cache_attn(p, c, q[:, :4], [0, 1, 2], [100, 300]),
                 lambda: m.cache_append(fp32, c, new.float(), new.float(), [0, 1, 2], [100, 300]),
                 lambda: m.cache_append(p, part, new, new, [0, 1, 2], [100, 320]),
                 lambda: m.cache_compress_k(p, part, kc, [100, 300], [100, 321]),
                 lambda: m.cache_compress_k(other, c, torch.zeros((2, 4, 20, 64), device="cuda"), [0, 0], [100, 300]),
                 lambda: m.decode_blocks(p, q, kc[:, :1].contiguous(), [100, 300]),
                 lambda: m.decode_blocks(p, q, kc, [100, 300], out=torch.empty((2, 2, 3), dtype=torch.int32, device="cuda"))):
        with pytest.raises(AssertionError):
            call()
    m.cache_append(p, part, new[:, :1], new[:, :1], [0, 1, 1], [319, 320])   # the last row that fits
    with pytest.raises(m.InfllmV2Error):
        m.cache_attn(p, c, q, [0, 1, 2], [100, 100000])
