"""Attention over the paged cache with numbers at the edges of their types: infinities among the values, sums next to the largest float, logits far
below zero, and how exact the weights are."""
import math

import pytest
import torch

import paged
from test_gpu_cache import _filled, _gen, _params, m  # noqa: F401

pytestmark = pytest.mark.gpu

# One token, a few and a chunk of each sequence: the kernel of 16 columns in one launch and in splits, tiles of eight wavefronts, with weights of two
# pieces (8 tokens) and of one
FORMS = [(1, 1), (1, 300), (1, 9001), (3, 200), (3, 6003), (8, 33000), (200, 6001)]
HEADS = [(32, 2, 128), (8, 2, 64)]


def _value(c, b, t):
    """where token t of sequence b is: page, row"""
    return int(c.page_table[b, t // 64]), t % 64


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", *HEADS[0]), ("bf16", *HEADS[1]), ("fp32", 4, 1, 64)])
@pytest.mark.parametrize("n,ctx", FORMS)
def test_infinite_values_keep_their_sign(m, dtype, hq, hkv, d, n, ctx):  # noqa: F811
    """An infinity among the values of a visible key, whatever its weight (1 for the key with the largest logit, or any other): the same infinity in its
    channel, every other channel as without it, bit for bit."""
    p = _params(m, dtype, hq, hkv, d)
    c, _, _ = _filled(m, p, [ctx], "native", 3)
    q = torch.randn((n, hq, d), generator=_gen(4), device="cuda").to(p.torch_dtype)
    page, row = _value(c, 0, 0)                             # the key with the largest logit of head 0's last token
    c.k[page, 0, row] = q[-1, 0] * (4 / q[-1, 0].float().norm())
    clean, clean_lse = m.cache_attn(p, c, q, [0, n], [ctx])
    for sign, t, ch in ((1, 0, 5), (-1, ctx // 2, 7)):
        page, row = _value(c, 0, t)
        was = c.v[page, :, row, ch].clone()
        c.v[page, :, row, ch] = sign * float("inf")
        out, lse = m.cache_attn(p, c, q, [0, n], [ctx])
        assert torch.equal(lse, clean_lse)
        sees = torch.arange(ctx - n, ctx, device="cuda") >= t
        assert bool((out[sees][..., ch] == sign * float("inf")).all()), (t, out[sees][..., ch].flatten()[:4])
        rest = [x for x in range(d) if x != ch]
        assert torch.equal(out[..., rest], clean[..., rest]) and torch.equal(out[~sees], clean[~sees])
        c.v[page, :, row, ch] = was


@pytest.mark.parametrize("kv", ["native", "e4m3"])
@pytest.mark.parametrize("n,ctx", [(1, 200), (1, 33000), (2, 200), (4, 33000), (5, 33000), (8, 33000), (8, 500)])
def test_weights_of_a_few_tokens(m, kv, n, ctx):  # noqa: F811
    """Values that cancel show the weights alone.  Channel i is made for column i (a token and a head of KV head 0): four keys B of value 1 and weight w below
    1, five keys A of weight 1 whose values add up to -4 w as nearly as five rounded numbers do, every other key of weight 0.
    Derivation, bf16 data: a weight enters as two bf16 pieces, the second rounded to nearest: off by at most 2^-16 of it, either way; 1 is the sum of two such
    pieces, and B's are half of the sum of p |v|: 2^-17 of that.  9 terms in 32 bits whose sum stays below that half: 9 * 2^-24 / 2 < 2^-21.8; w itself (the
    exponential, the scale's rounding): 2^-22 of a half and less.  A result's own rounding: 2^-8 of it.  Roundings to nearest are as often up as down: over N
    weights their mean is within 4 / sqrt(N) of the largest."""
    hq, hkv, d, few, many = 32, 2, 128, 5, 4
    p = _params(m, "bf16", hq, hkv, d, softmax_scale=1.0)
    pages = (ctx + 63) // 64
    c = m.PagedCache.empty(p, pages, torch.arange(pages, dtype=torch.int32, device="cuda")[None].contiguous(), kv)
    a, b = torch.arange(2, 2 + few), torch.arange(30, 30 + many)
    columns = [(ch % (16 * n) // 16, ch % 16) for ch in range(d)]
    seeds, errors = 8 if ctx <= 500 else 1, 0.0
    for seed in range(seeds):
        z = (-torch.rand((n, hq), generator=_gen(seed), device="cuda") * 2).to(torch.bfloat16)
        q = torch.zeros((n, hq, d), device="cuda", dtype=torch.bfloat16)
        q[..., 0], q[..., 1] = z, 200.0                     # logits: z for B, 0 for A, -200 for the others
        k, v = torch.zeros((ctx, d), device="cuda"), torch.zeros((ctx, d), device="cuda", dtype=torch.float64)
        k[:, 1] = -1.0
        k[a] = k[b] = 0.0
        k[b, 0] = 1.0
        w = torch.stack([z[i, h].double().exp() for i, h in columns])
        v[b] = 1.0
        left, s = -many * w, paged.scale_for(float(many * w.max()))
        for t in a.tolist():
            v[t] = left.to(torch.bfloat16).double() if kv == "native" else paged.to_codes(left / s).double() * s
            left = left - v[t]
        m.cache_append(p, c, *(x[None].expand(hkv, -1, -1).to(torch.bfloat16) for x in (k, v)), [0, ctx], [0])
        sc = None if kv == "native" else c.v_scale
        assert torch.equal(paged.rows_of(c.v, sc, c.page_table, 0, ctx, 0)[0], v)
        out, _ = m.cache_attn(p, c, q, [0, n], [ctx])
        got = torch.stack([out[i, h, ch] for ch, (i, h) in enumerate(columns)]).double()
        want, mass = (many * w + v[a].sum(0)) / (few + many * w), (many * w + v[a].abs().sum(0)) / (few + many * w)
        tol = 2.0 ** -8 * want.abs() + (2.0 ** -17 + 2.0 ** -21.8 + 2.0 ** -23) * mass
        assert bool(((got - want).abs() <= tol).all()), float(((got - want).abs() / tol).max())
        errors += float(((got - want) / mass).mean()) / seeds
    assert abs(errors) <= 2.0 ** -17 * 4 / (seeds * min(d, 16 * n)) ** 0.5 + 2.0 ** -21.8 + 2.0 ** -23


def _large(m, dtype, kv, hq, hkv, d, ctx, seed=5):  # noqa: F811
    """A cache of one sequence whose logits are its first key channel alone"""
    p = _params(m, dtype, hq, hkv, d, softmax_scale=1.0)
    c, _, _ = _filled(m, p, [ctx], kv, seed)
    pages = (ctx + 63) // 64
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None].contiguous()
    return p, m.PagedCache.empty(p, pages, table, kv)


def _write(m, p, c, k0, v):  # noqa: F811
    """keys with k0 [ctx] in channel 0 and nothing else, values v [ctx, d], for every KV head"""
    ctx, d = v.shape
    k = torch.zeros((p.num_kv_heads, ctx, d), device="cuda")
    k[..., 0] = k0
    m.cache_append(p, c, k.to(p.torch_dtype), v[None].expand(p.num_kv_heads, -1, -1).contiguous().to(p.torch_dtype), [0, ctx], [0])


@pytest.mark.parametrize("kv", ["native", "e4m3"])
@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", *HEADS[0]), ("bf16", *HEADS[1]), ("bf16", 5, 5, 64), ("fp32", 4, 1, 64), ("fp32", 6, 2, 128)])
@pytest.mark.parametrize("n,ctx", FORMS + [(700, 6001)])
def test_sums_of_large_values_stay_finite(m, kv, dtype, hq, hkv, d, n, ctx):  # noqa: F811
    """A mean of values next to the largest float is one of them, however many keys and whatever the softmax is taken relative to; values of other
    channels are not touched by that, bit for bit."""
    p, c = _large(m, dtype, kv, hq, hkv, d, ctx)
    q = torch.zeros((n, hq, d), device="cuda", dtype=p.torch_dtype)
    q[..., 0] = 1.0
    gen = _gen(11)
    v = torch.zeros((ctx, d), device="cuda")
    v[:, 8:] = torch.randn((ctx, d - 8), generator=gen, device="cuda")
    k0 = torch.randn(ctx, generator=gen, device="cuda") * 0.25
    _write(m, p, c, k0, v)
    top = 1.75 * 2.0 ** 127 if dtype == "bf16" or kv == "e4m3" else 3.0e38
    if kv == "e4m3":                # (the scale of a page that holds such values: the others are zeros in it)
        v[:, 8:] = 0
        _write(m, p, c, k0, v)
    clean, clean_lse = m.cache_attn(p, c, q, [0, n], [ctx])
    v[:, 0], v[:, 1], v[:, 2], v[:, 3] = top, -top, 2.0 ** 120, top / 2
    _write(m, p, c, k0, v)
    out, lse = m.cache_attn(p, c, q, [0, n], [ctx])
    assert torch.equal(lse, clean_lse) and torch.equal(out[..., 8:], clean[..., 8:])
    for ch, x in ((0, top), (1, -top), (2, 2.0 ** 120), (3, top / 2)):
        # a mean of equal values: the weights' rounding (2^-8 each at most, bf16 tiles) and the result's own
        worst = (out[..., ch].double() / x - 1).abs().max()
        assert bool(worst <= (2.0 ** -7 if dtype == "bf16" else 1e-4)), (ch, float(worst))


@pytest.mark.parametrize("hq,hkv,d,n,ctx", [(32, 2, 128, 1, 9001), (32, 2, 128, 8, 33000), (32, 2, 128, 200, 6001), (8, 2, 64, 701, 6000), (32, 2, 128, 1400, 3001), (8, 2, 64, 2000, 6000)])
def test_the_largest_value_of_the_type(m, hq, hkv, d, n, ctx):  # noqa: F811
    """A mean of the largest bf16 number is that number, although a weight of exp(-0.6875), all keys' but one, is rounded up by 0.2 % in eight bits."""
    p, c = _large(m, "bf16", "native", hq, hkv, d, ctx)
    q = torch.zeros((n, hq, d), device="cuda", dtype=torch.bfloat16)
    q[..., 0] = 1.0
    k0 = torch.full((ctx,), -0.6875, device="cuda")
    k0[0] = 0.0
    top = torch.finfo(torch.bfloat16).max
    v = torch.full((ctx, d), top, device="cuda")
    v[:, 1::2] = -top
    _write(m, p, c, k0, v)
    out, _ = m.cache_attn(p, c, q, [0, n], [ctx])
    assert bool((out == v[0]).all())


@pytest.mark.parametrize("kv", ["native", "e4m3"])
@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", *HEADS[0]), ("fp32", 4, 1, 64)])
@pytest.mark.parametrize("news,topk", [([1, 1], 8), ([1, 1], 40), ([1, 3], 40)])
def test_sums_of_large_values_over_lists(m, kv, dtype, hq, hkv, d, news, topk):  # noqa: F811
    """The same where blocks are listed: the pages of a second walk are those of the first."""
    ctxs = [6001, 700]
    p = _params(m, dtype, hq, hkv, d, softmax_scale=1.0, topk_total=topk, dense_threshold=0)
    c, _, _ = _filled(m, p, ctxs, kv, 5)
    top = 1.75 * 2.0 ** 127 if dtype == "bf16" or kv == "e4m3" else 3.0e38
    sign = torch.tensor([1.0, -1.0, 0.5, 0.0] * (d // 4), device="cuda")
    k = torch.zeros((hkv, sum(ctxs), d), device="cuda")
    k[..., 0] = torch.randn(sum(ctxs), generator=_gen(1), device="cuda") * 0.25
    v = (sign * top).expand(hkv, sum(ctxs), d).contiguous()
    m.cache_append(p, c, k.to(p.torch_dtype), v.to(p.torch_dtype), [0, ctxs[0], sum(ctxs)], [0, 0])
    T, gen = sum(news), torch.Generator().manual_seed(2)
    blocks = torch.full((T, hkv, topk), -1, dtype=torch.int32)
    for row, L in enumerate([ctxs[0]] * news[0] + [ctxs[1]] * news[1]):
        for h in range(hkv):
            x = torch.randperm((L - 3 + 63) // 64, generator=gen)[:topk]
            blocks[row, h, torch.randperm(topk, generator=gen)[:len(x)]] = x.to(torch.int32)
    q = torch.zeros((T, hq, d), device="cuda", dtype=p.torch_dtype)
    q[..., 0] = 1.0
    out, lse = m.cache_attn(p, c, q, [0, news[0], T], ctxs, blocks.cuda())
    want = sign.double() * top
    assert bool(torch.isfinite(lse).all())
    # a mean of equal values: the weights' rounding and the result's own
    assert bool(((out.double() - want).abs() <= (2.0 ** -7 if dtype == "bf16" else 1e-4) * want.abs()).all())


@pytest.mark.parametrize("hq,hkv,d,n,ctx", [(32, 2, 128, 3, 200), (8, 2, 64, 60, 700), (32, 2, 128, 8, 33000), (32, 2, 128, 200, 6001), (8, 2, 64, 701, 6000), (32, 2, 128, 1400, 3001)])
def test_infinities_beside_large_values(m, hq, hkv, d, n, ctx):  # noqa: F811
    """One channel's sums pass the largest float, another has an infinity that only the last tokens see, a third a NaN that all see: each token and channel has what
    is its own."""
    p, c = _large(m, "bf16", "native", hq, hkv, d, ctx)
    q = torch.zeros((n, hq, d), device="cuda", dtype=torch.bfloat16)
    q[..., 0] = 1.0
    v = torch.randn((ctx, d), generator=_gen(11), device="cuda")
    k0 = torch.randn(ctx, generator=_gen(12), device="cuda") * 0.25
    _write(m, p, c, k0, v)
    clean, clean_lse = m.cache_attn(p, c, q, [0, n], [ctx])
    top, late = 1.75 * 2.0 ** 127, ctx - 1 - n // 2
    v[:, 0], v[:, 9] = top, -top
    v[late, 5] = float("inf")
    v[3, 6] = float("nan")
    _write(m, p, c, k0, v)
    out, lse = m.cache_attn(p, c, q, [0, n], [ctx])
    sees = torch.arange(ctx - n, ctx, device="cuda") >= late
    assert torch.equal(lse, clean_lse)
    assert bool((out[sees][..., 5] == float("inf")).all()) and torch.equal(out[~sees][..., 5], clean[~sees][..., 5])
    assert bool(torch.isnan(out[..., 6]).all())
    for ch, x in ((0, top), (9, -top)):
        assert bool((out[..., ch].double() / x - 1).abs().max() <= 2.0 ** -7)
    rest = [x for x in range(d) if x not in (0, 5, 6, 9)]
    assert torch.equal(out[..., rest], clean[..., rest])


@pytest.mark.parametrize("hq,hkv,d,n,ctx", [(32, 2, 128, 200, 6001), (8, 2, 64, 701, 6000), (32, 2, 128, 1400, 3001), (32, 2, 128, 1, 9001), (32, 2, 128, 3, 100)])
def test_references_behind_the_largest_logit(m, hq, hkv, d, n, ctx):  # noqa: F811
    """One key of weight 1 and two of 59.75 in different half pages, V = 2^122: sums relative to the first key would be 2^128.9."""
    p, c = _large(m, "bf16", "native", hq, hkv, d, ctx)
    q = torch.zeros((n, hq, d), device="cuda", dtype=torch.bfloat16)
    q[..., 0] = 1.0
    k0 = torch.full((ctx,), -100.0, device="cuda")
    k0[0], k0[10], k0[40] = 0.0, 4.09375, 4.09375
    _write(m, p, c, k0, torch.full((ctx, d), 2.0 ** 122, device="cuda"))
    out, lse = m.cache_attn(p, c, q, [0, n], [ctx])
    assert bool((out.double() / 2.0 ** 122 - 1).abs().max() <= 2.0 ** -7)
    want = math.log(1 + 2 * math.exp(4.09375))
    assert float((lse.double() - want).abs().max()) <= 1e-5


@pytest.mark.parametrize("n,ctx", FORMS)
def test_small_weights_of_large_values_count(m, n, ctx):  # noqa: F811
    """A key 2^-100 times as heavy as another and of a value 2^110 times as large: most of the result.  (The other way round, weights that are cut off far
    below the largest would lose it.)"""
    hq, hkv, d = 32, 2, 128
    p, c = _large(m, "bf16", "native", hq, hkv, d, ctx)
    q = torch.zeros((n, hq, d), device="cuda", dtype=torch.bfloat16)
    q[..., 0] = 1.0
    k0 = torch.full((ctx,), -1000.0, device="cuda")
    v = torch.zeros((ctx, d), device="cuda")
    k0[0], v[0] = 0.0, 1.0
    want = 1.0
    if ctx - n >= 70:
        k0[69], v[69] = -69.5, 2.0 ** 110
        want += math.exp(-69.5) * 2.0 ** 110
    _write(m, p, c, k0, v)
    out, _ = m.cache_attn(p, c, q, [0, n], [ctx])
    # the weights' rounding and the result's: 2^-8 each; a logit of -69.5 in units of log2 (-100.27) to 2^-17 of a binary order
    assert bool((out.double() / want - 1).abs().max() <= 2.0 ** -7 + 2.0 ** -16)


@pytest.mark.parametrize("n,ctx", FORMS)
def test_logits_far_below_zero(m, n, ctx):  # noqa: F811
    """All logits at -2^127 ln 2, -1.7e38 in units of log2: a softmax over equal logits is a mean, wherever they are."""
    hq, hkv, d = 32, 2, 128
    p = _params(m, "bf16", hq, hkv, d, softmax_scale=math.log(2.0))
    _, c = _large(m, "bf16", "native", hq, hkv, d, ctx)
    q = torch.zeros((n, hq, d), device="cuda", dtype=torch.bfloat16)
    q[..., 0] = -(2.0 ** 64)
    v = torch.randn((ctx, d), generator=_gen(2), device="cuda").to(torch.bfloat16)
    _write(m, p, c, torch.full((ctx,), 2.0 ** 63, device="cuda"), v.float())
    out, lse = m.cache_attn(p, c, q, [0, n], [ctx])
    want = (v.double().cumsum(0) / torch.arange(1, ctx + 1, device="cuda")[:, None])[ctx - n:, None]
    mass = (v.double().abs().cumsum(0) / torch.arange(1, ctx + 1, device="cuda")[:, None])[ctx - n:, None]
    # equal weights: exact; sums in 32 bits of up to 6001 terms; the result's own rounding
    assert bool(((out.double() - want).abs() <= 2.0 ** -8 * want.abs() + ctx * 2.0 ** -24 * mass).all())
    assert float((lse.double() / -(2.0 ** 127 * math.log(2.0)) - 1).abs().max()) <= 1e-6
