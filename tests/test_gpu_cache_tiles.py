"""Chunks of prompts over the paged cache that are long enough for the tile kernel (csrc/cache_attn_tile.hip), for every head shape: lengths that end inside tiles
and pages, pages that are not there, splits along the keys, values that are not finite, a mixture with single tokens and lists."""
import pytest
import torch

from test_gpu_cache import _check_attn, _filled, _gen, _params, m  # noqa: F401

pytestmark = pytest.mark.gpu

# Small tiles (launch_rules.h), then large ones: one split and several
SHAPES = [(32, 2, 128, [150], [6001]), (8, 2, 64, [701], [6000]), (5, 5, 64, [703], [5990]), (12, 4, 128, [303], [6010]), (6, 6, 128, [257, 700], [2000, 5000]),
          (16, 1, 64, [400], [5000]), (14, 2, 64, [333], [5050]),
          (32, 2, 128, [1400], [3001]), (12, 4, 128, [901], [7000]), (14, 2, 64, [905], [9000]), (5, 5, 64, [1703], [9001]), (8, 2, 64, [2000, 2005], [6000, 2005])]


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("hq,hkv,d,news,ctxs", SHAPES)
def test_chunks(m, kv, hq, hkv, d, news, ctxs):  # noqa: F811
    p = _params(m, "bf16", hq, hkv, d)
    c, _, _ = _filled(m, p, ctxs, kv, 81, "tokens" if hkv == 2 else "heads")
    q = (torch.randn((sum(news), hq, d), generator=_gen(15), device="cuda") * 2).to(torch.bfloat16)
    _check_attn(m, p, c, q, news, ctxs)


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("hq,hkv,d,n,L", [(32, 2, 128, 130, 2990), (8, 2, 64, 600, 2990), (32, 2, 128, 700, 8100), (8, 2, 64, 1500, 8990)])
def test_beside_single_tokens_and_lists(m, kv, hq, hkv, d, n, L):  # noqa: F811
    """One call: a chunk, single tokens, a skipped sequence, and (second) sequences with block lists; pages that are not there."""
    p = _params(m, "bf16", hq, hkv, d, topk_total=8, dense_threshold=3000)
    news, ctxs = [1, n, 0, 1, n, 7], [2000, L, 100, 6000, n, 2900]
    c, _, _ = _filled(m, p, ctxs, kv, 91)
    c.page_table[1, 0] = c.page_table[1, 7] = c.page_table[1, 20] = -1
    c.page_table[1, (L - n // 2) // 64] = c.k.shape[0] + 5
    q = torch.randn((sum(news), hq, d), generator=_gen(16), device="cuda").to(torch.bfloat16)
    _check_attn(m, p, c, q, news, ctxs)
    blocks = torch.full((sum(news), hkv, 8), -1, dtype=torch.int32, device="cuda")
    blocks[n + 1, :, :3] = torch.tensor([93, 5, 40], dtype=torch.int32)
    blocks[1:n + 1, :, 2] = 3                                # (L over the threshold: the chunk's as well)
    _check_attn(m, p, c, q, news, ctxs, blocks)


def test_no_page_at_all(m):  # noqa: F811
    p = _params(m, "bf16", 32, 2, 128)
    c, _, _ = _filled(m, p, [6000], "e4m3", 7)
    c.page_table[0, 1:] = -1
    c.page_table[0, 0] = c.k.shape[0]
    q = torch.randn((200, 32, 128), generator=_gen(1), device="cuda").to(torch.bfloat16)
    out, lse = m.cache_attn(p, c, q, [0, 200], [6000])
    assert bool((out == 0).all()) and bool((lse == -float("inf")).all())


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("hq,hkv,d,n,ctx", [(32, 2, 128, 150, 6001), (8, 2, 64, 701, 6000), (5, 5, 64, 703, 5990),
                                            (32, 2, 128, 700, 7990), (14, 2, 64, 902, 9000)])
def test_values_that_are_not_finite(m, kv, hq, hkv, d, n, ctx):  # noqa: F811
    """Rows behind a token, of the last page's end and one channel of an earlier row hold infinities and NaN: who does not see them is as if they were not
    there, bit for bit; who does gets them in their channels."""
    p = _params(m, "bf16", hq, hkv, d)
    c, _, _ = _filled(m, p, [ctx], kv, 95)
    q = torch.randn((n, hq, d), generator=_gen(17), device="cuda").to(torch.bfloat16)
    clean, clean_lse = _check_attn(m, p, c, q, [n], [ctx])
    bits = c.v.view(torch.uint8) if kv == "e4m3" else c.v
    kbits = c.k.view(torch.uint8) if kv == "e4m3" else c.k
    bad = 0x7f if kv == "e4m3" else -float("inf")

    def row(t):
        return int(c.page_table[0, t // 64]), t % 64
    for t in range(ctx - 3, (ctx + 63) // 64 * 64):       # the last three tokens, and the rest of the last page
        g, r = row(t)
        bits[g, :, r] = bad
        kbits[g, :, r] = 0xff if kv == "e4m3" else float("nan")
    first = ctx - n + n // 2                               # a token in the middle of the chunk: its value has one odd channel
    g, r = row(first)
    bits[g, 0, r, 5] = bad
    out, lse = m.cache_attn(p, c, q, [0, n], [ctx])
    assert torch.equal(out[:n // 2], clean[:n // 2]) and torch.equal(lse[:n - 3], clean_lse[:n - 3])
    G = hq // hkv
    seen = out[n // 2:n - 3, :G].float()
    assert bool((torch.isnan(seen[..., 5]) if kv == "e4m3" else seen[..., 5] == -float("inf")).all())
    keep = [x for x in range(d) if x != 5]
    assert torch.equal(out[n // 2:n - 3, :G][..., keep], clean[n // 2:n - 3, :G][..., keep])
    assert torch.equal(out[n // 2:n - 3, G:], clean[n // 2:n - 3, G:])
    assert bool(torch.isnan(out[n - 1]).all())


def test_logits_far_apart(m):  # noqa: F811
    """References that move by hundreds in later pages, logits of minus infinity, a query of infinities beside others."""
    p = _params(m, "bf16", 32, 2, 128)
    c, _, _ = _filled(m, p, [6000], "native", 99)
    scale = torch.linspace(0.1, 30, 94, device="cuda")
    for j in range(94):                                    # keys grow page by page
        c.k[int(c.page_table[0, j])] *= scale[j]
    q = torch.randn((160, 32, 128), generator=_gen(18), device="cuda").to(torch.bfloat16)
    cu = [0, 160]
    import paged
    want, want_lse, mass = paged.attention(q, c.k, c.v, None, c.page_table, [160], [6000], p.softmax_scale)
    out, lse = m.cache_attn(p, c, q, cu, [6000])
    # logits of up to some 300 in 32 bits: products of 128 terms summed in 32 bits, off by at most 128 * 2^-24 of 128 * 4 * 30 * 4 / 11.3; weights as in the other tests
    slack = 128 * 2.0 ** -24 * 128 * 4 * 120 / 11.3
    assert bool(((out.double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2 * slack) * mass).all())
    assert float((lse.double() - want_lse).abs().max()) <= slack
    q2 = q.clone()
    q2[77] = float("inf")
    out2, _ = m.cache_attn(p, c, q2, cu, [6000])
    rest = [i for i in range(160) if i != 77]
    assert bool(torch.isnan(out2[77]).all()) and torch.equal(out2[rest], out[rest])
