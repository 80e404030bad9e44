"""Batches of the paged cache with more sequences than a search looks at in one step (64), and ragged ones."""
import pytest
import torch

import paged
from test_gpu_cache import _filled, _params, m  # noqa: F401

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
