"""Trees of more sequences than a wavefront has lanes, ragged and of one size, in both kernels; tables that are part of wider ones; sequences that share the pages of a context."""
import pytest
import torch

import paged
from paged import PAGE
from test_gpu_cache import _filled, _params, m  # noqa: F401
from test_gpu_tree import _check, _lists, _masks, _q

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 32, 2, 128), ("bf16", 8, 2, 64), ("fp32", 4, 1, 64)])
@pytest.mark.parametrize("sizes", ["ragged", "few", "alike", "alike few"])
@pytest.mark.parametrize("listed", [False, True])
def test_many_sequences(m, kv, dtype, hq, hkv, d, sizes, listed):  # noqa: F811
    p = _params(m, dtype, hq, hkv, d, topk_total=6, dense_threshold=150)
    B = 133
    news = {"ragged": [(7 * b) % 23 for b in range(B)], "few": [(5 * b) % 9 for b in range(B)], "alike": [11] * B, "alike few": [3] * B}[sizes]
    ctxs = [n + (389 * b) % 700 for b, n in enumerate(news)]
    ctxs[70], ctxs[-1] = news[70] + 5000, news[-1] + 3100              # (two that are split)
    c, _, _ = _filled(m, p, [max(x, 1) for x in ctxs], kv, 81)
    wide = torch.full((B + 2, c.page_table.shape[1] + 5), 1 << 30, dtype=torch.int32, device="cuda")
    wide[:B, :-5] = c.page_table
    c = m.PagedCache(p, c.k, c.v, wide[:, :-5], c.k_scale, c.v_scale)
    _check(m, p, c, _q(p, news, 20), news, ctxs, _masks(m, news, ctxs, 21), _lists(p, news, ctxs, 22) if listed else None)


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 32, 2, 128), ("fp32", 4, 1, 64)])
def test_sequences_that_share_a_context(m, kv, dtype, hq, hkv, d):  # noqa: F811
    """Whole pages of one prompt in the tables of several sequences, each with a tree of its own behind it."""
    p = _params(m, dtype, hq, hkv, d)
    news, front = [20, 1, 8, 33], 10 * PAGE
    ctxs = [front + n for n in news]
    c, _, _ = _filled(m, p, ctxs, kv, 83)
    c.page_table[1:, :10] = c.page_table[0, :10]
    out, _ = _check(m, p, c, _q(p, news, 23), news, ctxs, _masks(m, news, ctxs, 24))
    alone = m.PagedCache(p, c.k, c.v, c.page_table[3:], c.k_scale, c.v_scale)
    q, mask = _q(p, news, 23)[29:].contiguous(), _masks(m, news, ctxs, 24)[29:].contiguous()
    one, _ = m.cache_tree_attn(p, alone, q, [0, 33], ctxs[3:], mask)
    # each is off by its own rounding and its weights' (2^-8 of |v| <= 6 at most)
    tol = 2 * (2.0 ** -8 * out[29:].double().abs() + 2.0 ** -8 * 6) if dtype == "bf16" else 2e-4
    assert bool(((one.double() - out[29:].double()).abs() <= tol).all())


def test_pages_past_four_gigabytes(m):  # noqa: F811
    """Attention, accepted paths and copies at both ends of a pool of 4.6 GB of keys and as many of values."""
    p = _params(m, "bf16", 8, 2, 128)
    pages, n, ctx = 140000, 40, 300
    k, v = (torch.empty((pages, 2, PAGE, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.tensor([[pages - 1, 3, pages - 7, 140, pages - 2]], dtype=torch.int32, device="cuda")
    c = m.PagedCache(p, k, v, table)
    small, dk, dv = _filled(m, p, [ctx], "native", 85)
    m.cache_append(p, c, dk, dv, [0, ctx], [0])
    mask, q = _masks(m, [n], [ctx], 26), _q(p, [n], 27)
    want, _ = m.cache_tree_attn(p, small, q, [0, n], [ctx], mask)
    assert torch.equal(m.cache_tree_attn(p, c, q, [0, n], [ctx], mask)[0], want)
    path = torch.tensor([[0, 4, 9, 30, 39]], dtype=torch.int32, device="cuda")
    for x in (small, c):
        assert m.cache_accept(p, x, [0, n], [ctx], path).tolist() == [ctx - n + 5]
    rows = lambda x, y: paged.rows_of(y, None, x.page_table, 0, ctx - n + 5, 1)[0]  # noqa: E731
    assert torch.equal(rows(c, c.k), rows(small, small.k)) and torch.equal(rows(c, c.v), rows(small, small.v))
    m.cache_copy_pages(p, c, torch.tensor([[pages - 1, 1], [3, pages - 3]], dtype=torch.int32, device="cuda"))
    assert torch.equal(k[1], k[pages - 1]) and torch.equal(v[pages - 3], v[3])
