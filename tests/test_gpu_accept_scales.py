"""Accepted paths between pages of any scales: rows of zeros, pages of zeros, the smallest and the largest scale; equal to the definition to the last bit."""
import pytest
import torch

import trees
from test_gpu_cache import _cache, _gen, _params, _same, m  # noqa: F401
from test_gpu_pages import _state

pytestmark = pytest.mark.gpu

# rows 4 .. 63 of a sequence's first page come from its second and third, rows 0 .. 2 of its second from the third
FRONT, NEW, PATH = 4, 150, [0] + list(range(70, 132))


def _accepted(m, p, c, batch):  # noqa: F811
    k, v, ks, vs = _state(c)
    ctxs, news = [FRONT + NEW] * batch, [NEW] * batch
    want = trees.accept(k, v, (ks, vs), c.page_table, news, ctxs, [PATH] * batch)
    path = torch.tensor([PATH + [-1]] * batch, dtype=torch.int32, device="cuda")
    got = m.cache_accept(p, c, [NEW * b for b in range(batch + 1)], ctxs, path)
    assert got.tolist() == want
    assert torch.equal(c.k_scale, ks) and torch.equal(c.v_scale, vs)
    assert _same(c.k, k) and _same(c.v, v)


@pytest.mark.parametrize("dtype,hkv,d,layout", [("bf16", 2, 128, "heads"), ("bf16", 3, 64, "tokens"), ("fp32", 1, 64, "heads")])
@pytest.mark.parametrize("rows", ["zeros", "minus zeros", "one code", "any", "NaN"])
def test_scales_of_the_whole_range(m, dtype, hkv, d, layout, rows):  # noqa: F811
    """Each pair of scales of the page that rows come from and the page that they go to; the latter holds zeros, as cache_append leaves it at the smallest scale, or
    anything.  A row of zeros needs no scale: it is zeros at any."""
    p = _params(m, dtype, hkv, hkv, d)
    exps = [-100, -63, 0, 27, 28, 100, 119]
    pairs = [(a, b) for a in exps for b in exps]
    batch = 2 * len(pairs)
    c = _cache(m, p, [FRONT + NEW] * batch, "e4m3", 3, layout)
    gen = _gen(7)
    table = c.page_table.long()
    for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)):
        bits = x.view(torch.uint8)
        codes = torch.randint(0, 256, x.shape, generator=gen, device="cuda", dtype=torch.uint8)
        bits.copy_(codes)
        source = {"zeros": torch.zeros_like, "minus zeros": lambda y: torch.full_like(y, 0x80), "any": lambda y: y, "NaN": lambda y: torch.full_like(y, 0x7f),
                  "one code": lambda y: torch.where(torch.rand(y.shape, generator=gen, device="cuda") < 1 / 400, y & 0x81, torch.zeros_like(y))}[rows]
        for j in (1, 2):                      # pages that rows come from
            bits[table[:, j]] = source(codes[table[:, j]])
        bits[table[::2, 0]] = 0               # every other sequence: a first page of zeros
        for b in range(batch):
            up, to = pairs[b // 2]
            s[table[b, 0]], s[table[b, 1]], s[table[b, 2]] = 2.0 ** to, 2.0 ** up, 2.0 ** up
    _accepted(m, p, c, batch)


def test_zeros_that_were_appended(m):  # noqa: F811
    """Keys and values in one head of a sequence: tokens of zeros but for one of 1e12 behind them, in another page; the zeros are accepted and stay zeros."""
    p = _params(m, "bf16", 2, 2, 64)
    c = _cache(m, p, [FRONT + NEW], "e4m3", 4)
    k = torch.zeros((2, FRONT + NEW, 64), device="cuda")
    k[0, FRONT + NEW - 1] = 1e12
    k = k.to(torch.bfloat16)
    m.cache_append(p, c, k, k, [0, FRONT + NEW], [0])
    _accepted(m, p, c, 1)
    page = int(c.page_table[0, 0])
    assert bool((c.k[page].float() == 0).all()) and bool((c.v[page].float() == 0).all())
