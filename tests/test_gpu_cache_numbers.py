"""Attention over the paged cache with numbers at the edges of their types: infinities among the values."""
import pytest
import torch

from test_gpu_cache import _filled, _gen, _params, m  # noqa: F401

pytestmark = pytest.mark.gpu

# One token, a few and a chunk of each sequence: the kernel of 16 columns in one launch and in splits, tiles of eight wavefronts
FORMS = [(1, 1), (1, 300), (1, 9001), (3, 200), (3, 6003), (200, 6001)]
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
