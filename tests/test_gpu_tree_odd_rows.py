"""Values that are not finite in every drafted row at once, each in a channel of its own: whichever lane and wavefront meets one, the tokens that see the row get it and no
others do."""
import pytest
import torch

import trees
from test_gpu_cache import _filled, _params, m  # noqa: F401
from test_gpu_tree import _masks, _q

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv", ["e4m3", "native"])
@pytest.mark.parametrize("dtype,hq,hkv,d,n", [("fp32", 4, 1, 64, 64), ("fp32", 6, 2, 128, 50), ("bf16", 5, 5, 64, 64), ("bf16", 16, 16, 128, 40), ("bf16", 32, 2, 128, 7), ("bf16", 32, 2, 128, 64)])
@pytest.mark.parametrize("front", [0, 3, 37, 64, 700])
@pytest.mark.parametrize("only", [False, True])
def test_every_drafted_row(m, kv, dtype, hq, hkv, d, n, front, only):  # noqa: F811
    """only: one row at a time (the first lane's rows and others', alone)"""
    p = _params(m, dtype, hq, hkv, d)
    ctx = front + n
    c, _, _ = _filled(m, p, [ctx], kv, 66)
    q, mask = _q(p, [n], 18), _masks(m, [n], [ctx], 19)
    clean = m.cache_tree_attn(p, c, q, [0, n], [ctx], mask)[0]
    sees = torch.zeros((n, d), dtype=torch.bool)
    for i, s in enumerate(trees.to_sets(mask.cpu(), n)):
        sees[i, sorted(s)] = True
    raw, bad = (c.v.view(torch.uint8), 0x7f) if kv == "e4m3" else (c.v, float("inf"))
    at = [(int(c.page_table[0, t // 64]), t % 64) for t in range(front, ctx)]
    was = c.v.clone()
    for j in range(0, n, 5) if only else [None]:
        for i in range(n) if j is None else [j]:
            raw[at[i][0], :, at[i][1], i] = bad
        got = m.cache_tree_attn(p, c, q, [0, n], [ctx], mask)[0]
        c.v.view(torch.uint8).copy_(was.view(torch.uint8))
        who = sees if j is None else sees & (torch.arange(d) == j)
        want = torch.where(who[:, None, :].cuda(), torch.tensor(float("nan") if kv == "e4m3" else bad, device="cuda", dtype=clean.dtype), clean)
        assert bool(((got == want) | (got.isnan() & want.isnan())).all()), j
