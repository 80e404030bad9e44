"""Calls of the paged cache at the limits of what a launch holds, and scratch of calls with a few query tokens.  No GPU is needed (pointers here are not
device memory: a call that went on would fault), and with one nothing here is run that would go on."""
import ctypes
import random

import numpy as np
import pytest
import torch

from test_cache_host import HIP, UNSUPPORTED, _cache, _ints, m, one  # noqa: F401

no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="calls whose arguments are in order must end at the launch: no GPU")


def _append(m, d, n):  # noqa: F811
    p = m.Params.make("bf16", 1, 1, d)
    c = _cache(m, page=64 * d, head=64 * d, tok=d, stride=(n + 63) // 64)
    (_a, cu), (_b, prev) = _ints([0, n]), _ints([0])
    return m.lib().infllmv2_cache_append(ctypes.byref(p), ctypes.byref(c), None, one, one, d, n * d, cu, one, prev, one, None, 1, None)


def _attn(m, n, ctx, blocks, **over):  # noqa: F811
    p = m.Params.make("bf16", 32, 2, 128, n_init=1, n_local=1, topk_total=4, dense_threshold=0)
    c = _cache(m, page=2 * 64 * 128, head=64 * 128, tok=128, stride=(ctx + 63) // 64)
    (_a, cu), (_b, cx) = _ints([0, n]), _ints([ctx])
    return m.lib().infllmv2_cache_attn(ctypes.byref(p), ctypes.byref(c), one, cu, one, cx, one, 1, blocks, one, None, one, 1 << 60, None)


@pytest.mark.parametrize("d", [64, 128])
def test_appends_that_no_launch_holds(m, d):  # noqa: F811
    """A workgroup of 4 d threads per page, 2^32 threads in all."""
    assert _append(m, d, ((1 << 30) // d) * 64) == UNSUPPORTED
    assert _append(m, d, (1 << 31) - 128) == UNSUPPORTED


def test_attention_that_no_launch_holds(m):  # noqa: F811
    assert _attn(m, 1 << 23, 1 << 23, one) == UNSUPPORTED          # 2^24 workgroups of 256 threads, a token and KV head each
    assert _attn(m, 1 << 26, 1 << 26, None) == UNSUPPORTED         # 2^23 workgroups of 512, sixteen tokens and a KV head each


@no_gpu
def test_what_a_launch_just_holds(m):  # noqa: F811
    assert _append(m, 128, ((1 << 23) - 1) * 64) == HIP and _append(m, 64, ((1 << 24) - 1) * 64) == HIP
    assert _attn(m, (1 << 23) - 1, 1 << 23, one) == HIP and _attn(m, (1 << 26) - 16, 1 << 26, None) == HIP


@no_gpu
def test_scratch_for_a_few_tokens_is_enough(m):  # noqa: F811
    """Sequences of up to eight tokens alone, beside chunks and beside single tokens: the kernel that a call takes for them depends on all of it."""
    rng = random.Random(7)
    for i in range(300):
        hq, hkv, d = rng.choice([(32, 2, 128), (8, 2, 64), (16, 1, 64), (12, 4, 128), (16, 2, 128)])
        p = m.Params.make("bf16", hq, hkv, d, topk_total=8, n_init=1, n_local=1, dense_threshold=rng.choice([0, 1 << 30]))
        batch = rng.choice([1, 1, 2, 9, 70])
        news = [rng.choice([[4, 5, 8], [1, 8], [8, 9, 300], [4, 2000]][i % 4]) for _ in range(batch)]
        ctx = [max(n, int(400000 ** rng.random())) for n in news]
        cu = np.cumsum([0] + news).tolist()
        c = _cache(m, stride=(max(ctx) + 63) // 64, tok=d, head=64 * d, page=hkv * 64 * d)
        need = m.workspace_bytes(m.OP_CACHE_ATTN, p, batch, cu[-1], max(ctx))
        (_a, cu_h), (_b, cx) = _ints(cu), _ints(ctx)
        st = m.lib().infllmv2_cache_attn(ctypes.byref(p), ctypes.byref(c), one, cu_h, one, cx, one, batch, rng.choice([None, one]), one, None, one, need, None)
        assert st == HIP, (i, st, hq, hkv, d, news[:8], ctx[:8])
