"""Rotary positions and the paged cache, what the host decides: frequency tables, refusals, sizes of scratch.  No GPU is needed (pointers here
are not device memory: a call that went on would fault)."""
import ctypes
import math
import random

import numpy as np
import pytest
import torch

INVALID, UNSUPPORTED, TOO_SMALL, HIP = -1, -2, -3, -4
one = ctypes.c_void_p(256)


@pytest.fixture(scope="module")
def m():
    import paper_2509_24663_amd as m
    m.lib()
    return m


def _ints(x):
    a = np.asarray(x, np.int32)
    return a, a.ctypes.data_as(ctypes.c_void_p)


def test_struct_layouts(m):
    import os
    import re

    from paper_2509_24663_amd import binding
    hdr = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "infllmv2.h")).read()
    for name, mirror, size in (("rotary", binding._RotaryC, 24), ("cache", binding._CacheC, 80)):
        body = re.search(r"typedef struct infllmv2_%s \{(.*?)\} infllmv2_%s;" % (name, name), hdr, re.S).group(1)
        body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
        fields = []
        for line in body.split(";"):
            names = re.findall(r"\*?\b([a-z_0-9]+)\s*(?=,|$)", line.strip())
            fields += names
        assert fields == [f[0] for f in mirror._fields_]
        assert ctypes.sizeof(mirror) == size


@pytest.mark.parametrize("scaling,factor", [("none", 1.0), ("linear", 4.0), ("base", 8.0), ("parts", 16.0)])
@pytest.mark.parametrize("rot_dim", [4, 50, 128])
def test_frequency_tables(m, rot_dim, scaling, factor):
    turns = m.rotary_turns(rot_dim, 10000.0, scaling, factor, original_len=4096, device="cpu").tolist()
    base = 10000.0 * factor ** (rot_dim / (rot_dim - 2)) if scaling == "base" else 10000.0
    for i, t in enumerate(turns):
        f = base ** (-2 * i / rot_dim) / (2 * math.pi)
        if scaling == "linear":
            f /= factor
        if scaling == "parts":
            keep = min(max((4096 * f - 1) / 31, 0), 1)
            f *= keep + (1 - keep) / factor
        # 64-bit arithmetic, a few roundings
        assert abs((t % 2 ** 64) / 2 ** 64 - f) <= 1e-14 * f + 2.0 ** -64
    if scaling == "base":       # the slowest pair is stretched by the factor
        assert abs(turns[-1] % 2 ** 64 * factor / (10000.0 ** (-(rot_dim - 2) / rot_dim) / (2 * math.pi) * 2 ** 64) - 1) < 1e-12


def test_frequency_table_refusals(m):
    buf = (ctypes.c_uint64 * 64)()
    f = lambda r=64, base=1e4, s=0, fac=1.0, n=4096.0, bf=32.0, bs=1.0, to=buf: m.lib().infllmv2_rotary_turns(r, base, s, fac, n, bf, bs, to)  # noqa: E731
    assert f() == 0
    for kw in (dict(r=0), dict(r=63), dict(r=-2), dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")), dict(fac=0.5), dict(to=None),
               dict(fac=float("inf")), dict(s=2, r=2), dict(s=3, n=0.0), dict(s=3, bs=0.0), dict(s=3, bf=1.0), dict(s=3, n=float("nan"))):
        assert f(**kw) == INVALID, kw
    assert f(s=4) == f(s=-1) == UNSUPPORTED


def test_rotary_refusals(m):
    from paper_2509_24663_amd import binding
    p = m.Params.make("bf16", 8, 2, 64)
    L = m.lib()

    def call(fn=L.infllmv2_rotary_fwd, p=p, r=(64, 0, 1.0, 0, 256), x=one, xt=512, xh=64, y=ctypes.c_void_p(1 << 20), yt=512, yh=64, pos=one, tokens=10, heads=8):
        rc = None if r is None else ctypes.byref(binding._RotaryC(*r))
        return fn(ctypes.byref(p), rc, x, xt, xh, y, yt, yh, pos, tokens, heads, None)

    bad = m.Params.make("bf16", 8, 2, 96)
    for fn in (L.infllmv2_rotary_fwd, L.infllmv2_rotary_bwd):
        assert call(fn, p=bad) == UNSUPPORTED
        for kw in (dict(r=None), dict(r=(0, 0, 1.0, 0, 256)), dict(r=(63, 0, 1.0, 0, 256)), dict(r=(66, 0, 1.0, 0, 256)), dict(r=(64, 0, 0.0, 0, 256)),
                   dict(r=(64, 0, float("nan"), 0, 256)), dict(r=(64, 0, 1.0, 1, 256)), dict(r=(64, 0, 1.0, 0, 260)), dict(r=(64, 0, 1.0, 0, 0)),
                   dict(x=None), dict(y=None), dict(pos=None), dict(tokens=-1), dict(heads=-1), dict(xt=-512), dict(yt=64), dict(yh=32), dict(yh=0),
                   dict(yt=500), dict(yt=512, yh=512), dict(x=one, y=one, xt=1024), dict(x=one, y=one, xh=128, yt=1024)):
            assert call(fn, **kw) == INVALID, kw
        assert call(fn, r=(64, 2, 1.0, 0, 256)) == UNSUPPORTED
        assert call(fn, tokens=1 << 40, yt=512, xt=0) == UNSUPPORTED
        assert call(fn, heads=2 ** 31 - 1, xt=1 << 50, yt=1 << 50) == UNSUPPORTED and call(fn, tokens=1 << 40, yt=1 << 40) == INVALID
        assert call(fn, tokens=0, x=None, y=None, pos=None) == 0 and call(fn, heads=0) == 0


def _cache(m, **over):
    from paper_2509_24663_amd import binding
    a = dict(kv_type=1, num_pages=10, k=256, v=256, page=2 * 64 * 64, head=64 * 64, tok=64, ks=256, vs=256, table=256, stride=4, reserved=0)
    a.update(over)
    return binding._CacheC(*a.values())


BAD_CACHES = [(dict(kv_type=2), UNSUPPORTED), (dict(num_pages=0), INVALID), (dict(k=0), INVALID), (dict(k=264), INVALID), (dict(page=63), INVALID),
              (dict(head=0), INVALID), (dict(tok=32), INVALID), (dict(tok=72), INVALID), (dict(kv_type=0, tok=68), INVALID), (dict(ks=0), INVALID),
              (dict(table=0), INVALID), (dict(stride=1), INVALID), (dict(reserved=1), INVALID)]
BAD_VALUES = [(dict(v=0), INVALID), (dict(v=257), INVALID), (dict(vs=0), INVALID)]


def test_append_refusals(m):
    from paper_2509_24663_amd import binding
    p = m.Params.make("bf16", 8, 2, 64)

    def call(cache=None, p=p, r=None, k=one, v=one, ts=64, hs=6400, cu=(0, 100), prev=(20,), batch=1, cu_d=one, prev_d=one):
        c = _cache(m, **(cache or {}))
        (_a, cu_h), (_b, pv_h) = _ints(cu), _ints(prev)
        return m.lib().infllmv2_cache_append(ctypes.byref(p), ctypes.byref(c), ctypes.byref(r) if r is not None else None, k, v, ts, hs, cu_h, cu_d,
                                             pv_h if prev else None, prev_d, None, batch, None)

    for over, want in BAD_CACHES + BAD_VALUES:
        assert call(over) == want, over
    assert m.lib().infllmv2_cache_append(ctypes.byref(p), None, None, one, one, 64, 6400, _ints([0, 5])[1], one, _ints([0])[1], one, None, 1, None) == INVALID
    for kw in (dict(k=None), dict(v=None), dict(ts=32), dict(hs=0), dict(cu=(1, 100)), dict(cu=(0, 50, 20), batch=2, prev=(0, 0)), dict(prev=(-1,)), dict(batch=-1),
               dict(prev=(200,)), dict(prev=(2 ** 31 - 50,)), dict(cu_d=None), dict(prev_d=None), dict(r=binding._RotaryC(66, 0, 1.0, 0, 256)),
               dict(r=binding._RotaryC(64, 0, 1.0, 0, 0))):
        assert call(**kw) == INVALID, kw
    assert call(p=m.Params.make("bf16", 8, 2, 96)) == UNSUPPORTED
    assert call(cu=(0, 0), k=None, v=None) == 0 and call(cu=(0,), prev=(), batch=0) == 0


def test_compress_refusals(m):
    p = m.Params.make("bf16", 8, 2, 64)

    def call(cache=None, kc=one, hs=64 * 100, prev=(20,), ctx=(200,), batch=1, dev=one):
        c = _cache(m, **(cache or {}))
        (_a, pv), (_b, cx) = _ints(prev), _ints(ctx)
        return m.lib().infllmv2_cache_compress_k(ctypes.byref(p), ctypes.byref(c), kc, hs, pv, dev, cx, dev, batch, None)

    for over, want in BAD_CACHES:
        assert call(over) == want, over
    for kw in (dict(kc=None), dict(hs=64), dict(prev=(201,)), dict(prev=(-1,)), dict(ctx=(2 ** 31 - 1,)), dict(batch=-1), dict(dev=None), dict(ctx=(300,))):
        assert call(**kw) == INVALID, kw
    assert call(prev=(33,), ctx=(47,), kc=None) == 0 and call(batch=0) == 0


def test_attention_refusals_and_scratch(m):
    p = m.Params.make("bf16", 8, 2, 64)

    def call(cache=None, p=p, q=one, out=one, cu=(0, 1), ctx=(200,), batch=1, ws=one, nbytes=1 << 30, dev=one):
        c = _cache(m, **(cache or {}))
        (_a, cu_h), (_b, cx) = _ints(cu), _ints(ctx)
        return m.lib().infllmv2_cache_attn(ctypes.byref(p), ctypes.byref(c), q, cu_h, dev, cx, dev, batch, None, out, None, ws, nbytes, None)

    for over, want in BAD_CACHES + BAD_VALUES:
        assert call(over) == want, over
    for kw in (dict(q=None), dict(out=None), dict(cu=(0, 201)), dict(ctx=(-1,)), dict(ctx=(257,)), dict(ctx=(2 ** 31 - 1,)), dict(batch=-1), dict(dev=None),
               dict(cu=(1, 2))):
        assert call(**kw) == INVALID, kw
    assert call(p=m.Params.make("bf16", 8, 2, 96)) == UNSUPPORTED
    assert call(cu=(0, 0), q=None, out=None) == 0 and call(batch=0, cu=(0,)) == 0
    # scratch: one sequence of 200 tokens needs none, one of 40000 does
    assert m.workspace_bytes(m.OP_CACHE_ATTN, p, 1, 1, 200) == 0
    need = m.workspace_bytes(m.OP_CACHE_ATTN, p, 1, 1, 40000)
    assert 0 < need <= 2048 * 16 * 66 * 4 + 256
    big = dict(stride=1000)
    assert call(big, ctx=(40000,), ws=None) == INVALID and call(big, ctx=(40000,), ws=ctypes.c_void_p(264)) == INVALID
    assert call(big, ctx=(40000,), nbytes=1024) == TOO_SMALL
    assert m.workspace_bytes(m.OP_CACHE_ATTN, m.Params.make("bf16", 8, 2, 96), 1, 1, 40000) == 0


@pytest.mark.skipif(torch.cuda.is_available(), reason="calls whose arguments are in order must end at the launch: no GPU")
def test_scratch_that_was_asked_for_is_enough(m):
    """The size from a batch's totals alone covers what any batch of these totals needs: single tokens, chunks, both, over lists and not."""
    rng = random.Random(3)
    for i in range(400):
        dtype, hq, hkv, d = rng.choice([("bf16", 32, 2, 128), ("bf16", 8, 2, 64), ("bf16", 5, 5, 64), ("fp32", 4, 1, 64), ("bf16", 16, 16, 128)])
        p = m.Params.make(dtype, hq, hkv, d, topk_total=rng.choice([4, 64, 1024]), n_init=1, n_local=1, dense_threshold=rng.choice([0, 4000, 1 << 30]))
        batch = rng.choice([1, 2, 7, 64, 700])
        far = rng.choice([100, 5000, 200000, 100000000])
        news = [rng.choice([0, 1, 1, 1, 3, 30, 200, 5000] if rng.random() < 0.5 else [1]) for _ in range(batch)]
        if rng.random() < 0.3:
            news = [1] * batch
        ctx = [max(n, int(far ** rng.random())) for n in news]
        cu = [0]
        for n in news:
            cu.append(cu[-1] + n)
        if cu[-1] == 0:
            continue
        c = _cache(m, stride=(max(ctx) + 63) // 64, tok=128, head=64 * 128, page=16 * 64 * 128)
        need = m.workspace_bytes(m.OP_CACHE_ATTN, p, batch, cu[-1], max(ctx))
        (_a, cu_h), (_b, cx) = _ints(cu), _ints(ctx)
        st = m.lib().infllmv2_cache_attn(ctypes.byref(p), ctypes.byref(c), one, cu_h, one, cx, one, batch, rng.choice([None, one]), one, None, one, need, None)
        assert st == HIP, (i, st, dtype, hq, hkv, d, news[:8], ctx[:8])


def test_decode_blocks_refusals(m):
    p = m.Params.make("bf16", 8, 2, 64)

    def call(p=p, q=one, kc=one, hs=64 * 100, ctx=(200,), batch=1, idx=one, ws=one, nbytes=1 << 30, dev=one):
        _a, cx = _ints(ctx)
        return m.lib().infllmv2_decode_blocks(ctypes.byref(p), q, kc, hs, cx, dev, batch, idx, ws, nbytes, None)

    for kw in (dict(q=None), dict(kc=None), dict(hs=64), dict(ctx=(0,)), dict(batch=-1), dict(idx=None), dict(ws=None), dict(ws=ctypes.c_void_p(8)), dict(dev=None)):
        assert call(**kw) == INVALID, kw
    assert call(nbytes=64) == TOO_SMALL and call(batch=0) == 0 and call(p=m.Params.make("bf16", 8, 2, 96)) == UNSUPPORTED
    assert m.workspace_bytes(m.OP_DECODE_BLOCKS, p, 4, 0, 5000) == m.decode_workspace_bytes(p, 4, 5000) > 0
