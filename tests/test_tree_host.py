"""Trees of drafted tokens and page tables, what the host decides: refusals, sizes of scratch.  No GPU is needed (pointers here are not device memory: a call
that went on would fault)."""
import ctypes
import os
import random
import re

import numpy as np
import pytest
import torch

from test_cache_host import BAD_CACHES, BAD_VALUES, HIP, INVALID, TOO_SMALL, UNSUPPORTED, _cache, _ints, m, one  # noqa: F401

no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="calls whose arguments are in order must end at the launch: no GPU")


def test_struct_layouts(m):  # noqa: F811
    from paper_2509_24663_amd import binding
    hdr = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "infllmv2.h")).read()
    body = re.sub(r"/\*.*?\*/", "", re.search(r"typedef struct infllmv2_pages \{(.*?)\} infllmv2_pages;", hdr, re.S).group(1), flags=re.S)
    fields = [x for line in body.split(";") for x in re.findall(r"\*?\b([a-z_0-9]+)\s*(?=,|$)", line.strip())]
    assert fields == [f[0] for f in binding._PagesC._fields_] and ctypes.sizeof(binding._PagesC) == 40
    assert re.search(r"typedef struct infllmv2_fork \{\s*int32_t src, dst, tokens, old_tokens;\s*\} infllmv2_fork;", hdr)
    assert m.TREE_MOST == int(re.search(r"INFLLMV2_TREE_MOST (\d+)", hdr).group(1))


def test_mask_refusals(m):  # noqa: F811
    def call(parents=one, cu=(0, 40), ctx=(100,), batch=1, mask=one, words=2, pos=one, cu_d=one, ctx_d=one):
        (_a, cu_h), (_b, cx) = _ints(cu), _ints(ctx)
        return m.lib().infllmv2_tree_masks(parents, cu_h, cu_d, cx if ctx else None, ctx_d, batch, mask, words, pos, None)

    for kw in (dict(parents=None), dict(mask=None), dict(cu=(1, 40)), dict(cu=(0, 40, 20), batch=2, ctx=(50, 50)), dict(batch=-1), dict(cu_d=None), dict(ctx_d=None),
               dict(ctx=()), dict(words=1), dict(words=-1), dict(words=0), dict(ctx=(39,)), dict(ctx=(2 ** 31 - 1,))):
        assert call(**kw) == INVALID, kw
    assert call(cu=(0, 1025), ctx=(2000,), words=33) == UNSUPPORTED
    assert call(words=4 * 65536) == UNSUPPORTED
    assert call(cu=(0, 0), parents=None, mask=None) == 0 and call(cu=(0,), batch=0) == 0


def test_outputs_over_inputs(m):  # noqa: F811
    """Lengths that a call reads are not where it writes the new ones, in whole or in part."""
    p, c = m.Params.make("bf16", 8, 2, 64), _cache(m)
    (_a, cu), (_b, cx) = _ints([0, 5, 9]), _ints([200, 100])
    apart = dict(cu=4096, ctx=8192, other=12288)          # (addresses of nothing: a refused call reads none)

    def accept(new):
        return m.lib().infllmv2_cache_accept(ctypes.byref(p), ctypes.byref(c), cu, apart["cu"], cx, apart["ctx"], 2, apart["other"], 4, new, None)

    def masks(pos):
        return m.lib().infllmv2_tree_masks(apart["other"], cu, apart["cu"], cx, apart["ctx"], 2, one, 1, pos, None)

    for call, others, mine in ((accept, 4 * 2 * 4, 4 * 2), (masks, 4 * 9, 4 * 9)):
        for name, size in (("cu", 4 * 3), ("ctx", 4 * 2), ("other", others)):
            for at in (apart[name], apart[name] + size - 4, apart[name] - mine + 4):
                assert call(at) == INVALID, (call.__name__, name, at)
            if not torch.cuda.is_available():
                for at in (apart[name] + size, apart[name] - mine):
                    assert call(at) == HIP, (call.__name__, name, at)


def test_accept_with_nothing_to_do(m):  # noqa: F811
    p, c = m.Params.make("bf16", 8, 2, 64), _cache(m)
    (_a, cu), (_b, cx) = _ints([0, 0]), _ints([200])
    assert m.lib().infllmv2_cache_accept(ctypes.byref(p), ctypes.byref(c), cu, one, cx, one, 1, None, 0, None, None) == 0


@no_gpu
def test_masks_without_positions_need_no_lengths(m):  # noqa: F811
    (_a, cu) = _ints([0, 40])
    assert m.lib().infllmv2_tree_masks(one, cu, one, None, None, 1, one, 2, None, None) == HIP


def test_attention_refusals_and_scratch(m):  # noqa: F811
    p = m.Params.make("bf16", 8, 2, 64)

    def call(cache=None, p=p, q=one, out=one, cu=(0, 5), ctx=(200,), batch=1, mask=one, words=1, idx=None, ws=one, nbytes=1 << 30, dev=one):
        c = _cache(m, **(cache or {}))
        (_a, cu_h), (_b, cx) = _ints(cu), _ints(ctx)
        return m.lib().infllmv2_cache_tree_attn(ctypes.byref(p), ctypes.byref(c), q, cu_h, dev, cx, dev, batch, mask, words, idx, out, None, ws, nbytes, None)

    for over, want in BAD_CACHES + BAD_VALUES + [(dict(tok=(1 << 24) + 64), UNSUPPORTED)]:
        assert call(over) == want, over
    for kw in (dict(q=None), dict(out=None), dict(mask=None), dict(words=0), dict(words=-3), dict(cu=(0, 33)), dict(cu=(0, 201), words=7), dict(ctx=(-1,)), dict(ctx=(257,)),
               dict(ctx=(2 ** 31 - 1,)), dict(batch=-1), dict(dev=None), dict(cu=(1, 2))):
        assert call(**kw) == INVALID, kw
    assert call(p=m.Params.make("bf16", 8, 2, 96)) == UNSUPPORTED
    assert call(cu=(0, 0), q=None, out=None, mask=None) == 0 and call(batch=0, cu=(0,)) == 0
    need = m.workspace_bytes(m.OP_CACHE_TREE_ATTN, p, 1, 5, 40000)
    assert need == m.workspace_bytes(m.OP_CACHE_ATTN, p, 1, 5, 40000) > 0
    big = dict(stride=1000)
    assert call(big, ctx=(40000,), ws=None) == INVALID and call(big, ctx=(40000,), ws=ctypes.c_void_p(264)) == INVALID
    assert call(big, ctx=(40000,), nbytes=1024) == TOO_SMALL


@no_gpu
def test_scratch_that_was_asked_for_is_enough(m):  # noqa: F811
    rng = random.Random(5)
    for i in range(400):
        dtype, hq, hkv, d = rng.choice([("bf16", 32, 2, 128), ("bf16", 8, 2, 64), ("bf16", 5, 5, 64), ("fp32", 4, 1, 64), ("bf16", 16, 16, 128)])
        p = m.Params.make(dtype, hq, hkv, d, topk_total=rng.choice([4, 64, 1024]), n_init=1, n_local=1, dense_threshold=rng.choice([0, 4000, 1 << 30]))
        batch, far = rng.choice([1, 2, 7, 64, 700]), rng.choice([100, 5000, 200000, 100000000])
        news = [rng.choice([0, 1, 3, 8, 9, 26, 64, 300]) for _ in range(batch)]
        if i % 2:                                        # trees of one size
            news = [rng.choice([1, 5, 8, 9, 26, 64, 300])] * batch
        ctx = [max(n, int(far ** rng.random())) for n in news]
        if i % 4 == 1:
            ctx = [max(ctx)] * batch
        cu = np.concatenate([[0], np.cumsum(news)]).tolist()
        if cu[-1] == 0:
            continue
        c = _cache(m, stride=(max(ctx) + 63) // 64, tok=128, head=64 * 128, page=16 * 64 * 128)
        need = m.workspace_bytes(m.OP_CACHE_TREE_ATTN, p, batch, cu[-1], max(ctx))
        (_a, cu_h), (_b, cx) = _ints(cu), _ints(ctx)
        st = m.lib().infllmv2_cache_tree_attn(ctypes.byref(p), ctypes.byref(c), one, cu_h, one, cx, one, batch, one, 10, rng.choice([None, one]), one, None, one, need, None)
        assert st == HIP, (i, st, dtype, hq, hkv, d, news[:8], ctx[:8])


def test_accept_refusals(m):  # noqa: F811
    p = m.Params.make("bf16", 8, 2, 64)

    def call(cache=None, p=p, cu=(0, 5), ctx=(200,), batch=1, path=one, stride=4, dev=one):
        c = _cache(m, **(cache or {}))
        (_a, cu_h), (_b, cx) = _ints(cu), _ints(ctx)
        return m.lib().infllmv2_cache_accept(ctypes.byref(p), ctypes.byref(c), cu_h, dev, cx, dev, batch, path, stride, None, None)

    for over, want in BAD_CACHES + BAD_VALUES:
        assert call(over) == want, over
    for kw in (dict(path=None), dict(stride=0), dict(stride=-1), dict(cu=(0, 201)), dict(ctx=(-1,)), dict(ctx=(257,)), dict(ctx=(2 ** 31 - 1,)), dict(batch=-1), dict(dev=None),
               dict(cu=(1, 2))):
        assert call(**kw) == INVALID, kw
    assert call(p=m.Params.make("bf16", 8, 2, 96)) == UNSUPPORTED
    assert call(batch=0, cu=(0,)) == 0


def _pages(**over):
    from paper_2509_24663_amd import binding
    a = dict(num_pages=10, rows=4, blocks=5, stride=5, table=256, refs=512, reserved=0)
    a.update(over)
    return binding._PagesC(*a.values())


BAD_PAGES = [dict(num_pages=0), dict(rows=0), dict(blocks=0), dict(stride=4), dict(table=0), dict(refs=0), dict(reserved=1)]


def test_resize_refusals(m):  # noqa: F811
    def call(pages=None, old=(0, 64), new=(320, 0), batch=2, dev=one):
        (_a, o), (_b, n) = _ints(old), _ints(new)
        return m.lib().infllmv2_pages_resize(ctypes.byref(_pages(**(pages or {}))), o, dev, n, dev, batch, None, None)

    for over in BAD_PAGES:
        assert call(over) == INVALID, over
    assert m.lib().infllmv2_pages_resize(None, None, None, None, None, 0, None, None) == INVALID
    for kw in (dict(batch=-1), dict(batch=5, old=[0] * 5, new=[0] * 5), dict(dev=None), dict(new=(321, 0)), dict(old=(321, 0)), dict(old=(-1, 0)), dict(new=(0, -1)),
               dict(new=(2 ** 31 - 1, 0))):
        assert call(**kw) == INVALID, kw
    assert call(batch=0) == 0 and call(old=(1, 64), new=(64, 2)) == 0           # (nothing changes hands, nothing is reported)
    assert call(dict(rows=5000), old=[0] * 4097, new=[0] * 4097, batch=4097) == UNSUPPORTED


def test_fork_refusals(m):  # noqa: F811
    def call(forks, pages=None, count=None, dev=one):
        a = np.asarray(forks, np.int32).reshape(-1, 4)
        return m.lib().infllmv2_pages_fork(ctypes.byref(_pages(**(pages or {}))), a.ctypes.data_as(ctypes.c_void_p), dev, len(a) if count is None else count, None, None, None)

    fine = [(0, 1, 100, 0), (0, 2, 320, 64)]
    for over in BAD_PAGES:
        assert call(fine, over) == INVALID, over
    for forks in ([(0, 0, 10, 0)], [(0, 1, 10, 0), (2, 1, 10, 0)], [(0, 1, 10, 0), (1, 2, 10, 0)], [(-1, 1, 10, 0)], [(4, 1, 10, 0)], [(0, 4, 10, 0)], [(0, -1, 10, 0)],
                  [(0, 1, -1, 0)], [(0, 1, 321, 0)], [(0, 1, 10, 321)], [(0, 1, 10, -5)]):
        assert call(forks) == INVALID, forks
    assert call(fine, count=-1) == INVALID and call(fine, dev=None) == INVALID and call(fine, dev=ctypes.c_void_p(264)) == INVALID
    assert call(fine, dict(rows=4097)) == UNSUPPORTED
    assert call(fine, count=0) == 0 and call([(0, 1, 0, 0)]) == 0


def test_compact_and_copy_refusals(m):  # noqa: F811
    def call(pages=None, out=None, lens=(320, 1), batch=2, moves=one, live=one, dev=one):
        _a, n = _ints(lens)
        return m.lib().infllmv2_pages_compact(ctypes.byref(_pages(**(pages or {}))), n, dev, batch, ctypes.byref(_pages(**(out or {}))), moves, live, None)

    for over in BAD_PAGES:
        assert call(over) == INVALID and call(out=over) == INVALID, over
    for kw in (dict(batch=-1), dict(batch=5, lens=[0] * 5), dict(lens=(321, 0)), dict(lens=(-1, 0)), dict(moves=None), dict(live=None), dict(dev=None),
               dict(out=dict(num_pages=9)), dict(out=dict(rows=1)), dict(out=dict(blocks=4, table=1024)), dict(out=dict(stride=6))):
        assert call(**kw) == INVALID, kw
    p = m.Params.make("bf16", 8, 2, 64)

    def copy(cache=None, p=p, pairs=one, count=3):
        return m.lib().infllmv2_cache_copy_pages(ctypes.byref(p), ctypes.byref(_cache(m, **(cache or {}))), pairs, count, None)

    for over, want in [x for x in BAD_CACHES if x[0] != dict(stride=1)] + BAD_VALUES:
        assert copy(over) == want, over
    assert copy(pairs=None) == copy(count=-1) == INVALID and copy(p=m.Params.make("bf16", 8, 2, 96)) == UNSUPPORTED
    assert copy(count=0, pairs=None) == 0 and copy(count=(1 << 24)) == UNSUPPORTED
