"""Trees of drafted tokens and page tables: one tensor of a call on the host, the others where they belong, or all on another device than the current one: refused."""
import pytest
import torch

from test_gpu_cache import _cache, _params, m  # noqa: F401

pytestmark = pytest.mark.gpu


def _calls(m):  # noqa: F811
    p = _params(m, "bf16", 8, 2, 64, topk_total=4, dense_threshold=0)
    cu, ctx = m.SeqInfo([0, 5]), m.DecodeInfo([400])
    c = _cache(m, p, [400], "e4m3", 1)
    pool = m.PagePool.empty(9, 2, 5)
    pool2 = m.PagePool.empty(9, 2, 5)
    forks = m.Forks([0], [1], [0])
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
    bf = lambda: torch.zeros((5, 8, 64), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    ws = torch.empty(m.workspace_bytes(m.OP_CACHE_TREE_ATTN, p, 1, 5, 400), dtype=torch.uint8, device="cuda")
    return [
        (lambda parents, mask, pos: m.tree_masks(parents, cu, ctx, mask, pos), [i32(5), i32(5, 1), i32(5)]),
        (lambda q, mask, idx, out, lse, ws: m.cache_tree_attn(p, c, q, cu, ctx, mask, idx, out, lse, ws),
         [bf(), i32(5, 1), i32(1, 2, 4), bf(), torch.zeros((5, 8), device="cuda"), ws]),
        (lambda path, lens: m.cache_accept(p, c, cu, ctx, path, lens), [i32(1, 3), i32(1)]),
        (lambda short: m.pages_resize(pool, [0, 0], [0, 0], short), [i32(1)]),
        (lambda copies, short: m.pages_fork(pool, forks, copies, short), [i32(1, 2), i32(1)]),
        (lambda moves, live: m.pages_compact(pool, [0, 0], None, moves, live), [i32(4, 2), i32(2)]),
        (lambda: m.pages_compact(pool, [0, 0], pool2), []),
        (lambda pairs: m.cache_copy_pages(p, c, pairs), [i32(2, 2)]),
        (lambda refs, table: m.PagePool(refs, table), [i32(9), i32(2, 5)]),
    ]


def test_one_tensor_on_the_host(m):  # noqa: F811
    for i, (call, tensors) in enumerate(_calls(m)):
        call(*tensors)
        for j in range(len(tensors)):
            with pytest.raises(AssertionError):
                call(*[x.cpu() if k == j else x for k, x in enumerate(tensors)])
                pytest.fail(f"call {i}, tensor {j}")


def test_parts_of_a_cache_on_the_host(m):  # noqa: F811
    p = _params(m, "bf16", 2, 2, 64)
    c = _cache(m, p, [400], "e4m3", 1)
    parts = [c.k, c.v, c.page_table, c.k_scale, c.v_scale]
    m.PagedCache(p, *parts)
    for j in range(5):
        with pytest.raises(AssertionError):
            m.PagedCache(p, *[x.cpu() if k == j else x for k, x in enumerate(parts)])


def test_another_device_is_the_current_one(m, monkeypatch):  # noqa: F811
    from paper_2509_24663_amd import binding
    calls = _calls(m)[:-1]                  # (a pool may be described while another device is the current one)
    monkeypatch.setattr(binding, "_current_device", lambda: 1)
    for i, (call, tensors) in enumerate(calls):
        with pytest.raises(AssertionError):
            call(*tensors)
            pytest.fail(f"call {i}")
