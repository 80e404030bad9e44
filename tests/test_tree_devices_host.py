"""Trees of drafted tokens and page tables: tensors that are not on the device are refused before a call hands their addresses on.  No GPU is needed."""
import pytest
import torch

from test_cache_host import m  # noqa: F401

ints = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731


@pytest.fixture
def on_host(monkeypatch):
    """lengths and caches whose copies are on the host as well"""
    monkeypatch.setattr(torch.Tensor, "cuda", lambda x, *a, **k: x.clone())


def test_tensors_on_the_host(m, on_host):  # noqa: F811
    p = m.Params.make("bf16", 8, 2, 64)
    cu, ctx = m.SeqInfo([0, 5]), m.DecodeInfo([60])
    pages = torch.zeros((4, 2, 64, 64), dtype=torch.bfloat16)
    c = m.PagedCache(p, pages, pages.clone(), ints(1, 1))
    calls = [lambda: m.tree_masks(ints(5), cu, ctx),
             lambda: m.tree_masks(ints(5), cu, ctx, ints(5, 1), ints(5)),
             lambda: m.cache_tree_attn(p, c, torch.zeros((5, 8, 64), dtype=torch.bfloat16), cu, ctx, ints(5, 1)),
             lambda: m.cache_accept(p, c, cu, ctx, ints(1, 3)),
             lambda: m.cache_copy_pages(p, c, ints(2, 2)),
             lambda: m.PagePool(ints(4), ints(1, 1)),
             lambda: m.PagePool.empty(4, 1, 1, device="cpu")]
    for i, call in enumerate(calls):
        with pytest.raises(AssertionError):
            call()
            pytest.fail(f"call {i} went on")
