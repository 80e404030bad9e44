"""ctypes binding of libinfllmv2.so: argument marshalling only, one function per C entry point."""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libinfllmv2.so")

FP32, BF16 = 0, 1


class InfllmV2Error(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


class Params(ctypes.Structure):
    """Mirror of `infllmv2_params` (paper notation: Sec. 3.2, 3.3, 4.1)."""

    _fields_ = [
        ("dtype", ctypes.c_int32), ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("block_size", ctypes.c_int32), ("cmp_len", ctypes.c_int32),
        ("cmp_stride", ctypes.c_int32), ("pool_len", ctypes.c_int32), ("pool_stride", ctypes.c_int32),
        ("pool_pad", ctypes.c_int32), ("n_init", ctypes.c_int32), ("n_local", ctypes.c_int32),
        ("topk_total", ctypes.c_int32), ("dense_threshold", ctypes.c_int32), ("softmax_scale", ctypes.c_float),
        ("lse_mode", ctypes.c_int32),
    ]

    @staticmethod
    def make(dtype: str, num_q_heads: int, num_kv_heads: int, head_dim: int, *, block_size=64, cmp_len=32,
             cmp_stride=16, pool_len=5, pool_stride=4, pool_pad=0, n_init=1, n_local=8, topk_total=64,
             dense_threshold=0, softmax_scale: Optional[float] = None, lse_mode=0) -> "Params":
        scale = float(head_dim) ** -0.5 if softmax_scale is None else float(softmax_scale)
        return Params({"fp32": FP32, "bf16": BF16}[dtype], num_q_heads, num_kv_heads, head_dim, block_size, cmp_len,
                      cmp_stride, pool_len, pool_stride, pool_pad, n_init, n_local, topk_total, dense_threshold,
                      scale, lse_mode)

    @staticmethod
    def from_config(cfg, **over) -> "Params":
        kw = dict(block_size=cfg.block_size, cmp_len=cfg.cmp_len, cmp_stride=cfg.cmp_stride,
                  pool_len=cfg.pool_len, pool_stride=cfg.pool_stride, pool_pad=cfg.pool_pad, n_init=cfg.n_init,
                  n_local=cfg.n_local, topk_total=cfg.topk_total, dense_threshold=cfg.dense_threshold,
                  softmax_scale=cfg.softmax_scale)
        kw.update(over)
        return Params.make(cfg.dtype, cfg.num_q_heads, cfg.num_kv_heads, cfg.head_dim, **kw)

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == BF16 else torch.float32


_lib = None
_P = ctypes.c_void_p
_I32, _I64, _SZ = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
_PP = ctypes.POINTER(Params)
_DBL = ctypes.c_double


class _RotaryC(ctypes.Structure):
    """Mirror of `infllmv2_rotary`."""

    _fields_ = [("rot_dim", ctypes.c_int32), ("layout", ctypes.c_int32), ("magnitude", ctypes.c_float),
                ("reserved", ctypes.c_int32), ("turns_d", ctypes.c_void_p)]


class _CacheC(ctypes.Structure):
    """Mirror of `infllmv2_cache`."""

    _fields_ = [("kv_type", ctypes.c_int32), ("num_pages", ctypes.c_int32), ("k_d", ctypes.c_void_p), ("v_d", ctypes.c_void_p),
                ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("tok_stride", ctypes.c_int64),
                ("k_scale_d", ctypes.c_void_p), ("v_scale_d", ctypes.c_void_p), ("page_table_d", ctypes.c_void_p),
                ("table_stride", ctypes.c_int32), ("reserved", ctypes.c_int32)]


_RP, _CP = ctypes.POINTER(_RotaryC), ctypes.POINTER(_CacheC)

_SIGNATURES = {
    "infllmv2_num_cmp": (_I32, [_PP, _I32]),
    "infllmv2_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "infllmv2_version": (ctypes.c_char_p, []),
    "infllmv2_compress_k": (ctypes.c_int, [_PP, _P, _I64, _I64, _P, _P, _I32, _P, _P, _I64, _P]),
    "infllmv2_compress_k_append": (ctypes.c_int, [_PP, _P, _I64, _I64, _I64, _P, _I64, _P, _P, _P, _P, _I32, _P]),
    "infllmv2_workspace_bytes": (_SZ, [ctypes.c_int, _PP, _I32, _I64, _I32]),
    "infllmv2_block_scores": (ctypes.c_int, [_PP, _P, _P, _I64, _P, _P, _P, _I32, _P, _I64, _P, _SZ, _P]),
    "infllmv2_topk_blocks": (ctypes.c_int, [_PP, _P, _I64, _P, _P, _I32, _P, _P]),
    "infllmv2_block_scores_pooled": (ctypes.c_int, [_PP, _P, _P, _I64, _P, _P, _P, _I32, _P, _I64, _P, _SZ, _P]),
    "infllmv2_topk_pooled": (ctypes.c_int, [_PP, _P, _I64, _P, _P, _I32, _P, _P]),
    "infllmv2_sparse_attn_fwd": (ctypes.c_int, [_PP, _P, _P, _P, _I64, _I64, _P, _P, _P, _I32, _P, _P, _P, _SZ, _P]),
    "infllmv2_dense_attn_fwd": (ctypes.c_int, [_PP, _P, _P, _P, _I64, _I64, _P, _P, _I32, _P, _P, _P, _SZ, _P]),
    "infllmv2_sparse_attn_bwd": (ctypes.c_int, [_PP, _P, _P, _P, _I64, _I64, _P, _P, _P, _P, _P, _P, _I32, _P, _P, _P,
                                                _P, _SZ, _P]),
    "infllmv2_sparse_decode": (ctypes.c_int, [_PP, _P, _P, _P, _I64, _I64, _I64, _P, _I64, _P, _P, _I32, _P, _P, _P,
                                              _P, _SZ, _P]),
    "infllmv2_decode_workspace_bytes": (_SZ, [_PP, _I32, _I32]),
    "infllmv2_sparse_decode_static": (ctypes.c_int, [_PP, _P, _P, _P, _I64, _I64, _I64, _P, _I64, _P, _P, _I32, _P, _P, _P,
                                                     _P]),
    "infllmv2_sparse_decode_static_capacity": (_SZ, []),
    "infllmv2_rotary_turns": (ctypes.c_int, [_I32, _DBL, _I32, _DBL, _DBL, _DBL, _DBL, _P]),
    "infllmv2_rotary_fwd": (ctypes.c_int, [_PP, _RP, _P, _I64, _I64, _P, _I64, _I64, _P, _I64, _I32, _P]),
    "infllmv2_rotary_bwd": (ctypes.c_int, [_PP, _RP, _P, _I64, _I64, _P, _I64, _I64, _P, _I64, _I32, _P]),
    "infllmv2_cache_append": (ctypes.c_int, [_PP, _CP, _RP, _P, _P, _I64, _I64, _P, _P, _P, _P, _P, _I32, _P]),
    "infllmv2_cache_compress_k": (ctypes.c_int, [_PP, _CP, _P, _I64, _P, _P, _P, _P, _I32, _P]),
    "infllmv2_decode_blocks": (ctypes.c_int, [_PP, _P, _P, _I64, _P, _P, _I32, _P, _P, _SZ, _P]),
    "infllmv2_cache_attn": (ctypes.c_int, [_PP, _CP, _P, _P, _P, _P, _P, _I32, _P, _P, _P, _P, _SZ, _P]),
}


def lib() -> ctypes.CDLL:
    """Load libinfllmv2.so (no fallback: a missing library is an error)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"{_LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'` "
                              "(or python paper_2509_24663_amd/build.py) first; there is no CPU fallback")
        L = ctypes.CDLL(_LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


def exported_symbols() -> Sequence[str]:
    return tuple(_SIGNATURES)


def status_string(status: int) -> str:
    return lib().infllmv2_status_string(int(status)).decode()


def version() -> str:
    return lib().infllmv2_version().decode()


def num_cmp(p: Params, n: int) -> int:
    return int(lib().infllmv2_num_cmp(ctypes.byref(p), int(n)))


def _check(st: int, where: str):
    if st != 0:
        raise InfllmV2Error(st, where)


# Addresses and the stream go over as plain integers: the signatures convert them, and a wrapper object per argument, or a
# torch.cuda.Stream per call (2.9 us of the 8 to 13 that a call took on the host; its number alone 0.1), is what short
# prompts and small decode steps wait for.
def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)      # (not part of torch's documented interface)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream():
    if _raw_stream is None or _device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device())


# `op` of infllmv2_workspace_bytes (enum infllmv2_op)
OP_COMPRESS_K, OP_BLOCK_SCORES, OP_TOPK_BLOCKS, OP_SPARSE_ATTN_FWD, OP_DENSE_ATTN_FWD, OP_SPARSE_DECODE = range(6)
OP_BLOCK_SCORES_POOLED, OP_TOPK_POOLED, OP_SPARSE_ATTN_BWD, OP_SPARSE_ATTN_BWD_MIN, OP_COMPRESS_K_APPEND = range(6, 11)
OP_CACHE_ATTN, OP_DECODE_BLOCKS = 11, 12


def workspace_bytes(op: int, p: Params, batch: int, total_tokens: int, max_seqlen: int) -> int:
    """Bytes of scratch call `op` needs at most for such a batch (host helper, no GPU needed)."""
    return int(lib().infllmv2_workspace_bytes(int(op), ctypes.byref(p), int(batch), int(total_tokens), int(max_seqlen)))


def _workspace(op: int, p: Params, si: "SeqInfo", device, given: Optional[torch.Tensor]):
    """The caller's scratch tensor, or a new one of the size the library asks for (None when it asks for none)."""
    if given is not None:
        return given
    need = workspace_bytes(op, p, si.batch, si.total, si.max_len)
    return torch.empty(need, dtype=torch.uint8, device=device) if need else None


def _ws_args(ws: Optional[torch.Tensor]):
    return (None, 0) if ws is None else (ws.data_ptr(), ws.numel() * ws.element_size())


class SeqInfo:
    """cu_seqlens as the ABI wants it: a host int32 array plus a device copy, made once and reused."""

    def __init__(self, cu_seqlens):
        self.cu_h = torch.as_tensor(cu_seqlens, dtype=torch.int32, device="cpu").contiguous()
        self.cu_d = self.cu_h.cuda()
        self.batch = self.cu_h.numel() - 1
        lens = (self.cu_h[1:] - self.cu_h[:-1])
        self.lens = lens.tolist()
        self.max_len = int(lens.max()) if self.batch else 0
        self.total = int(self.cu_h[-1])


def _seq_info(cu_seqlens) -> SeqInfo:
    """pass a SeqInfo to avoid the copy to the device on every call"""
    return cu_seqlens if isinstance(cu_seqlens, SeqInfo) else SeqInfo(cu_seqlens)


def _kv_strides(k: torch.Tensor):
    """k is [hkv, T, d] (head-major) or any view with d contiguous: returns (tok_stride, head_stride)."""
    assert k.dim() == 3 and k.stride(2) == 1
    return k.stride(1), k.stride(0)


# ---------------------------------------------------------------------------------- stage wrappers
def compress_k(p: Params, k: torch.Tensor, cu_seqlens, out=None):
    """Stage 1.  k [hkv, T, d] (device).  Returns kc [hkv, total_c, d] fp32, cu_seqlens_c (device int32).
    out: optional (kc, cu_seqlens_c) buffers to reuse."""
    si = _seq_info(cu_seqlens)
    cu_h, cu_d, batch = si.cu_h, si.cu_d, si.batch
    if out is None:
        total_c = sum(num_cmp(p, n) for n in si.lens)
        kc = torch.empty((p.num_kv_heads, max(total_c, 1), p.head_dim), dtype=torch.float32, device=k.device)
        cu_c = torch.empty(batch + 1, dtype=torch.int32, device=k.device)
    else:
        kc, cu_c = out
    ts, hs = _kv_strides(k)
    st = lib().infllmv2_compress_k(ctypes.byref(p), _ptr(k), ts, hs, _ptr(cu_h), _ptr(cu_d), batch, _ptr(kc),
                                   _ptr(cu_c), kc.shape[1], _stream())
    _check(st, "infllmv2_compress_k")
    return kc, cu_c


def compress_k_append(p: Params, k_cache: torch.Tensor, kc_cache: torch.Tensor, prev_lens, ctx_lens):
    """Brings a decode compressed-key cache up to date in place.  k_cache [B, hkv, Lmax, d]; kc_cache
    [B, hkv, max_nc, d] fp32; prev_lens / ctx_lens: sequences of ints or DecodeInfo (cache lengths then and now)."""
    pv = prev_lens if isinstance(prev_lens, DecodeInfo) else DecodeInfo(prev_lens)
    cx = ctx_lens if isinstance(ctx_lens, DecodeInfo) else DecodeInfo(ctx_lens)
    assert k_cache.dim() == 4 and k_cache.stride(3) == 1 and kc_cache.dim() == 4 and kc_cache.is_contiguous()
    st = lib().infllmv2_compress_k_append(ctypes.byref(p), _ptr(k_cache), k_cache.stride(0), k_cache.stride(1),
                                          k_cache.stride(2), _ptr(kc_cache), kc_cache.stride(1), _ptr(pv.ctx_h),
                                          _ptr(pv.ctx_d), _ptr(cx.ctx_h), _ptr(cx.ctx_d), cx.batch, _stream())
    _check(st, "infllmv2_compress_k_append")
    return kc_cache


def block_scores(p: Params, q: torch.Tensor, kc: torch.Tensor, cu_seqlens, cu_seqlens_c: torch.Tensor,
                 out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Stage 2.  q [T, hq, d]; returns S^shared [hkv, T, row_stride] fp32 (entries beyond v(t) unspecified).
    workspace: a uint8 device tensor of workspace_bytes(OP_BLOCK_SCORES, ...) bytes to reuse (else made here)."""
    assert q.is_contiguous() and kc.is_contiguous()
    si = _seq_info(cu_seqlens)
    cu_h, cu_d, batch = si.cu_h, si.cu_d, si.batch
    if out is None:
        rs = max(4, (num_cmp(p, si.max_len) + 3) // 4 * 4)
        out = torch.empty((p.num_kv_heads, q.shape[0], rs), dtype=torch.float32, device=q.device)
    ws = _workspace(OP_BLOCK_SCORES, p, si, q.device, workspace)
    st = lib().infllmv2_block_scores(ctypes.byref(p), _ptr(q), _ptr(kc), kc.shape[1], _ptr(cu_h), _ptr(cu_d),
                                     _ptr(cu_seqlens_c), batch, _ptr(out), out.shape[2], *_ws_args(ws), _stream())
    _check(st, "infllmv2_block_scores")
    return out


def topk_blocks(p: Params, s_shared: torch.Tensor, cu_seqlens, out: Optional[torch.Tensor] = None):
    """Stage 3.  s_shared [hkv, T, row_stride] -> block_idx [hkv, T, topk_total] int32."""
    si = _seq_info(cu_seqlens)
    cu_h, cu_d, batch = si.cu_h, si.cu_d, si.batch
    if out is None:
        out = torch.empty((p.num_kv_heads, s_shared.shape[1], p.topk_total), dtype=torch.int32, device=s_shared.device)
    st = lib().infllmv2_topk_blocks(ctypes.byref(p), _ptr(s_shared), s_shared.shape[2], _ptr(cu_h), _ptr(cu_d), batch,
                                    _ptr(out), _stream())
    _check(st, "infllmv2_topk_blocks")
    return out


def block_scores_pooled(p: Params, q: torch.Tensor, kc: torch.Tensor, cu_seqlens, cu_seqlens_c: torch.Tensor,
                        out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Stages 2 with the max-pooling fused.  Returns S^cmp [hkv, T, row_stride >= ceil(max len / 64)] fp32; entry j of
    a row is written iff the block's pooling window holds a visible key."""
    si = _seq_info(cu_seqlens)
    cu_h, cu_d, batch = si.cu_h, si.cu_d, si.batch
    if out is None:
        rs = max(1, (si.max_len + p.block_size - 1) // p.block_size)
        out = torch.empty((p.num_kv_heads, q.shape[0], rs), dtype=torch.float32, device=q.device)
    assert q.is_contiguous() and kc.is_contiguous()
    ws = _workspace(OP_BLOCK_SCORES_POOLED, p, si, q.device, workspace)
    st = lib().infllmv2_block_scores_pooled(ctypes.byref(p), _ptr(q), _ptr(kc), kc.shape[1], _ptr(cu_h), _ptr(cu_d),
                                            _ptr(cu_seqlens_c), batch, _ptr(out), out.shape[2], *_ws_args(ws),
                                            _stream())
    _check(st, "infllmv2_block_scores_pooled")
    return out


def topk_pooled(p: Params, s_cmp: torch.Tensor, cu_seqlens, out: Optional[torch.Tensor] = None):
    """Stage 3 on pooled scores.  s_cmp [hkv, T, row_stride] -> block_idx [hkv, T, topk_total] int32."""
    si = _seq_info(cu_seqlens)
    cu_h, cu_d, batch = si.cu_h, si.cu_d, si.batch
    if out is None:
        out = torch.empty((p.num_kv_heads, s_cmp.shape[1], p.topk_total), dtype=torch.int32, device=s_cmp.device)
    st = lib().infllmv2_topk_pooled(ctypes.byref(p), _ptr(s_cmp), s_cmp.shape[2], _ptr(cu_h), _ptr(cu_d), batch,
                                    _ptr(out), _stream())
    _check(st, "infllmv2_topk_pooled")
    return out


def sparse_attn_fwd(p: Params, q, k, v, block_idx, cu_seqlens, out=None, lse=None, workspace=None):
    """Stage 4.  Returns (out [T, hq, d], lse [hq, T]).  workspace: scratch tensor to reuse (else made here)."""
    si = _seq_info(cu_seqlens)
    cu_h, cu_d, batch = si.cu_h, si.cu_d, si.batch
    out = torch.empty_like(q) if out is None else out
    lse = torch.empty((p.num_q_heads, q.shape[0]), dtype=torch.float32, device=q.device) if lse is None else lse
    ts, hs = _kv_strides(k)
    assert _kv_strides(v) == (ts, hs)
    assert q.is_contiguous() and out.is_contiguous() and lse.is_contiguous() and block_idx.is_contiguous()
    ws = _workspace(OP_SPARSE_ATTN_FWD, p, si, q.device, workspace)
    st = lib().infllmv2_sparse_attn_fwd(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), ts, hs, _ptr(block_idx),
                                        _ptr(cu_h), _ptr(cu_d), batch, _ptr(out), _ptr(lse), *_ws_args(ws), _stream())
    _check(st, "infllmv2_sparse_attn_fwd")
    return out, lse


def dense_attn_fwd(p: Params, q, k, v, cu_seqlens, out=None, lse=None, workspace=None):
    """Dense causal GQA attention.  Returns (out [T, hq, d], lse [hq, T])."""
    si = _seq_info(cu_seqlens)
    cu_h, cu_d, batch = si.cu_h, si.cu_d, si.batch
    out = torch.empty_like(q) if out is None else out
    lse = torch.empty((p.num_q_heads, q.shape[0]), dtype=torch.float32, device=q.device) if lse is None else lse
    ts, hs = _kv_strides(k)
    assert _kv_strides(v) == (ts, hs)
    assert q.is_contiguous() and out.is_contiguous() and lse.is_contiguous()
    ws = _workspace(OP_DENSE_ATTN_FWD, p, si, q.device, workspace)
    st = lib().infllmv2_dense_attn_fwd(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), ts, hs, _ptr(cu_h), _ptr(cu_d),
                                       batch, _ptr(out), _ptr(lse), *_ws_args(ws), _stream())
    _check(st, "infllmv2_dense_attn_fwd")
    return out, lse


def sparse_attn_bwd(p: Params, q, k, v, block_idx, out, lse, dout, cu_seqlens, dq=None, dk=None, dv=None,
                    workspace=None, sel_bitmap_max_bytes: int = 512 << 20):
    """Gradients of stage 4 for a given selection (block_idx None: dense).  Returns (dq like q, dk, dv float32
    [hkv, T, d]).  workspace: scratch tensor to reuse; when it is made here it includes room for the selection
    bitmap unless that would take more than sel_bitmap_max_bytes (0: never)."""
    si = _seq_info(cu_seqlens)
    cu_h, cu_d, batch = si.cu_h, si.cu_d, si.batch
    ts, hs = _kv_strides(k)
    assert _kv_strides(v) == (ts, hs)
    T = q.shape[0]
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty((p.num_kv_heads, T, p.head_dim), dtype=torch.float32, device=q.device) if dk is None else dk
    dv = torch.empty((p.num_kv_heads, T, p.head_dim), dtype=torch.float32, device=q.device) if dv is None else dv
    assert dout.is_contiguous() and out.is_contiguous() and dq.is_contiguous() and dk.is_contiguous() and dv.is_contiguous()
    assert q.is_contiguous() and lse.is_contiguous()
    if workspace is None:
        full = workspace_bytes(OP_SPARSE_ATTN_BWD, p, batch, T, si.max_len)
        least = workspace_bytes(OP_SPARSE_ATTN_BWD_MIN, p, batch, T, si.max_len)
        need = full if block_idx is not None and full - least <= sel_bitmap_max_bytes else least
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    st = lib().infllmv2_sparse_attn_bwd(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), ts, hs, _ptr(block_idx), _ptr(out),
                                        _ptr(lse), _ptr(dout), _ptr(cu_h), _ptr(cu_d), batch, _ptr(dq), _ptr(dk),
                                        _ptr(dv), *_ws_args(workspace), _stream())
    _check(st, "infllmv2_sparse_attn_bwd")
    return dq, dk, dv


def decode_workspace_bytes(p: Params, batch: int, max_ctx_len: int) -> int:
    return int(lib().infllmv2_decode_workspace_bytes(ctypes.byref(p), int(batch), int(max_ctx_len)))


class DecodeInfo:
    """ctx_lens as the ABI wants them (host + device copy), made once per step and reusable."""

    def __init__(self, ctx_lens):
        self.ctx_h = torch.as_tensor(ctx_lens, dtype=torch.int32, device="cpu").contiguous()
        self.ctx_d = self.ctx_h.cuda()
        self.batch = self.ctx_h.numel()
        self.max_ctx = int(self.ctx_h.max()) if self.batch else 0


def sparse_decode(p: Params, q, k_cache, v_cache, kc_cache, ctx_lens, workspace=None, return_idx=True, out=None,
                  lse=None, idx=None):
    """Decode step.  q [B, hq, d]; k_cache/v_cache [B, hkv, Lmax, d]; kc_cache [B, hkv, max_nc, d] fp32.
    ctx_lens: a sequence of ints or a DecodeInfo.  out / lse / idx / workspace: optional buffers to reuse.
    Returns (out [B, hq, d], lse [B, hq], block_idx [B, hkv, topk_total] or None)."""
    di = ctx_lens if isinstance(ctx_lens, DecodeInfo) else DecodeInfo(ctx_lens)
    B = q.shape[0]
    if workspace is None:
        workspace = torch.empty(max(decode_workspace_bytes(p, B, di.max_ctx), 256), dtype=torch.uint8, device=q.device)
    out = torch.empty_like(q) if out is None else out
    lse = torch.empty((B, p.num_q_heads), dtype=torch.float32, device=q.device) if lse is None else lse
    if idx is None and return_idx:
        idx = torch.empty((B, p.num_kv_heads, p.topk_total), dtype=torch.int32, device=q.device)
    assert k_cache.dim() == 4 and k_cache.stride(3) == 1 and k_cache.stride() == v_cache.stride()
    assert kc_cache.dim() == 4 and kc_cache.is_contiguous()
    st = lib().infllmv2_sparse_decode(ctypes.byref(p), _ptr(q), _ptr(k_cache), _ptr(v_cache), k_cache.stride(0),
                                      k_cache.stride(1), k_cache.stride(2), _ptr(kc_cache), kc_cache.stride(1),
                                      _ptr(di.ctx_h), _ptr(di.ctx_d), B, _ptr(idx), _ptr(out), _ptr(lse),
                                      _ptr(workspace), workspace.numel(), _stream())
    _check(st, "infllmv2_sparse_decode")
    return out, lse, idx


def sparse_decode_static_capacity() -> int:
    return int(lib().infllmv2_sparse_decode_static_capacity())


def sparse_decode_static(p: Params, q, k_cache, v_cache, kc_cache, ctx_lens, out, lse, idx=None):
    """Decode step through the entry point that allocates nothing: scratch is a fixed array inside the library, and
    every output buffer is the caller's (out [B, hq, d], lse [B, hq], idx [B, hkv, topk_total] or None)."""
    di = ctx_lens if isinstance(ctx_lens, DecodeInfo) else DecodeInfo(ctx_lens)
    assert k_cache.dim() == 4 and k_cache.stride(3) == 1 and k_cache.stride() == v_cache.stride()
    assert kc_cache.dim() == 4 and kc_cache.is_contiguous() and q.is_contiguous() and out.is_contiguous()
    st = lib().infllmv2_sparse_decode_static(ctypes.byref(p), _ptr(q), _ptr(k_cache), _ptr(v_cache), k_cache.stride(0),
                                             k_cache.stride(1), k_cache.stride(2), _ptr(kc_cache), kc_cache.stride(1),
                                             _ptr(di.ctx_h), _ptr(di.ctx_d), q.shape[0], _ptr(idx), _ptr(out), _ptr(lse),
                                             _stream())
    _check(st, "infllmv2_sparse_decode_static")
    return out, lse, idx


def sparse_prefill(p: Params, q, k, v, cu_seqlens, buffers: Optional[dict] = None, fused_pool: bool = False):
    """The four stages back to back (a convenience for tests and the benchmark; no arithmetic here).
    buffers: a dict returned by an earlier call, whose tensors are then reused (nothing is allocated).
    fused_pool: stages 2 and 3 through the pooled entry points (s_cmp instead of s_shared in the result).
    Returns dict(out, lse, block_idx, s_shared | s_cmp, kc, cu_seqlens_c)."""
    b = buffers or {}
    si = _seq_info(cu_seqlens)
    kc, cu_c = compress_k(p, k, si, out=(b["kc"], b["cu_seqlens_c"]) if b else None)
    ws_scores = b.get("ws_scores")
    if ws_scores is None:
        ws_scores = _workspace(OP_BLOCK_SCORES_POOLED if fused_pool else OP_BLOCK_SCORES, p, si, q.device, None)
    if fused_pool:
        sc = block_scores_pooled(p, q, kc, si, cu_c, out=b.get("s_cmp"), workspace=ws_scores)
        idx = topk_pooled(p, sc, si, out=b.get("block_idx"))
        scores = dict(s_cmp=sc)
    else:
        sh = block_scores(p, q, kc, si, cu_c, out=b.get("s_shared"), workspace=ws_scores)
        idx = topk_blocks(p, sh, si, out=b.get("block_idx"))
        scores = dict(s_shared=sh)
    ws_attn = b.get("ws_attn")
    if ws_attn is None:
        ws_attn = _workspace(OP_SPARSE_ATTN_FWD, p, si, q.device, None)
    out, lse = sparse_attn_fwd(p, q, k, v, idx, si, out=b.get("out"), lse=b.get("lse"), workspace=ws_attn)
    return dict(out=out, lse=lse, block_idx=idx, kc=kc, cu_seqlens_c=cu_c, ws_attn=ws_attn, ws_scores=ws_scores,
                **scores)


# ---------------------------------------------------------------------------------- rotary positions
SCALINGS = {"none": 0, "linear": 1, "base": 2, "parts": 3}
LAYOUTS = {"half": 0, "interleaved": 1}
CACHE_NATIVE, CACHE_E4M3 = 0, 1


def rotary_turns(rot_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, *, original_len: float = 4096,
                 beta_fast: float = 32.0, beta_slow: float = 1.0, device="cuda") -> torch.Tensor:
    """Frequencies of rot_dim / 2 pairs of channels as 64-bit fractions of a turn per position (int64 bit patterns, device)."""
    turns = torch.empty(max(int(rot_dim), 0) // 2, dtype=torch.int64)
    st = lib().infllmv2_rotary_turns(int(rot_dim), float(base), SCALINGS[scaling], float(factor), float(original_len),
                                     float(beta_fast), float(beta_slow), turns.data_ptr())
    _check(st, "infllmv2_rotary_turns")
    return turns.to(device)


class Rotary:
    """How keys and queries are turned by their positions: the frequency table (rotary_turns) and how channels are paired."""

    def __init__(self, turns: torch.Tensor, rot_dim: int, layout: str = "half", magnitude: float = 1.0):
        assert turns.dtype == torch.int64 and turns.is_contiguous() and turns.numel() == int(rot_dim) // 2
        self.turns = turns
        self.c = _RotaryC(int(rot_dim), LAYOUTS[layout], float(magnitude), 0, turns.data_ptr())
        self.ref = ctypes.byref(self.c)


# (The checks below take shapes and strides as whole tuples: each question to a tensor is 0.1 to 0.3 us, and these calls are short.)
def _rotary(fn, p: Params, rot: Rotary, x: torch.Tensor, positions: torch.Tensor, out: Optional[torch.Tensor]):
    tokens, heads, d = x.shape
    x_tok, x_head, one = x.stride()
    assert one == 1 and d == p.head_dim and x.dtype is p.torch_dtype
    assert positions.dtype is torch.int32 and positions.is_contiguous() and positions.shape == (tokens,)
    if out is None:
        y_tok, y_head = heads * d, d
        out = torch.empty_like(x) if x_tok == y_tok and x_head == d else torch.empty_like(x, memory_format=torch.contiguous_format)
    else:
        y_tok, y_head, one = out.stride()
        assert one == 1 and out.shape == x.shape and out.dtype is x.dtype
    st = fn(ctypes.byref(p), rot.ref, x.data_ptr(), x_tok, x_head, out.data_ptr(), y_tok, y_head, positions.data_ptr(), tokens, heads, _stream())
    if st:
        _check(st, fn.__name__)
    return out


def rotary_fwd(p: Params, rot: Rotary, x: torch.Tensor, positions: torch.Tensor, out: Optional[torch.Tensor] = None):
    """x [T, heads, d] (any strides, d contiguous) turned by positions (device int32 [T]).  out: optional buffer, x itself allowed."""
    return _rotary(lib().infllmv2_rotary_fwd, p, rot, x, positions, out)


def rotary_bwd(p: Params, rot: Rotary, dy: torch.Tensor, positions: torch.Tensor, out: Optional[torch.Tensor] = None):
    """Gradient of rotary_fwd with respect to its input, from that of its output."""
    return _rotary(lib().infllmv2_rotary_bwd, p, rot, dy, positions, out)


# ---------------------------------------------------------------------------------- the paged cache
class PagedCache:
    """A K/V cache in pages of 64 tokens: k, v [num_pages, hkv, 64, d] (any strides, d contiguous; the data's type, or
    torch.float8_e4m3fn with float32 scales [num_pages, hkv]) and page_table [batch, blocks] (device int32)."""

    def __init__(self, p: Params, k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
                 v_scale: Optional[torch.Tensor] = None):
        coded = k.dtype == torch.float8_e4m3fn
        assert k.shape == v.shape and k.dtype == v.dtype and k.stride() == v.stride() and k.stride(3) == 1
        assert k.shape[1:] == (p.num_kv_heads, p.block_size, p.head_dim) and (coded or k.dtype == p.torch_dtype)
        assert page_table.dim() == 2 and page_table.dtype == torch.int32 and page_table.stride(1) == 1
        for s in (k_scale, v_scale) if coded else ():
            assert s.dtype == torch.float32 and s.is_contiguous() and s.shape == k.shape[:2]
        self.k, self.v, self.page_table, self.k_scale, self.v_scale = k, v, page_table, k_scale, v_scale
        self.batch, blocks = page_table.shape
        self.rows = (p.num_kv_heads, p.head_dim, p.dtype)
        # (rows of a table that is part of a wider one end before the library's check of their stride does)
        self.room = blocks * p.block_size if self.batch > 1 and page_table.stride(0) > blocks else None
        self.c = _CacheC(CACHE_E4M3 if coded else CACHE_NATIVE, k.shape[0], k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1),
                         k.stride(2), _ptr(k_scale), _ptr(v_scale), page_table.data_ptr(),
                         page_table.stride(0) if self.batch > 1 else blocks, 0)
        self.ref = ctypes.byref(self.c)

    def _holds(self, p: Params, max_ctx: int) -> bool:
        return self.rows == (p.num_kv_heads, p.head_dim, p.dtype) and (self.room is None or max_ctx <= self.room)

    @staticmethod
    def empty(p: Params, num_pages: int, page_table: torch.Tensor, kv_type: str = "e4m3") -> "PagedCache":
        """A cache with nothing in it."""
        shape, dev = (num_pages, p.num_kv_heads, p.block_size, p.head_dim), page_table.device
        dtype = {"e4m3": torch.float8_e4m3fn, "native": p.torch_dtype}[kv_type]
        k, v = (torch.empty(shape, dtype=dtype, device=dev) for _ in range(2))
        scales = [torch.ones(shape[:2], dtype=torch.float32, device=dev) for _ in range(2)] if kv_type == "e4m3" else [None, None]
        return PagedCache(p, k, v, page_table, *scales)


def _decode_info(lens) -> "DecodeInfo":
    return lens if isinstance(lens, DecodeInfo) else DecodeInfo(lens)


def cache_append(p: Params, cache: PagedCache, k: torch.Tensor, v: torch.Tensor, cu_new, prev_lens, rotary: Optional[Rotary] = None,
                 positions: Optional[torch.Tensor] = None):
    """New keys and values k, v [hkv, T, d] (packed by cu_new) written behind the prev_lens[b] tokens that sequence b has; keys turned by
    `rotary` (positions: device int32 [T], else a token's place in its sequence).  Returns the cache."""
    si, pv = _seq_info(cu_new), _decode_info(prev_lens)
    hs, ts, one = stride = k.stride()
    dtype, batch = p.torch_dtype, si.batch
    assert one == 1 and v.stride() == stride and k.dtype is dtype and v.dtype is dtype
    assert k.shape == v.shape == (p.num_kv_heads, si.total, p.head_dim) and batch == pv.batch <= cache.batch
    assert positions is None or (positions.dtype == torch.int32 and positions.is_contiguous() and positions.numel() == si.total)
    assert cache._holds(p, 0 if cache.room is None else max((n and n + t for n, t in zip(si.lens, pv.ctx_h.tolist())), default=0))
    st = lib().infllmv2_cache_append(ctypes.byref(p), cache.ref, rotary.ref if rotary is not None else None,
                                     k.data_ptr(), v.data_ptr(), ts, hs, si.cu_h.data_ptr(), si.cu_d.data_ptr(), pv.ctx_h.data_ptr(),
                                     pv.ctx_d.data_ptr(), _ptr(positions), batch, _stream())
    _check(st, "infllmv2_cache_append")
    return cache


def cache_compress_k(p: Params, cache: PagedCache, kc_cache: torch.Tensor, prev_lens, ctx_lens):
    """compress_k_append from the pages: kc_cache [B, hkv, max_nc, d] fp32 brought up to date in place."""
    pv, cx = _decode_info(prev_lens), _decode_info(ctx_lens)
    planes, hkv, rows, d = kc_cache.shape
    assert kc_cache.is_contiguous() and kc_cache.dtype is torch.float32 and hkv == p.num_kv_heads and d == p.head_dim
    assert pv.batch == cx.batch <= cache.batch and cx.batch <= planes and cache._holds(p, cx.max_ctx)
    st = lib().infllmv2_cache_compress_k(ctypes.byref(p), cache.ref, kc_cache.data_ptr(), rows * d, pv.ctx_h.data_ptr(),
                                         pv.ctx_d.data_ptr(), cx.ctx_h.data_ptr(), cx.ctx_d.data_ptr(), cx.batch, _stream())
    _check(st, "infllmv2_cache_compress_k")
    return kc_cache


def decode_blocks(p: Params, q: torch.Tensor, kc_cache: torch.Tensor, ctx_lens, out: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None):
    """Stages 2 and 3 of a decode step: q [B, hq, d], kc_cache [B, hkv, max_nc, d] fp32 -> block_idx [B, hkv, topk_total] int32."""
    di = _decode_info(ctx_lens)
    assert q.is_contiguous() and q.dtype == p.torch_dtype and q.shape == (di.batch, p.num_q_heads, p.head_dim)
    assert kc_cache.dim() == 4 and kc_cache.is_contiguous() and kc_cache.dtype == torch.float32 and kc_cache.shape[0] >= di.batch
    assert kc_cache.shape[1] == p.num_kv_heads and kc_cache.shape[3] == p.head_dim
    if out is None:
        out = torch.empty((di.batch, p.num_kv_heads, p.topk_total), dtype=torch.int32, device=q.device)
    assert out.is_contiguous() and out.dtype == torch.int32 and out.shape == (di.batch, p.num_kv_heads, p.topk_total)
    if workspace is None:
        need = workspace_bytes(OP_DECODE_BLOCKS, p, di.batch, 0, di.max_ctx)
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    st = lib().infllmv2_decode_blocks(ctypes.byref(p), _ptr(q), _ptr(kc_cache), kc_cache.stride(1), _ptr(di.ctx_h), _ptr(di.ctx_d),
                                      di.batch, _ptr(out), *_ws_args(workspace), _stream())
    _check(st, "infllmv2_decode_blocks")
    return out


def cache_attn(p: Params, cache: PagedCache, q: torch.Tensor, cu_seqlens_q, ctx_lens, block_idx: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Attention of the newest tokens of each sequence over its pages.  q [T, hq, d], packed by cu_seqlens_q; sequence b has ctx_lens[b]
    cached tokens, its queries the last of them.  block_idx [T, hkv, topk_total] int32 (decode_blocks makes that of a decode step) or None (all
    keys).  Returns (out [T, hq, d], lse [T, hq])."""
    si, cx = _seq_info(cu_seqlens_q), _decode_info(ctx_lens)
    tokens, hq, _ = shape = q.shape
    assert q.is_contiguous() and q.dtype is p.torch_dtype and shape == (si.total, p.num_q_heads, p.head_dim)
    assert si.batch == cx.batch <= cache.batch and cache._holds(p, cx.max_ctx)
    if block_idx is not None:
        assert block_idx.is_contiguous() and block_idx.dtype is torch.int32 and block_idx.shape == (tokens, p.num_kv_heads, p.topk_total)
    if out is None:
        out = torch.empty_like(q)
    else:
        assert out.is_contiguous() and out.shape == shape and out.dtype is q.dtype
    if lse is None:
        lse = q.new_empty((tokens, hq), dtype=torch.float32)
    else:
        assert lse.is_contiguous() and lse.shape == (tokens, hq) and lse.dtype is torch.float32
    if workspace is None:
        need = workspace_bytes(OP_CACHE_ATTN, p, si.batch, si.total, cx.max_ctx)
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    st = lib().infllmv2_cache_attn(ctypes.byref(p), cache.ref, q.data_ptr(), si.cu_h.data_ptr(), si.cu_d.data_ptr(),
                                   cx.ctx_h.data_ptr(), cx.ctx_d.data_ptr(), si.batch, _ptr(block_idx), out.data_ptr(), lse.data_ptr(),
                                   *_ws_args(workspace), _stream())
    _check(st, "infllmv2_cache_attn")
    return out, lse
