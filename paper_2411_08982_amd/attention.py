"""Binding of the attention half of a decode step (include/lynx/attention.h): argument marshalling only, as in binding.py.

Tensors of three dimensions [T, heads, D] may be parts of wider rows (a fused projection): heads and channels dense, any distance
between tokens.  All other tensors are contiguous.  A cache of dtype bfloat16 or float8_e4m3fn names its own format.
"""
from __future__ import annotations

import functools
from ctypes import c_float, c_int, c_int64, c_size_t, c_void_p

import torch

from . import binding
from .binding import BF16, F32, I32, _check, _ptr

ATTENTION_SYMBOLS = ["lynx_kv_assign", "lynx_qk_norm_rope", "lynx_attention_workspace_bytes", "lynx_attention", "lynx_attention_prefix"]
MAX_REQUESTS, MAX_STEP_TOKENS, MAX_PAGES, MAX_PAGE_SIZE = 1024, 65536, 1048576, 1024
KV_NO_PAGES, KV_NO_ROWS, KV_TOO_LONG, KV_LOST_PAGES = 1, 2, 4, 8
CACHE_BF16, CACHE_FP8 = 0, 1
F64, FP8 = torch.float64, torch.float8_e4m3fn
_FORMATS = {BF16: CACHE_BF16, FP8: CACHE_FP8}

_lib = None
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)        # (its handle, as binding._stream has it)


def lib():
    """liblynx.so with the argument types of the calls of this module."""
    global _lib
    if _lib is None:
        L = binding.lib()
        P, I, F, S = c_void_p, c_int, c_float, c_int64
        L.lynx_kv_assign.argtypes = [P, P, I, I, I, I, I, I] + [P] * 10
        L.lynx_qk_norm_rope.argtypes = [P, S, P, S, P, S, P, P, F, P, P, P, I, I, I, I, I, I, P, S, P, P, I, F, F, I, I, P]
        L.lynx_attention_workspace_bytes.argtypes = [I] * 6
        cache = [P, S, P, P, I, F, F, I, I, P, I, P, P]
        L.lynx_attention.argtypes = cache + [I] * 6 + [F, I, I, P, S, P, P, P]
        L.lynx_attention_prefix.argtypes = cache + [P, I] + [I] * 6 + [F, P, S, P, P, P]
        for name in ATTENTION_SYMBOLS:
            getattr(L, name).restype = c_int
        L.lynx_attention_workspace_bytes.restype = c_size_t
        _lib = L
    return _lib


# The host spends longer on these calls than the GPU does on a small batch, so every check is one pass over a tensor, and tensors that
# a call has just allocated are not checked (host time: lynx_kv_assign 17.7 -> 10.7 us, lynx_qk_norm_rope 14.1 -> 11.2; lynx_attention
# takes 13.8, with two launches of 3.6 each).
def _here(t, what):
    """The current device, on which kernels run; t: the call's first tensor."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what}: expected a CUDA/HIP tensor")
    return torch._C._cuda_getDevice()


def _at(t, dtype, n, here, what):
    """Address of a contiguous tensor of n elements (None: any number) on the current device, which is where kernels run."""
    if type(t) is torch.Tensor and t.dtype is dtype and t.get_device() == here and t.is_contiguous() and (n is None or t.numel() == n):
        return t.data_ptr()
    if t is None:
        return None
    _ptr(t, dtype, what)
    if t.get_device() != here:
        raise ValueError(f"{what}: on {t.device}, the current device is cuda:{here}")
    if n is not None and t.numel() != n:
        raise ValueError(f"{what}: expected {n} elements, got {t.numel()}")
    return t.data_ptr()


def _rows(t, heads, D, here, what):
    """Address and token distance of a [T, heads, D] tensor whose tokens are dense (heads, D: None for any)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what}: expected a CUDA/HIP tensor")
    if t.dtype is not BF16:
        raise TypeError(f"{what}: expected {BF16}, got {t.dtype}")
    if t.dim() != 3:
        raise ValueError(f"{what}: expected [tokens, heads, channels]")
    if t.get_device() != here:
        raise ValueError(f"{what}: on {t.device}, the current device is cuda:{here}")
    T, h, d = t.shape
    step, a, b = t.stride()
    if b != 1 or (h > 1 and a != d):
        raise ValueError(f"{what}: the heads of a token must be contiguous")
    if d != D or (heads is not None and h != heads):
        raise ValueError(f"{what}: the shapes do not match each other and the cache")
    # (a single token's distance to the next means nothing, and may be anything)
    return t.data_ptr(), (step if T > 1 else h * d)


def _cache(k_cache, v_cache):
    """(key heads, page size, channels, pages, format) of a paged cache."""
    fmt = _FORMATS.get(k_cache.dtype)
    if fmt is None or v_cache.dtype is not k_cache.dtype:
        raise TypeError("k_cache, v_cache: expected bfloat16 or float8_e4m3fn, both the same")
    if k_cache.dim() != 4:
        raise ValueError("k_cache: expected [pages, key heads, page size, channels]")
    pages, KVH, page_size, D = k_cache.shape
    if v_cache.shape != (pages, KVH, D, page_size):
        raise ValueError("v_cache: expected [pages, key heads, channels, page size] of the same sizes")
    return KVH, page_size, D, pages, fmt


def _pages(k_cache, v_cache, here):
    """Addresses of a cache whose sizes _cache has looked at."""
    if k_cache.get_device() == here and v_cache.get_device() == here and k_cache.is_contiguous() and v_cache.is_contiguous():
        return k_cache.data_ptr(), v_cache.data_ptr()
    return _at(k_cache, k_cache.dtype, None, here, "k_cache"), _at(v_cache, v_cache.dtype, None, here, "v_cache")


def new_cache(num_pages, KVH, page_size, D, dtype=BF16, device="cuda"):
    """(k_cache, v_cache) of one layer, uninitialised."""
    if dtype not in _FORMATS:
        raise TypeError("dtype: expected bfloat16 or float8_e4m3fn")
    return (torch.empty((num_pages, KVH, page_size, D), dtype=dtype, device=device),
            torch.empty((num_pages, KVH, D, page_size), dtype=dtype, device=device))


_ASSIGN_OUT = ("q_start", "seq_len", "positions", "slots", "ring_state", "status")


def lynx_kv_assign(ctx_len, new_len, T, page_size, block_table, free_ring, ring_state, shared_pages=0, out=None):
    """Pages and slots of a step's tokens: ctx_len, new_len [B] i32, block_table [B, max_pages] i32 and free_ring [num_pages] i32
    (both updated), ring_state [2] i32 = head, count -> dict(q_start [B+1], seq_len [B], positions [T], slots [T],
    ring_state [2], status [1]), all i32.  out: such a dict; its seq_len may be ctx_len, its ring_state may be ring_state."""
    here = _here(ctx_len, "ctx_len")
    B = ctx_len.numel()
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise ValueError("block_table: expected [requests, max_pages]")
    sizes = (B + 1, B, T, T, 2, 1)
    if out is None:
        parts = torch.empty(sum(sizes), dtype=I32, device=ctx_len.device).split_with_sizes(sizes)      # one allocation
        out = dict(zip(_ASSIGN_OUT, parts))
        made = [t.data_ptr() for t in parts]
    else:
        made = [_at(out[n], I32, m, here, n) for n, m in zip(_ASSIGN_OUT, sizes)]
    _check(lib().lynx_kv_assign(_at(ctx_len, I32, B, here, "ctx_len"), _at(new_len, I32, B, here, "new_len"), B, T, page_size,
                                free_ring.numel(), block_table.shape[1], shared_pages, _at(block_table, I32, None, here, "block_table"),
                                _at(free_ring, I32, None, here, "free_ring"), _at(ring_state, I32, 2, here, "ring_state"), *made, _current_stream(here)))
    return out


def lynx_qk_norm_rope(q, k, v, positions, slots, freqs, k_cache, v_cache, q_weight=None, k_weight=None, eps=1e-6,
                      interleaved=False, k_scale=1.0, v_scale=1.0, q_out=None):
    """Norms and rotation of q [T, QH, D] and k [T, KVH, D], k and v written to their slots of the cache -> q_out [T, QH, D].
    positions, slots [T] i32; freqs [rot/2] f64 (radians per position; None or empty: no rotation); weights [D] bf16 or None."""
    KVH, page_size, D, pages, fmt = _cache(k_cache, v_cache)
    here = _here(q, "q")
    qp, qs = _rows(q, None, D, here, "q")
    T, QH, _ = q.shape
    kp, ks = _rows(k, KVH, D, here, "k")
    vp, vs = _rows(v, KVH, D, here, "v")
    if q_out is None:
        q_out = q.new_empty(T, QH, D)
        op, os_ = q_out.data_ptr(), QH * D
    else:
        op, os_ = _rows(q_out, QH, D, here, "q_out")
    if k.shape[0] != T or v.shape[0] != T or q_out.shape[0] != T:
        raise ValueError("q, k, v, q_out: the shapes do not match each other and the cache")
    rot = 0 if freqs is None else 2 * freqs.numel()
    k_at, v_at = _pages(k_cache, v_cache, here)
    _check(lib().lynx_qk_norm_rope(qp, qs, kp, ks, vp, vs, _at(q_weight, BF16, D, here, "q_weight"), _at(k_weight, BF16, D, here, "k_weight"),
                                   eps, _at(positions, I32, T, here, "positions"), _at(slots, I32, T, here, "slots"),
                                   _at(freqs, F64, None, here, "freqs"), rot, 1 if interleaved else 0, T, QH, KVH, D, op, os_,
                                   k_at, v_at, fmt, k_scale, v_scale, pages, page_size, _current_stream(here)))
    return q_out


@functools.lru_cache(maxsize=4096)
def attention_workspace_bytes(B, T, QH, KVH, D, prefix_len=0) -> int:
    return int(lib().lynx_attention_workspace_bytes(B, T, QH, KVH, D, prefix_len))


def new_attention_workspace(B, T, QH, KVH, D, prefix_len=0, device="cuda"):
    return torch.empty(max(attention_workspace_bytes(B, T, QH, KVH, D, prefix_len), 256), dtype=torch.uint8, device=device)


def _attention(q, k_cache, v_cache, block_table, q_start, seq_len, max_new, scale, k_scale, v_scale, out, lse, workspace, prefix, tail):
    KVH, page_size, D, pages, fmt = _cache(k_cache, v_cache)
    here = _here(q, "q")
    qp, qs = _rows(q, None, D, here, "q")
    T, QH, _ = q.shape
    if block_table.dim() != 2:
        raise ValueError("block_table: expected [requests, max_pages]")
    B, max_pages = block_table.shape
    if out is None:
        out = q.new_empty(T, QH, D)
        op, os_ = out.data_ptr(), QH * D
    else:
        op, os_ = _rows(out, QH, D, here, "out")
        if out.shape[0] != T:
            raise ValueError("out: expected the shape of q")
    need = attention_workspace_bytes(B, T, QH, KVH, D, prefix[1] if prefix else 0)
    if workspace is None:
        workspace = q.new_empty(max(need, 256) // 2)         # (as bf16: need is a multiple of 256)
    elif workspace.get_device() != here or not workspace.is_contiguous() or workspace.numel() * workspace.element_size() < need:
        raise ValueError(f"workspace: on {workspace.device}, {workspace.numel() * workspace.element_size()} bytes; needed {need} contiguous on cuda:{here}")
    if prefix:
        call = lib().lynx_attention_prefix
        prefix = (_at(prefix[0], I32, -(-prefix[1] // page_size), here, "prefix_table"), prefix[1])
    else:
        call = lib().lynx_attention
    _check(call(qp, qs, *_pages(k_cache, v_cache, here), fmt, k_scale, v_scale, pages, page_size, _at(block_table, I32, None, here, "block_table"),
                max_pages, _at(q_start, I32, B + 1, here, "q_start"), _at(seq_len, I32, B, here, "seq_len"), *prefix, B, T, max_new, QH, KVH, D,
                D ** -0.5 if scale is None else scale, *tail, op, os_, _at(lse, F32, T * QH, here, "lse"), workspace.data_ptr(), _current_stream(here)))
    return out


def lynx_attention(q, k_cache, v_cache, block_table, q_start, seq_len, max_new, scale=None, window=0, sinks=0, k_scale=1.0,
                   v_scale=1.0, out=None, lse=None, workspace=None):
    """Attention of q [T, QH, D] over the paged cache -> out [T, QH, D].  block_table [B, max_pages], q_start [B+1], seq_len [B]
    i32; max_new: the largest number of new tokens of a request, as far as known; scale: 1 / sqrt(D) if None; lse: [T, QH] f32
    that receives the logarithm of each row's sum of weights, or None."""
    return _attention(q, k_cache, v_cache, block_table, q_start, seq_len, max_new, scale, k_scale, v_scale, out, lse, workspace, (),
                      (window, sinks))


def lynx_attention_prefix(q, k_cache, v_cache, block_table, q_start, seq_len, max_new, prefix_table, prefix_len, scale=None,
                          k_scale=1.0, v_scale=1.0, out=None, lse=None, workspace=None):
    """lynx_attention for a batch whose sequences all begin with the same prefix_len tokens, held by the pages of prefix_table
    [ceil(prefix_len / page size)] i32: they are read once for the whole batch."""
    return _attention(q, k_cache, v_cache, block_table, q_start, seq_len, max_new, scale, k_scale, v_scale, out, lse, workspace,
                      (prefix_table, prefix_len), ())
