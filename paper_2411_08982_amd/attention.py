"""Binding of the attention half of a decode step (include/lynx/attention.h): argument marshalling only, as in binding.py.

Tensors of three dimensions [T, heads, D] may be parts of wider rows (a fused projection): heads and channels dense, any distance
between tokens.  All other tensors are contiguous.  A cache of dtype bfloat16 or float8_e4m3fn names its own format.
"""
from __future__ import annotations

from ctypes import c_float, c_int, c_int64, c_size_t, c_void_p

import torch

from . import binding
from .binding import BF16, F32, I32, _check, _ptr, _stream

ATTENTION_SYMBOLS = ["lynx_kv_assign", "lynx_qk_norm_rope", "lynx_attention_workspace_bytes", "lynx_attention", "lynx_attention_prefix"]
MAX_REQUESTS, MAX_STEP_TOKENS, MAX_PAGES, MAX_PAGE_SIZE = 1024, 65536, 1048576, 1024
KV_NO_PAGES, KV_NO_ROWS, KV_TOO_LONG = 1, 2, 4
CACHE_BF16, CACHE_FP8 = 0, 1
F64, FP8 = torch.float64, torch.float8_e4m3fn
_FORMATS = {BF16: CACHE_BF16, FP8: CACHE_FP8}

_lib = None


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


def _rows(t, what):
    """Address and token distance of a [T, heads, D] tensor whose tokens are dense."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what}: expected a CUDA/HIP tensor")
    if t.dtype is not BF16:
        raise TypeError(f"{what}: expected {BF16}, got {t.dtype}")
    if t.dim() != 3:
        raise ValueError(f"{what}: expected [tokens, heads, channels]")
    T, heads, D = t.shape
    s = t.stride()
    if s[2] != 1 or (heads > 1 and s[1] != D):
        raise ValueError(f"{what}: the heads of a token must be contiguous")
    # (a single token's distance to the next means nothing, and may be anything)
    return t.data_ptr(), (s[0] if T > 1 else heads * D)


def _same_device(*tensors):
    """Kernels run on the current device: all tensors have to be there."""
    here = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != here:
            raise ValueError(f"a tensor is on {t.device}, the current device is cuda:{here}")


def _vector(t, n, dtype, what):
    if t is not None and t.numel() != n:
        raise ValueError(f"{what}: expected {n} elements, got {t.numel()}")
    return _ptr(t, dtype, what)


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
    B = ctx_len.numel()
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise ValueError("block_table: expected [requests, max_pages]")
    dev = ctx_len.device
    T = int(T)
    if out is None:
        e = lambda n: torch.empty(n, dtype=I32, device=dev)
        out = dict(q_start=e(B + 1), seq_len=e(B), positions=e(T), slots=e(T), ring_state=e(2), status=e(1))
    _same_device(ctx_len, new_len, block_table, free_ring, ring_state, *[out[n] for n in _ASSIGN_OUT])
    sizes = (B + 1, B, T, T, 2, 1)
    _check(lib().lynx_kv_assign(_vector(ctx_len, B, I32, "ctx_len"), _vector(new_len, B, I32, "new_len"), B, T, int(page_size),
                                free_ring.numel(), block_table.shape[1], int(shared_pages), _ptr(block_table, I32, "block_table"),
                                _ptr(free_ring, I32, "free_ring"), _vector(ring_state, 2, I32, "ring_state"),
                                *[_vector(out[n], m, I32, n) for n, m in zip(_ASSIGN_OUT, sizes)], _stream()))
    return out


def lynx_qk_norm_rope(q, k, v, positions, slots, freqs, k_cache, v_cache, q_weight=None, k_weight=None, eps=1e-6,
                      interleaved=False, k_scale=1.0, v_scale=1.0, q_out=None):
    """Norms and rotation of q [T, QH, D] and k [T, KVH, D], k and v written to their slots of the cache -> q_out [T, QH, D].
    positions, slots [T] i32; freqs [rot/2] f64 (radians per position; None or empty: no rotation); weights [D] bf16 or None."""
    KVH, page_size, D, pages, fmt = _cache(k_cache, v_cache)
    T, QH = q.shape[0], q.shape[1] if q.dim() == 3 else 0
    if q_out is None:
        q_out = torch.empty((T, QH, D), dtype=BF16, device=q.device)
    _same_device(q, k, v, positions, slots, freqs, k_cache, v_cache, q_weight, k_weight, q_out)
    (qp, qs), (kp, ks), (vp, vs), (op, os_) = _rows(q, "q"), _rows(k, "k"), _rows(v, "v"), _rows(q_out, "q_out")
    if q.shape[2] != D or k.shape != (T, KVH, D) or v.shape != (T, KVH, D) or q_out.shape != q.shape:
        raise ValueError("q, k, v, q_out: shapes do not match each other and the cache")
    rot = 0 if freqs is None else 2 * freqs.numel()
    _check(lib().lynx_qk_norm_rope(qp, qs, kp, ks, vp, vs, _vector(q_weight, D, BF16, "q_weight"), _vector(k_weight, D, BF16, "k_weight"),
                                   float(eps), _vector(positions, T, I32, "positions"), _vector(slots, T, I32, "slots"),
                                   _ptr(freqs, F64, "freqs"), rot, int(bool(interleaved)), T, QH, KVH, D, op, os_,
                                   _ptr(k_cache, k_cache.dtype, "k_cache"), _ptr(v_cache, v_cache.dtype, "v_cache"), fmt,
                                   float(k_scale), float(v_scale), pages, page_size, _stream()))
    return q_out


def attention_workspace_bytes(B, T, QH, KVH, D, prefix_len=0) -> int:
    return int(lib().lynx_attention_workspace_bytes(B, T, QH, KVH, D, prefix_len))


def new_attention_workspace(B, T, QH, KVH, D, prefix_len=0, device="cuda"):
    return torch.empty(max(attention_workspace_bytes(B, T, QH, KVH, D, prefix_len), 256), dtype=torch.uint8, device=device)


def _attention(q, k_cache, v_cache, block_table, q_start, seq_len, max_new, scale, k_scale, v_scale, out, lse, workspace, prefix, tail):
    KVH, page_size, D, pages, fmt = _cache(k_cache, v_cache)
    qp, qs = _rows(q, "q")
    T, QH, Dq = q.shape
    if Dq != D:
        raise ValueError("q: channels do not match the cache")
    if block_table.dim() != 2:
        raise ValueError("block_table: expected [requests, max_pages]")
    B, max_pages = block_table.shape
    dev = q.device
    if out is None:
        out = torch.empty((T, QH, D), dtype=BF16, device=dev)
    op, os_ = _rows(out, "out")
    if out.shape != q.shape:
        raise ValueError("out: expected the shape of q")
    prefix_len = prefix[1] if prefix else 0
    need = lib().lynx_attention_workspace_bytes(B, T, QH, KVH, D, prefix_len)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    elif workspace.numel() * workspace.element_size() < need:
        raise ValueError(f"workspace too small: {workspace.numel() * workspace.element_size()} < {need}")
    _same_device(q, k_cache, v_cache, block_table, q_start, seq_len, out, lse, workspace, prefix[0] if prefix else None)
    args = (qp, qs, _ptr(k_cache, k_cache.dtype, "k_cache"), _ptr(v_cache, v_cache.dtype, "v_cache"), fmt, float(k_scale),
            float(v_scale), pages, page_size, _ptr(block_table, I32, "block_table"), max_pages, _vector(q_start, B + 1, I32, "q_start"),
            _vector(seq_len, B, I32, "seq_len"))
    if prefix:
        args += (_vector(prefix[0], -(-prefix_len // page_size), I32, "prefix_table"), prefix_len)
    call = lib().lynx_attention_prefix if prefix else lib().lynx_attention
    _check(call(*args, B, T, int(max_new), QH, KVH, D, float(D ** -0.5 if scale is None else scale), *tail, op, os_,
                _vector(lse, T * QH, F32, "lse"), workspace.data_ptr(), _stream()))
    return out


def lynx_attention(q, k_cache, v_cache, block_table, q_start, seq_len, max_new, scale=None, window=0, sinks=0, k_scale=1.0,
                   v_scale=1.0, out=None, lse=None, workspace=None):
    """Attention of q [T, QH, D] over the paged cache -> out [T, QH, D].  block_table [B, max_pages], q_start [B+1], seq_len [B]
    i32; max_new: the largest number of new tokens of a request, as far as known; scale: 1 / sqrt(D) if None; lse: [T, QH] f32
    that receives the logarithm of each row's sum of weights, or None."""
    return _attention(q, k_cache, v_cache, block_table, q_start, seq_len, max_new, scale, k_scale, v_scale, out, lse, workspace, None,
                      (int(window), int(sinks)))


def lynx_attention_prefix(q, k_cache, v_cache, block_table, q_start, seq_len, max_new, prefix_table, prefix_len, scale=None,
                          k_scale=1.0, v_scale=1.0, out=None, lse=None, workspace=None):
    """lynx_attention for a batch whose sequences all begin with the same prefix_len tokens, held by the pages of prefix_table
    [ceil(prefix_len / page size)] i32: they are read once for the whole batch."""
    return _attention(q, k_cache, v_cache, block_table, q_start, seq_len, max_new, scale, k_scale, v_scale, out, lse, workspace,
                      (prefix_table, int(prefix_len)), ())
