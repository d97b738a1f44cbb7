"""include/lynx/attention.h without a GPU: every declared symbol is exported, the limits match the binding, bad arguments are
refused before anything is enqueued, and the host oracle of the GPU tests agrees with a dense computation."""
import ctypes
import os
import re

import pytest
import torch

import attention_ref as ref
import paper_2411_08982_amd as L
from paper_2411_08982_amd import attention as A
from paper_2411_08982_amd import check_code
from paper_2411_08982_amd.build import LIB

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "lynx", "attention.h")


def _header():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def test_library_exports_every_declared_symbol():
    names = set(re.findall(r"\b(lynx_[a-z0-9_]+)\s*\(", _header()))
    assert names == set(L.ATTENTION_SYMBOLS)
    for n in names:
        assert getattr(A.lib(), n).argtypes is not None


def test_header_limits_match_binding():
    vals = {m[0]: int(m[1]) for m in re.findall(r"#define LYNX_(\w+) (\d+)", _header())}
    assert (vals["MAX_REQUESTS"], vals["MAX_STEP_TOKENS"], vals["MAX_PAGES"], vals["MAX_PAGE_SIZE"]) == (
        A.MAX_REQUESTS, A.MAX_STEP_TOKENS, A.MAX_PAGES, A.MAX_PAGE_SIZE)
    assert (vals["KV_NO_PAGES"], vals["KV_NO_ROWS"], vals["KV_TOO_LONG"]) == (A.KV_NO_PAGES, A.KV_NO_ROWS, A.KV_TOO_LONG)
    assert (vals["CACHE_BF16"], vals["CACHE_FP8"]) == (A.CACHE_BF16, A.CACHE_FP8)


one, odd = ctypes.c_void_p(4096), ctypes.c_void_p(4098)     # never dereferenced: every call below fails on its checks


def _assign(B=4, T=4, page=16, pages=8, per_row=4, shared=0, **kw):
    a = dict(ctx=one, new=one, table=one, ring=one, state=one, q_start=one, seq=one, pos=one, slots=one, state_out=one, status=one)
    a.update(kw)
    return A.lib().lynx_kv_assign(a["ctx"], a["new"], B, T, page, pages, per_row, shared, a["table"], a["ring"], a["state"], a["q_start"],
                                  a["seq"], a["pos"], a["slots"], a["state_out"], a["status"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), -1), (dict(T=-1), -1), (dict(page=0), -1), (dict(pages=0), -1), (dict(per_row=0), -1), (dict(shared=-1), -1),
    (dict(shared=5), -1), (dict(B=1025), -2), (dict(T=65537), -2), (dict(page=24), -2), (dict(page=2048), -2),
    (dict(pages=(1 << 20) + 1), -2), (dict(per_row=1 << 26), -2), (dict(ctx=None), -1), (dict(new=None), -1), (dict(table=None), -1),
    (dict(ring=None), -1), (dict(state=None), -1), (dict(q_start=None), -1), (dict(seq=None), -1), (dict(pos=None), -1),
    (dict(slots=None), -1), (dict(state_out=None), -1), (dict(status=None), -1)])
def test_kv_assign_refuses(kw, code):
    assert _assign(**kw) == code
    assert b"lynx_kv_assign" in A.lib().lynx_last_error()


def _rope(T=4, QH=4, KVH=2, D=128, rot=128, eps=1e-6, fmt=0, ks=1.0, vs=1.0, pages=8, page=16, qs=None, **kw):
    a = dict(q=one, k=one, v=one, qw=one, kw=one, pos=one, slots=one, freqs=one, out=one, kc=one, vc=one)
    a.update(kw)
    qs = QH * D if qs is None else qs
    return A.lib().lynx_qk_norm_rope(a["q"], qs, a["k"], KVH * D, a["v"], KVH * D, a["qw"], a["kw"], eps, a["pos"], a["slots"], a["freqs"],
                                     rot, 0, T, QH, KVH, D, a["out"], QH * D, a["kc"], a["vc"], fmt, ks, vs, pages, page, None)


CACHE_REFUSALS = [
    (dict(QH=5), -1), (dict(KVH=0), -1), (dict(QH=0), -1), (dict(D=96), -2), (dict(D=256), -2), (dict(pages=0), -1), (dict(page=8), -2),
    (dict(page=20), -2), (dict(page=2048), -2), (dict(QH=2048), -2), (dict(QH=514, KVH=2), -2), (dict(fmt=2), -1), (dict(fmt=1, ks=0.0), -1),
    (dict(fmt=1, vs=float("nan")), -1), (dict(fmt=1, ks=float("inf")), -1), (dict(ks=2.0), -1), (dict(kc=None), -1), (dict(vc=None), -1),
    (dict(kc=odd), -1), (dict(T=-1), -1), (dict(T=65537), -2), (dict(q=None), -1), (dict(q=odd), -1), (dict(qs=100), -1),
    (dict(qs=515), -1), (dict(out=None), -1), (dict(out=odd), -1)]


@pytest.mark.parametrize("kw,code", CACHE_REFUSALS + [
    (dict(rot=24), -1), (dict(rot=144), -1), (dict(rot=-16), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(pos=None), -1),
    (dict(slots=None), -1), (dict(freqs=None), -1), (dict(qw=odd), -1), (dict(kw=odd), -1), (dict(k=None), -1), (dict(v=odd), -1)])
def test_qk_norm_rope_refuses(kw, code):
    assert _rope(**kw) == code
    assert b"lynx_qk_norm_rope" in A.lib().lynx_last_error()


def _attn(prefix=False, T=4, B=4, QH=4, KVH=2, D=128, fmt=0, ks=1.0, vs=1.0, pages=8, page=16, per_row=4, max_new=1, scale=0.1,
          window=0, sinks=0, plen=20, qs=None, **kw):
    a = dict(q=one, kc=one, vc=one, table=one, q_start=one, seq=one, out=one, ws=one, pt=one)
    a.update(kw)
    qs = QH * D if qs is None else qs
    head = (a["q"], qs, a["kc"], a["vc"], fmt, ks, vs, pages, page, a["table"], per_row, a["q_start"], a["seq"])
    tail = (a["out"], QH * D, None, a["ws"], None)
    if prefix:
        return A.lib().lynx_attention_prefix(*head, a["pt"], plen, B, T, max_new, QH, KVH, D, scale, *tail)
    return A.lib().lynx_attention(*head, B, T, max_new, QH, KVH, D, scale, window, sinks, *tail)


ATTENTION_REFUSALS = CACHE_REFUSALS + [
    (dict(B=0), -1), (dict(B=1025), -2), (dict(per_row=0), -1), (dict(per_row=1 << 26), -2), (dict(max_new=-1), -1), (dict(scale=0.0), -1),
    (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(table=None), -1), (dict(q_start=None), -1), (dict(seq=None), -1),
    (dict(ws=None), -1)]


@pytest.mark.parametrize("kw,code", ATTENTION_REFUSALS + [(dict(window=-1), -1), (dict(sinks=-1), -1)])
def test_attention_refuses(kw, code):
    assert _attn(**kw) == code
    assert b"lynx_attention:" in A.lib().lynx_last_error()


@pytest.mark.parametrize("kw,code", ATTENTION_REFUSALS + [(dict(plen=-1), -1), (dict(plen=65), -1), (dict(pt=None), -1)])
def test_attention_prefix_refuses(kw, code):
    assert _attn(prefix=True, **kw) == code
    assert b"lynx_attention_prefix:" in A.lib().lynx_last_error()


def test_nothing_to_do_is_no_error():
    assert _rope(T=0, q=None, k=None, v=None, out=None, pos=None, slots=None) == 0
    assert _attn(T=0, q=None, out=None) == 0 and _attn(prefix=True, T=0, q=None, out=None) == 0
    assert L.attention_workspace_bytes(0, 1, 8, 2, 128) == 0 and L.attention_workspace_bytes(4, 4, 8, 2, 128) > 0


def test_binding_refuses_before_it_calls():
    q = torch.zeros(2, 4, 128, dtype=torch.bfloat16)
    kc, vc = torch.zeros(3, 2, 16, 128, dtype=torch.bfloat16), torch.zeros(3, 2, 128, 16, dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError, match="CUDA"):
        L.lynx_attention(q, kc, vc, i.view(1, 2), i, i[:1], 1)
    with pytest.raises(TypeError, match="float8"):
        L.lynx_attention(q, kc.half(), vc.half(), i.view(1, 2), i, i[:1], 1)
    with pytest.raises(ValueError, match="v_cache"):
        L.lynx_attention(q, kc, kc, i.view(1, 2), i, i[:1], 1)
    with pytest.raises(ValueError, match="key heads"):
        L.lynx_attention(q, kc[0], vc[0], i.view(1, 2), i, i[:1], 1)
    with pytest.raises(TypeError, match="dtype"):
        L.new_cache(2, 2, 16, 64, torch.float16, device="cpu")


def test_the_oracle_agrees_with_a_dense_computation():
    g = torch.Generator().manual_seed(1)
    n, D, ps = 21, 64, 16
    k, v, q = (torch.randn(n, 1, D, generator=g, dtype=torch.float64) for _ in range(3))
    kc, vc = torch.zeros(3, 1, ps, D, dtype=torch.float64), torch.zeros(3, 1, D, ps, dtype=torch.float64)
    table = [[2, 0]]
    for j in range(n):
        kc[table[0][j // ps], 0, j % ps], vc[table[0][j // ps], 0, :, j % ps] = k[j, 0], v[j, 0]
    out, lse, tol = ref.attention(q, kc, vc, table, [0, n], [n], 0.125, window=6, sinks=2)
    z = 0.125 * q[:, 0] @ k[:, 0].T
    i, j = torch.arange(n)[:, None], torch.arange(n)[None, :]
    z = z.masked_fill(~((j <= i) & ((j > i - 6) | (j < 2))), float("-inf"))
    assert torch.allclose(out[:, 0], torch.softmax(z, 1) @ v[:, 0], atol=1e-12) and torch.allclose(lse[:, 0], z.logsumexp(1), atol=1e-12)
    # rotation: lengths of pairs stay, position 0 changes nothing
    x, _ = ref.norm_rope(q, None, 0.0, torch.zeros(n), torch.ones(D // 2, dtype=torch.float64), True)
    assert torch.allclose(x, q)
    x, _ = ref.norm_rope(q, None, 0.0, torch.arange(n), torch.rand(D // 2, generator=g, dtype=torch.float64), False)
    assert torch.allclose(x[..., :32] ** 2 + x[..., 32:] ** 2, q[..., :32] ** 2 + q[..., 32:] ** 2)
    # pages: two requests grow, one ends, and what it held is given out in the next step
    r = ref.kv_assign([15, 16, 3], [2, 1, -1], 4, 16, [[1, -1], [2, -1], [3, -1]], [9, 5, 4, 9, 9, 9], [1, 2])
    assert r["table"] == [[1, 5], [2, 4], [3, -1]] and r["ring"] == [9, 5, 4, 3, 9, 9] and r["ring_state"] == [3, 1]
    assert r["q_start"] == [0, 2, 3, 3] and r["slots"] == [31, 80, 64, -1] and r["seq_len"] == [17, 17, 0] and r["status"] == [0]


@pytest.mark.skipif(not os.path.exists(LIB), reason="the library is not built")
def test_block_buffers_lie_in_the_first_64_kib():
    assert sum(check_code.check_attention_placement(notes) for notes, _ in check_code.code_object_texts(LIB)) == 8    # D, cache format, with tiles or without
    notes = "\n  - .group_segment_fixed_size: %d\n    .name:           _ZN4lynx11attn_kernelILi128ELb0ELb1EEEvNS_10AttnParamsE\n"
    assert check_code.check_attention_placement(notes % (65536 + 16383)) == 1
    with pytest.raises(RuntimeError, match="first 65536"):
        check_code.check_attention_placement(notes % (65536 + 16384))


def test_scores_out_of_range_and_results_over_queries_are_refused():
    other = ctypes.c_void_p(8192)
    for kw in (dict(scale=1e-40), dict(scale=1e30, ks=1e30, fmt=1), dict(scale=1e-30, ks=1e-30, fmt=1)):
        assert _attn(out=other, **kw) == -1 and b"scale * k_scale" in A.lib().lynx_last_error()
        assert _attn(prefix=True, out=other, **kw) == -1
    assert _attn(q=one, out=one) == -1 and b"out must not be q" in A.lib().lynx_last_error()


def test_workspace_of_sizes_out_of_range_is_nothing():
    # (sizes, some of which would be a division by zero or overflow an int on the way)
    for sizes in ((4, 4, 2, 8, 128, 100), (4, 4, 6, 4, 128, 100), (1, 2 ** 31 - 1, 1024, 4, 128, 64), (1, 65537, 8, 8, 64, 64), (1, 1, 2 ** 31 - 1, 1, 64, 64),
                  (1025, 4, 8, 2, 128, 64), (4, 4, 512, 1, 128, 64), (4, 4, 8, 2, 96, 64), (4, 4, 8, 0, 128, 64), (4, 4, -8, -2, 128, 64), (4, 4, 8, 2, 128, -1)):
        assert L.attention_workspace_bytes(*sizes) == 0, sizes
    assert L.attention_workspace_bytes(1024, 65536, 1024, 1024, 128, 2 ** 29) > L.attention_workspace_bytes(1024, 65536, 1024, 1024, 128) > 0
