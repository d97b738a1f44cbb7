"""Plain implementations, in 64 bits or whole numbers on the host, of the calls of include/lynx/attention.h, and the bounds that
their roundings give."""
import math

import torch

E4M3_MAX = 448.0


def pages_needed(tokens, page_size):
    return -(-tokens // page_size)


def kv_assign(ctx, new, T, page_size, table, ring, state, shared=0):
    """Lists in, dict of lists out (table: list of rows, ring: list; both copied)."""
    B, cap, num = len(ctx), len(table[0]) * page_size, len(ring)
    table, ring = [list(r) for r in table], list(ring)
    head, count = state
    free = [ring[(head + i) % num] for i in range(count)]
    taken, status, stop = 0, 0, False
    back, rows, q_start, seq, where = [], 0, [0], [], []
    want_rows = want_pages = 0
    for b in range(B):
        c, n = ctx[b], new[b]
        if c < 0 or c > cap or c + max(n, 0) > cap:
            status |= 4
            c, n = min(max(c, 0), cap), 0
        held = pages_needed(c, page_size)
        if n < 0:
            back += table[b][shared:held]
            seq.append(0)
        else:
            have = max(held, shared)
            take = max(pages_needed(c + n, page_size) - have, 0)
            want_rows, want_pages = want_rows + n, want_pages + take
            if n and (stop or want_rows > T or want_pages > count):
                stop = True
                status |= (2 if want_rows > T else 0) | (1 if want_pages > count else 0)
                n = take = 0
            for i in range(take):
                table[b][have + i] = free[taken]
                taken += 1
            where += [(b, c + i) for i in range(n)]
            rows += n
            seq.append(c + n)
        q_start.append(rows)
    for i, page in enumerate(back):
        ring[(head + count + i) % num] = page
    slot = lambda b, p: table[b][p // page_size] * page_size + p % page_size if 0 <= table[b][p // page_size] < num else -1
    pad = T - len(where)
    return dict(q_start=q_start, seq_len=seq, positions=[p for _, p in where] + [0] * pad,
                slots=[slot(b, p) for b, p in where] + [-1] * pad, ring_state=[(head + taken) % num, count - taken + len(back)],
                status=[status], table=table, ring=ring)


def norm_rope(x, weight, eps, positions, freqs, interleaved):
    """x [T, heads, D] float64 -> (rotated rows, magnitude that roundings in fp32 are relative to)."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * weight.double()
    size = x.abs().clone()
    if freqs is not None and freqs.numel():
        half = freqs.numel()
        phi = (positions.double()[:, None] * freqs[None, :])[:, None, :]
        i, j = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
        a, b = x[..., i].clone(), x[..., j].clone()
        x[..., i], x[..., j] = a * phi.cos() - b * phi.sin(), b * phi.cos() + a * phi.sin()
        size[..., i] = size[..., j] = a.abs() + b.abs()
    return x, size


def gather(cache_k, cache_v, row, n, page_size):
    """Tokens 0 .. n-1 of one row of the block table: k, v [n, KVH, D] float64 (nan where there is no such page)."""
    j = torch.arange(n)
    page = torch.as_tensor(row)[j // page_size].long()
    ok = (page >= 0) & (page < cache_k.shape[0])
    page = torch.where(ok, page, 0)
    k = cache_k[page, :, j % page_size].double()
    v = cache_v[page, :, :, j % page_size].double()
    return k, v, ok


def attention(q, cache_k, cache_v, table, q_start, seq, scale, window=0, sinks=0, k_scale=1.0, v_scale=1.0):
    """Host tensors (q [T, QH, D]; the caches as float32 or 64 values of their codes) -> out, lse and the bound on out's error.

    Bound: each weight and the result are rounded to bf16 (2^-8 of the value each); scores are fp32 sums over D terms and go through a
    few more fp32 roundings on their way into the exponential (16 of them counted), which moves a weight by that much, and the sum
    by as much again."""
    T, QH, D = q.shape
    KVH, ps = cache_k.shape[1], cache_k.shape[2]
    G = QH // KVH
    out = torch.zeros(q.shape, dtype=torch.float64)
    lse = torch.full((T, QH), -math.inf, dtype=torch.float64)
    tol = torch.zeros(q.shape, dtype=torch.float64)
    cap = len(table[0]) * ps
    for b in range(len(seq)):
        lo, hi = q_start[b], q_start[b + 1]
        n, m = hi - lo, min(seq[b], cap)
        if n == 0 or m <= 0:
            continue
        k, v, ok = gather(cache_k, cache_v, table[b], m, ps)
        k, v = k * k_scale, v * v_scale
        j = torch.arange(m)
        for i in range(n):
            pos = m - n + i
            seen = ok & (j <= pos)
            if window:
                seen &= (j > pos - window) | (j < sinks)
            at = j[seen]
            if at.numel() == 0:
                continue
            for h in range(QH):
                kk, vv, qq = k[at, h // G], v[at, h // G], q[lo + i, h].double()
                z = scale * (kk @ qq)
                w = torch.softmax(z, 0)
                out[lo + i, h] = w @ vv
                lse[lo + i, h] = torch.logsumexp(z, 0)
                size = w @ vv.abs()
                shake = (D + 16) * 2.0 ** -24 * float(scale * (kk.abs() @ qq.abs()).max())
                tol[lo + i, h] = 2.0 ** -8 * (size + out[lo + i, h].abs()) * 1.02 + 2 * shake * size
    return out, lse, tol
