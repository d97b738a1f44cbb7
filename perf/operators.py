"""The attention half of a serving engine's step, as cases that can be timed and checked.

Around the MoE layer of a decode step stand: the assignment of cache pages to the step's tokens (lynx_kv_assign), the norms
and the rotation of queries and keys with the write into the paged cache (lynx_qk_norm_rope), the attention over the cache
(lynx_attention: any mix of single tokens and prompt chunks, full or with a sliding window and first tokens that stay
visible), and the attention of a batch that shares a long prefix (lynx_attention_prefix).  Head layouts are generic ones
(groups of 1 to 16 query heads per key head, 64 or 128 channels).

Cache layout: keys [pages, key heads, page, D], values [pages, key heads, D, page]; page numbers are scattered over the pool
as a pool in use has them.  Request lengths are part of a case (drawn from its `lens` number), values come from the seed.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False      # True: run() calls the library; False: it computes the plain forms

EPS = 1e-6
THETA = 1000000.0
KSCALE, VSCALE = 0.75, 1.25     # of 8-bit caches in the attention cases


def _attn(kind, B, new, ctx, heads, page, lens, window=0, sinks=0, fp8=False, prefix=0, name=None):
    QH, KVH, D = heads
    c = dict(kind=kind, B=B, new_lo=new[0], new_hi=new[1], ctx_lo=ctx[0], ctx_hi=ctx[1], QH=QH, KVH=KVH, D=D, page=page,
             lens=lens, window=window, sinks=sinks, fp8=fp8, prefix=prefix)
    if name:
        c["name"] = name
    return c


def _rope(T, heads, page, far, norm=True, rot=0, interleaved=False, fp8=False, name=None):
    QH, KVH, D = heads
    c = dict(kind="rope", T=T, QH=QH, KVH=KVH, D=D, page=page, far=far, norm=norm, rot=rot or D, interleaved=interleaved, fp8=fp8)
    if name:
        c["name"] = name
    return c


def _assign(B, new, ctx, page, lens, ends=0.0, name=None):
    c = dict(kind="assign", B=B, new_lo=new[0], new_hi=new[1], ctx_lo=ctx[0], ctx_hi=ctx[1], page=page, lens=lens, ends=ends)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # A decode step of 64 sequences: the bookkeeping before the first layer.  Latency only.
        _assign(64, (1, 1), (1, 9000), 16, 1, name="assign_64"),
        # A full batch with prompt chunks among the decoding sequences, some of which end and hand their pages back.
        _assign(1000, (1, 60), (0, 4000), 64, 2, ends=0.05, name="assign_1000_chunks"),
        # Queries and keys of a small decode batch.  Latency.
        _rope(32, (32, 4, 128), 16, 40000, name="rope_32"),
        # A prompt chunk deep inside a very long context: the angles of far positions.
        _rope(8001, (32, 8, 128), 64, 1000000, name="rope_8001_far"),
        # One sequence decoding alone: too few rows to fill the chip without cutting the context.
        _attn("attention", 1, (1, 1), (9000, 9000), (32, 8, 128), 16, 3, name="decode_1x9001"),
        # A decode batch of ragged contexts: reading the cache is all there is.
        _attn("attention", 64, (1, 1), (500, 12000), (32, 4, 128), 16, 4, name="decode_64"),
        # A large decode batch with a sliding window, first tokens that stay visible and an 8-bit cache.
        _attn("attention", 256, (1, 1), (100, 16000), (32, 8, 128), 64, 5, window=2048, sinks=4, fp8=True, name="decode_256_window_fp8"),
        # Prompt chunks: the matrix products carry it.
        _attn("attention", 5, (700, 2048), (0, 9000), (32, 8, 128), 64, 6, name="chunks_5"),
        # Decoding sequences and prompt chunks in one step, small heads, a short window.
        _attn("attention", 40, (1, 400), (0, 6000), (64, 8, 64), 32, 7, window=1000, sinks=4, name="mixed_40_d64"),
        # A few sequences behind one system prompt, a key head per query head.
        _attn("prefix", 12, (1, 1), (0, 300), (16, 16, 128), 16, 8, prefix=2000, name="prefix_12x2000"),
        # Many sequences behind one long document.
        _attn("prefix", 256, (1, 1), (10, 2000), (32, 4, 128), 64, 9, prefix=30000, name="prefix_256x30000"),
        # Several drafted tokens per sequence to verify, 8-bit cache; the prefix ends inside a page.
        _attn("prefix", 100, (2, 5), (0, 700), (32, 8, 128), 32, 10, fp8=True, prefix=8011, name="prefix_100x8011_fp8"),
    ]


def _size(rng, lo, hi):
    return int(round(2.0 ** rng.uniform(math.log2(lo), math.log2(hi))))


def _cost(c):
    w = work(c)
    return w["bytes"] / 6e6 + w["flops"] / 4e8


def draw(rng):
    limit = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["assign", "rope", "attention", "attention", "attention", "prefix", "prefix"])
        page = rng.choice([16, 16, 32, 48, 64, 128])
        lens = rng.randrange(1 << 30)
        KVH = rng.choice([1, 2, 4, 4, 8, 8, 16])
        QH = KVH * rng.choice([g for g in (1, 2, 4, 5, 7, 8, 16) if g * KVH <= 64])
        heads = (QH, KVH, rng.choice([64, 128, 128]))
        fp8 = rng.random() < 0.35
        if kind == "assign":
            B, hi = _size(rng, 1, 1000), rng.choice([1, 1, 4, 64])
            c = _assign(B, (1, hi), (0, _size(rng, 100, 20000)), page, lens, ends=rng.choice([0.0, 0.05]))
        elif kind == "rope":
            D = heads[2]
            c = _rope(_size(rng, 1, 8000), heads, page, _size(rng, 1000, 2000000), norm=rng.random() < 0.6,
                      rot=rng.choice([D, D, D // 2]), interleaved=rng.random() < 0.3, fp8=fp8)
        else:
            window = rng.choice([0, 0, _size(rng, 100, 5000)]) if kind == "attention" else 0
            style = rng.choice(["decode", "decode", "draft", "chunk"] if kind == "attention" else ["decode", "decode", "draft"])
            if style == "chunk":
                B, new = _size(rng, 1, 16), (1, _size(rng, 20, 2000))
            else:
                B, new = _size(rng, 1, 300), (1, 1 if style == "decode" else rng.randint(2, 6))
            ctx = (0, _size(rng, 50, 20000 if kind == "attention" else 2000))
            prefix = _size(rng, 200, 30000) if kind == "prefix" else 0
            c = _attn(kind, B, new, ctx, heads, page, lens, window, rng.choice([0, 1, 4, 30]) if window else 0, fp8, prefix)
            shown = sum(ctx) + new[1] if not window else min(sum(ctx), window) + new[1] + 30
            if B * QH * new[1] * shown * 4 > 6 << 30 or B * (shown + 1) * heads[1] * heads[2] * 4 > 8 << 30 or \
                    B * QH * new[1] * prefix * 4 > 6 << 30 or B * sum(ctx) * heads[1] * heads[2] * 4 > 24 << 30:
                continue
        if _cost(c) <= limit:
            return c


# ---- what a case's lengths are ---------------------------------------------------------------------------------------

def _lengths(c):
    """(tokens already cached, new tokens) per request, numpy int64; the shared prefix counts as cached."""
    rng = np.random.default_rng([int(c["lens"]), 77])
    B = c["B"]
    spread = lambda lo, hi: np.minimum(hi, np.floor(np.exp(rng.uniform(math.log(lo + 1), math.log(hi + 2), B)) - 1).astype(np.int64))
    ctx = np.maximum(spread(c["ctx_lo"], c["ctx_hi"]), c["ctx_lo"]) + c.get("prefix", 0)
    new = np.maximum(spread(c["new_lo"], c["new_hi"]), c["new_lo"])
    if c["kind"] == "assign" and c["ends"]:
        new[rng.random(B) < c["ends"]] = -1
    return ctx, new


def _shown(c):
    """Per request: tokens of its own (behind the prefix) that some new token sees, and visible (token, cached token) pairs."""
    ctx, new = _lengths(c)
    P, W, S = c["prefix"], c["window"], c["sinks"]
    tokens, pairs = [], 0
    for a, n in zip(ctx.tolist(), new.tolist()):
        if not W:
            tokens.append(a + n - P)
            pairs += n * (a + 1) + n * (n - 1) // 2
        else:
            lo = max(0, a - W + 1)
            tokens.append(a + n - lo + min(S, lo))
            p = np.arange(a, a + n)
            first = np.maximum(0, p - W + 1)
            pairs += int((p - first + 1 + np.minimum(S, first)).sum())
    return tokens, pairs


def work(c):
    e = 1 if c.get("fp8") else 2
    if c["kind"] == "assign":
        ctx, new = _lengths(c)
        n = np.maximum(new, 0)
        pages = int((-(-(ctx + n) // c["page"]) + (-ctx // c["page"])).sum())
        return {"bytes": 16 * c["B"] + 8 * int(n.sum()) + 8 * pages, "flops": 0}
    if c["kind"] == "rope":
        T, q, k = c["T"], c["QH"] * c["D"], c["KVH"] * c["D"]
        return {"bytes": T * (4 * q + 4 * k + 2 * k * e + 8), "flops": T * (q + k) * 10}
    tokens, pairs = _shown(c)
    T = int(_lengths(c)[1].sum())
    return {"bytes": 4 * T * c["QH"] * c["D"] + (sum(tokens) + c["prefix"]) * c["KVH"] * c["D"] * 2 * e,
            "flops": 4 * pairs * c["QH"] * c["D"]}


# ---- inputs ------------------------------------------------------------------------------------------------------------

def _dev(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a), device="cuda").to(dtype)


def _normal(g, shape, dtype, std=1.0):
    """N(0, std^2) in `dtype`, drawn in slices so that no large 32-bit copy is held."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    step = 1 << 28
    for s in range(0, flat.numel(), step):
        m = min(step, flat.numel() - s)
        flat[s:s + m] = (torch.randn(m, generator=g, device="cuda", dtype=torch.float32) * std).to(dtype)
    return out


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 13)
    rng = np.random.default_rng([int(seed), 5])
    cache = torch.float8_e4m3fn if c.get("fp8") else torch.bfloat16
    ps = c["page"]
    s = {"case": c}
    if c["kind"] == "assign":
        ctx, new = _lengths(c)
        have = -(-ctx // ps)
        need = -(-(ctx + np.maximum(new, 0)) // ps)
        pool = int(need.sum()) + 64
        ids = rng.permutation(pool)
        table = np.full((c["B"], int(need.max()) + 2), -1)
        table[np.arange(table.shape[1])[None, :] < have[:, None]] = ids[:int(have.sum())]
        free, head = ids[int(have.sum()):], int(rng.integers(0, pool))
        ring = np.full(pool, -1)
        ring[(head + np.arange(free.size)) % pool] = free
        s.update(ctx=_dev(ctx), new=_dev(new), table=_dev(table), ring=_dev(ring), state=_dev(np.array([head, free.size])),
                 T=int(np.maximum(new, 0).sum()) + 3)       # three rows more than there are tokens, as a fixed batch has
    elif c["kind"] == "rope":
        T, QH, KVH, D = c["T"], c["QH"], c["KVH"], c["D"]
        pages = -(-T // ps) + 3
        qkv = _normal(g, (T, (QH + 2 * KVH) * D), torch.bfloat16)
        slots = rng.permutation(pages)[np.arange(T) // ps] * ps + np.arange(T) % ps      # runs of a page, pages scattered
        slots[rng.random(T) < 0.01] = -1
        first = int(rng.integers(0, max(1, c["far"] - T)))
        pos = first + np.arange(T) if T > 256 else rng.integers(0, c["far"], T)
        w = lambda: (1 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(torch.bfloat16) if c["norm"] else None
        s.update(q=qkv[:, :QH * D].view(T, QH, D), k=qkv[:, QH * D:(QH + KVH) * D].view(T, KVH, D),
                 v=qkv[:, (QH + KVH) * D:].view(T, KVH, D), wq=w(), wk=w(), pos=_dev(pos), slots=_dev(slots),
                 freqs=_dev(THETA ** (-np.arange(0, c["rot"], 2) / c["rot"]), torch.float64),
                 kc=_normal(g, (pages, KVH, ps, D), cache), vc=_normal(g, (pages, KVH, D, ps), cache))
    else:
        ctx, new = _lengths(c)
        B, P, KVH, D = c["B"], c["prefix"], c["KVH"], c["D"]
        seq = ctx + new
        held = -(-seq // ps)
        common = P // ps                                     # whole pages of the prefix are shared, the rest is copied
        pages = int((held - common).sum()) + common
        ids = rng.permutation(pages)
        table = np.zeros((B, int(held.max()) + 1), np.int64)
        table[:, :common] = ids[:common]
        behind = (np.arange(table.shape[1])[None, :] >= common) & (np.arange(table.shape[1])[None, :] < held[:, None])
        table[behind] = ids[common:]
        kc, vc = _normal(g, (pages, KVH, ps, D), cache), _normal(g, (pages, KVH, D, ps), cache)
        if P % ps:                                            # the last tokens of the prefix, in every request's own page
            at = torch.as_tensor(table[:, common], device="cuda")
            kc.view(torch.uint8 if c["fp8"] else torch.int16)[at, :, :P % ps] = \
                kc.view(torch.uint8 if c["fp8"] else torch.int16)[at[:1], :, :P % ps]
            vc.view(torch.uint8 if c["fp8"] else torch.int16)[at, :, :, :P % ps] = \
                vc.view(torch.uint8 if c["fp8"] else torch.int16)[at[:1], :, :, :P % ps]
        T = int(new.sum())
        s.update(q=_normal(g, (T, c["QH"], D), torch.bfloat16, 1.5), kc=kc, vc=vc, table=_dev(table),
                 q_start=_dev(np.concatenate([[0], np.cumsum(new)])), seq=_dev(seq), max_new=int(new.max()), max_seq=int(seq.max()),
                 kscale=KSCALE if c["fp8"] else 1.0, vscale=VSCALE if c["fp8"] else 1.0)
        s["prefix_table"] = s["table"][0, :-(-P // ps)].contiguous() if P else None
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------------

def run(s):
    c = s["case"]
    if own:
        import paper_2411_08982_amd as L
        if c["kind"] == "assign":
            r = L.lynx_kv_assign(s["ctx"], s["new"], s["T"], c["page"], s["table"], s["ring"], s["state"])
            return [r["q_start"], r["seq_len"], r["positions"], r["slots"], s["table"], s["ring"], r["ring_state"], r["status"]]
        if c["kind"] == "rope":
            q = L.lynx_qk_norm_rope(s["q"], s["k"], s["v"], s["pos"], s["slots"], s["freqs"], s["kc"], s["vc"], q_weight=s["wq"],
                                    k_weight=s["wk"], eps=EPS, interleaved=c["interleaved"])
            return [q, s["kc"], s["vc"]]
        if c["kind"] == "attention":
            return L.lynx_attention(s["q"], s["kc"], s["vc"], s["table"], s["q_start"], s["seq"], s["max_new"], window=c["window"],
                                    sinks=c["sinks"], k_scale=s["kscale"], v_scale=s["vscale"])
        return L.lynx_attention_prefix(s["q"], s["kc"], s["vc"], s["table"], s["q_start"], s["seq"], s["max_new"],
                                       s["prefix_table"], c["prefix"], k_scale=s["kscale"], v_scale=s["vscale"])
    return {"assign": _plain_assign, "rope": _plain_rope, "attention": _plain_attention, "prefix": _plain_prefix}[c["kind"]](s)


# ---- the plain forms -----------------------------------------------------------------------------------------------------

def _plain_assign(s):
    ps, T, table, ring = s["case"]["page"], s["T"], s["table"], s["ring"]
    ctx, new = s["ctx"].long(), s["new"].long()
    n, head, count, size = new.clamp(min=0), s["state"][0].long(), s["state"][1].long(), ring.numel()
    have, total = (ctx + ps - 1) // ps, (ctx + n + ps - 1) // ps
    q_end = n.cumsum(0)
    taken = torch.where(new < 0, 0, total - have)
    taken_end = taken.cumsum(0)
    back = torch.where(new < 0, have, 0)
    back_end = back.cumsum(0)
    col = torch.arange(table.shape[1], device="cuda")[None, :]
    # pages that are handed back go behind the free ones, in request and page order
    gone = col < back[:, None]
    at = (head + count + (back_end - back)[:, None] + col) % size
    ring[at[gone]] = table[gone]
    # new pages from the front of the ring
    fresh = (col >= have[:, None]) & (col < (have + taken)[:, None])
    from_ring = ring[(head + (taken_end - taken)[:, None] + col - have[:, None]) % size]
    table.copy_(torch.where(fresh, from_ring, table))
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(q_end, t, right=True).clamp(max=n.numel() - 1)
    real = t < q_end[-1]
    pos = torch.where(real, ctx[b] + t - (q_end - n)[b], 0)
    slots = torch.where(real, table[b, pos // ps].long() * ps + pos % ps, -1)
    moved = taken_end[-1]
    return [torch.cat([torch.zeros_like(q_end[:1]), q_end]).int(), torch.where(new < 0, 0, ctx + n).int(), pos.int(), slots.int(),
            table, ring, torch.stack([(head + moved) % size, count - moved + back_end[-1]]).int(),
            torch.zeros(1, dtype=torch.int32, device="cuda")]


def _plain_rope(s):
    c = s["case"]
    ps, rot = c["page"], c["rot"]
    turns = torch.frac(s["pos"].double()[:, None] * s["freqs"][None, :] / (2 * math.pi)) * (2 * math.pi)
    cos, sin = turns.cos().float()[:, None, :], turns.sin().float()[:, None, :]

    def norm(x, w):
        x = x.float()
        return x if w is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()

    def turn(x):
        if c["interleaved"]:
            a, b = x[..., 0:rot:2], x[..., 1:rot:2]
            return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., rot:]], -1)
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., rot:]], -1)

    def to_cache(x):
        return (x.float().clamp(-448, 448) if c["fp8"] else x.float()).to(s["kc"].dtype)

    bits = torch.uint8 if c["fp8"] else torch.int16
    keep = s["slots"] >= 0
    at = s["slots"][keep].long()
    s["kc"].view(bits)[at // ps, :, at % ps] = to_cache(turn(norm(s["k"], s["wk"])))[keep].view(bits)
    s["vc"].view(bits)[at // ps, :, :, at % ps] = to_cache(s["v"])[keep].view(bits)
    return [turn(norm(s["q"], s["wq"])).to(torch.bfloat16), s["kc"], s["vc"]]


def _gathered(s, j):
    """Keys and values [B, key heads, tokens, D] in 32 bits of the tokens j [B, n]."""
    ps = s["case"]["page"]
    page = s["table"].gather(1, j // ps).long()
    k = s["kc"][page, :, j % ps].float() * s["kscale"]
    v = s["vc"][page, :, :, j % ps].float() * s["vscale"]
    return k.transpose(1, 2), v.transpose(1, 2)


def _padded(s):
    """Row of q for (request, new token) [B, max_new], which of them exist, and their positions."""
    start, i = s["q_start"][:-1].long()[:, None], torch.arange(s["max_new"], device="cuda")[None, :]
    n = (s["q_start"][1:] - s["q_start"][:-1]).long()[:, None]
    return torch.where(i < n, start + i, 0), i < n, s["seq"].long()[:, None] - n + i


def _scores(s, q, k):
    """q [B, n, QH, D], k [B, KVH, m, D] -> [B, KVH, G, n, m]."""
    B, n, QH, D = q.shape
    KVH = k.shape[1]
    q = q.view(B, n, KVH, QH // KVH, D).permute(0, 2, 3, 1, 4).reshape(B, KVH, QH // KVH * n, D)
    return (q @ k.transpose(-1, -2)).view(B, KVH, QH // KVH, n, -1) * (1 / math.sqrt(D))


def _plain_attention(s):
    c = s["case"]
    W, S = c["window"], c["sinks"]
    row, real, pos = _padded(s)
    seq = s["seq"].long()[:, None]
    if W:
        # the first tokens, then from the first token that the first new one sees
        lo = (pos[:, :1] - W + 1).clamp(min=S)
        j = torch.arange(min(S + W + s["max_new"] - 1, s["max_seq"] + S), device="cuda")[None, :]
        j = torch.where(j < S, j, lo + j - S)
    else:
        j = torch.arange(s["max_seq"], device="cuda")[None, :].expand(seq.shape[0], -1)
    seen = (j < seq)[:, None, :] & (j[:, None, :] <= pos[:, :, None])
    if W:
        seen &= (j[:, None, :] > pos[:, :, None] - W) | (j[:, None, :] < S)
    k, v = _gathered(s, torch.where(j < seq, j, 0))
    z = _scores(s, s["q"][row].float(), k)
    z.masked_fill_(~seen[:, None, None], -math.inf)
    z -= z.amax(-1, keepdim=True)
    z.exp_()
    total = z.sum(-1, keepdim=True)
    B, KVH, G, n, m = z.shape
    o = (z.view(B, KVH, G * n, m) @ v).view(B, KVH, G, n, -1) / total
    return o.permute(0, 3, 1, 2, 4).reshape(B, n, c["QH"], c["D"])[real].to(torch.bfloat16)


def _plain_prefix(s):
    c = s["case"]
    P, ps, KVH, D = c["prefix"], c["page"], c["KVH"], c["D"]
    G = c["QH"] // KVH
    # the prefix: one product per key head for the rows of the whole batch
    j = torch.arange(P, device="cuda")
    page = s["prefix_table"][j // ps].long()
    kp = s["kc"][page, :, j % ps].float().transpose(0, 1) * s["kscale"]           # [KVH, P, D]
    vp = s["vc"][page, :, :, j % ps].float().transpose(0, 1) * s["vscale"]
    T = s["q"].shape[0]
    q = s["q"].float().view(T, KVH, G, D).permute(1, 0, 2, 3).reshape(KVH, T * G, D)
    z = (q @ kp.transpose(-1, -2)) * (1 / math.sqrt(D))
    mp = z.amax(-1, keepdim=True)
    z -= mp
    z.exp_()
    lp, op = z.sum(-1, keepdim=True), z @ vp
    # each request's own tokens
    row, real, pos = _padded(s)
    seq = s["seq"].long()[:, None]
    j = P + torch.arange(s["max_seq"] - P, device="cuda")[None, :].expand(seq.shape[0], -1)
    k, v = _gathered(s, torch.where(j < seq, j, 0))
    z = _scores(s, s["q"][row].float(), k)
    z.masked_fill_(~(j[:, None, :] <= pos[:, :, None])[:, None, None], -math.inf)
    mo = z.amax(-1, keepdim=True)
    z -= mo
    z.exp_()
    B, _, _, n, m = z.shape
    lo, oo = z.sum(-1, keepdim=True), (z.view(B, KVH, G * n, m) @ v).view(B, KVH, G, n, D)
    back = lambda x: x.permute(0, 3, 1, 2, 4).reshape(B, n, c["QH"], -1)[real]     # -> [T, QH, .]
    mo, lo, oo = back(mo), back(lo), back(oo)
    flat = lambda x: x.view(KVH, T, G, -1).permute(1, 0, 2, 3).reshape(T, c["QH"], -1)
    mp, lp, op = flat(mp), flat(lp), flat(op)
    top = torch.maximum(mp, mo)
    a, b = (mp - top).exp(), (mo - top).exp()
    return ((a * op + b * oo) / (a * lp + b * lo)).to(torch.bfloat16)


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    ps = c["page"]
    if c["kind"] == "assign":
        return None                                            # whole numbers only
    if c["kind"] == "rope":
        T, D, rot = c["T"], c["D"], c["rot"]
        angle = s["pos"].double().view(T, 1, 1) * s["freqs"].view(1, 1, -1)
        first, second = (slice(0, rot, 2), slice(1, rot, 2)) if c["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))

        def whole(x, w):
            x = x.double()
            if w is not None:
                x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / D + EPS) * w.double()
            y = x.clone()
            z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.ones_like(angle), angle)
            y[..., first], y[..., second] = z.real, z.imag
            return y

        kc, vc = s["kc"].double(), s["vc"].double()
        kk, at = whole(s["k"], s["wk"]), s["slots"].long()
        if c["fp8"]:
            kk = kk.clamp(-448, 448)
        t = torch.arange(T, device="cuda")[at >= 0]
        at = at[at >= 0]
        kc[at // ps, :, at % ps] = kk[t]
        vc[at // ps, :, :, at % ps] = s["v"].double()[t]
        return [whole(s["q"], s["wq"]), kc, vc]
    _, pairs = _shown(c)
    if 4 * pairs * c["QH"] * c["D"] > 4e12:
        return None
    KVH, G, D, W, S = c["KVH"], c["QH"] // c["KVH"], c["D"], c["window"], c["sinks"]
    ends, seq = s["q_start"].tolist(), s["seq"].tolist()
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        n, m = ends[b + 1] - ends[b], seq[b]
        lo = max(0, m - n - W + 1) if W else 0
        j = torch.tensor(list(range(min(S, lo))) + list(range(lo, m)), device="cuda")
        page = s["table"][b].long()[j // ps]
        k = s["kc"][page, :, j % ps].double() * s["kscale"]      # [m, KVH, D]
        v = s["vc"][page, :, :, j % ps].double() * s["vscale"]
        pos = torch.arange(m - n, m, device="cuda")
        hidden = j[None, :] > pos[:, None]
        if W:
            hidden |= (j[None, :] <= pos[:, None] - W) & (j[None, :] >= S)
        for h in range(KVH):
            q = s["q"][ends[b]:ends[b + 1], h * G:(h + 1) * G].double()
            z = torch.tensordot(q, k[:, h], dims=([2], [1])) / math.sqrt(D)
            p = torch.softmax(z.masked_fill(hidden[:, None, :], -math.inf), -1)
            out[ends[b]:ends[b + 1], h * G:(h + 1) * G] = torch.tensordot(p, v[:, h], dims=1)
    return out
