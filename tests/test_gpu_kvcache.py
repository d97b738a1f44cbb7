"""lynx_kv_assign and lynx_qk_norm_rope on the GPU against the host oracle (whole numbers exactly; rows within the bounds that their
roundings give), with the cases where bookkeeping goes wrong: nothing to do, pages or rows that run out, requests that end,
shared pages, rows too short, page numbers outside the cache, padding, odd strides, far positions."""
import math

import numpy as np
import pytest
import torch

import attention_ref as ref
import paper_2411_08982_amd as L

pytestmark = pytest.mark.gpu


def i32(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def run_assign(ctx, new, T, ps, table, ring, state, shared=0):
    t, r = i32(table), i32(ring)
    o = L.lynx_kv_assign(i32(ctx), i32(new), T, ps, t, r, i32(state), shared)
    return dict({n: o[n].tolist() for n in o}, table=t.tolist(), ring=r.tolist())


def make_pool(rng, ctx, new, ps, per_row, spare, shared=0):
    """A table that holds ctx, and a ring with `spare` free pages in a random place of the ring."""
    held = [max(ref.pages_needed(min(max(c, 0), per_row * ps), ps), shared) for c in ctx]
    num = shared + sum(h - shared for h in held) + spare + 3
    ids = rng.permutation(num).tolist()
    table = [[-1] * per_row for _ in ctx]
    at = shared
    for row, h in zip(table, held):
        row[:shared] = ids[:shared]
        row[shared:h] = ids[at:at + h - shared]
        at += h - shared
    head = int(rng.integers(0, num))
    ring = [-7] * num
    for i in range(spare):
        ring[(head + i) % num] = ids[at + i]
    return table, ring, [head, spare]


@pytest.mark.parametrize("B,ps,new_hi,ends,spare,T,shared", [
    (1, 16, 1, 0.0, 2, 1, 0),
    (3, 16, 1, 0.0, 0, 3, 0),            # no free page at all: only requests with room in their last page go on
    (64, 16, 1, 0.1, 64, 64, 0),
    (65, 48, 40, 0.2, 500, 3000, 0),
    (200, 64, 9, 0.1, 20, 1500, 2),      # pages run out, shared pages in front
    (200, 64, 9, 0.1, 900, 333, 2),      # rows run out
    (1024, 16, 30, 0.05, 3000, 20000, 0),
    (1000, 128, 3, 0.0, 10, 4100, 1),
    (7, 1024, 900, 0.0, 40, 7000, 0),
    (40, 32, 3, 1.0, 5, 10, 1),          # all end
])
def test_assign_equals_the_oracle(B, ps, new_hi, ends, spare, T, shared):
    rng = np.random.default_rng([B, ps, spare])
    per_row = 40 if ps < 128 else 4
    ctx = [int(c) for c in rng.integers(shared * ps, per_row * ps - new_hi // 2, B)]
    new = [int(n) for n in rng.integers(0, new_hi + 1, B)]
    new = [-int(rng.integers(1, 4)) if rng.random() < ends else n for n in new]
    table, ring, state = make_pool(rng, ctx, new, ps, per_row, spare, shared)
    assert run_assign(ctx, new, T, ps, table, ring, state, shared) == ref.kv_assign(ctx, new, T, ps, table, ring, state, shared)


def test_assign_passes_over_what_does_not_fit_a_row():
    ctx, new = [60, -5, 70, 64, 10, 2 ** 31 - 1, 0], [5, 1, -1, 0, 2 ** 31 - 1, 3, 64]
    table, ring, state = make_pool(np.random.default_rng(3), ctx, new, 16, 4, 9)
    want = ref.kv_assign(ctx, new, 80, 16, table, ring, state)
    got = run_assign(ctx, new, 80, 16, table, ring, state)
    assert want["status"] == [4] and want["seq_len"] == [60, 0, 64, 64, 10, 64, 64] and got == want


def test_assign_with_bad_page_numbers_and_ring_state():
    # page numbers outside the cache give no slot; a ring state outside the ring is brought into it; nothing is written outside
    got = run_assign([16, 16], [1, 3], 6, 16, [[0, 1, 9], [5, 99, 9]], [77, -3, 1], [4, 2])
    assert got["table"] == [[0, -3, 9], [5, 1, 9]] and got["slots"] == [-1, 16, 17, 18, -1, -1] and got["ring_state"] == [0, 0]
    got = run_assign([0], [1], 1, 16, [[3]], [4, 5], [2 ** 31 - 1, 2 ** 31 - 1])
    assert got["table"] == [[5]] and got["slots"] == [-1] and got["status"] == [0]


def test_assign_steps_in_place_and_replayed_as_a_graph():
    """Thirty steps of a batch in which requests grow, end and start again: eager calls, replays of one captured step and the oracle
    go through the same states; seq_len is ctx_len and ring_state goes on from itself."""
    rng = np.random.default_rng(9)
    B, T, ps, per_row = 33, 40, 16, 6
    table, ring, state = make_pool(rng, [0] * B, [0] * B, ps, per_row, 60)

    def device():
        d = dict(len=i32([0] * B), new=i32([0] * B), table=i32(table), ring=i32(ring), state=i32(state))
        d["out"] = dict(q_start=i32([0] * (B + 1)), seq_len=d["len"], positions=i32([0] * T), slots=i32([0] * T), ring_state=d["state"], status=i32([0]))
        return d

    def step(d):
        L.lynx_kv_assign(d["len"], d["new"], T, ps, d["table"], d["ring"], d["state"], out=d["out"])

    eager, captured = device(), device()
    step(eager)
    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(captured)
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        step(captured)
    lens = [0] * B
    for i in range(30):
        new = [int(rng.choice([-1, 0, 1, 1, 1, 1, 2])) for _ in range(B)]
        want = ref.kv_assign(lens, new, T, ps, table, ring, state)
        table, ring, state, lens = want.pop("table"), want.pop("ring"), want["ring_state"], want["seq_len"]
        for d in (eager, captured):
            d["new"].copy_(i32(new))
        step(eager)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for d in (eager, captured):
            assert {n: t.tolist() for n, t in d["out"].items()} == want, i
            assert d["table"].tolist() == table and d["ring"].tolist() == ring, i


# ---- norms and rotation ------------------------------------------------------------------------------------------------

def rope_case(T, QH, KVH, D, ps, fp8, norm, rot, interleaved, far, seed=0, fused=True):
    g = torch.Generator().manual_seed(seed + T)
    W = (QH + 2 * KVH) * D
    qkv = torch.randn(T, W + 8, generator=g).to(torch.bfloat16)[:, :W]     # rows further apart than they are long
    pages = ref.pages_needed(T, ps) + 2
    slots = torch.randperm(pages * ps, generator=g)[:T].int()
    if T > 3:
        slots[1], slots[3] = -1, pages * ps                                 # outside the cache: not written
    w = lambda: (1 + 0.3 * torch.randn(D, generator=g)).to(torch.bfloat16) if norm else None
    return dict(qkv=qkv, wq=w(), wk=w(), slots=slots, pages=pages,
                pos=torch.randint(0, far, (T,), generator=g, dtype=torch.int32),
                freqs=(1e4 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)) if rot else None)


@pytest.mark.parametrize("T,QH,KVH,D,ps,fp8,norm,rot,interleaved,far", [
    (1, 8, 2, 128, 16, False, True, 128, False, 50),
    (37, 8, 2, 128, 16, False, True, 128, True, 4000),
    (130, 4, 4, 64, 48, True, True, 64, False, 100000),
    (50, 5, 1, 64, 32, True, False, 32, True, 2 ** 31 - 1),
    (64, 16, 2, 128, 64, True, True, 64, False, 2 ** 31 - 1),
    (33, 7, 7, 128, 16, False, False, 0, False, 10),
    (19, 3, 1, 64, 1024, False, True, 16, False, 1000000),
    (300, 64, 8, 128, 16, False, False, 112, False, 30000),
])
def test_norm_rope_equals_the_oracle(T, QH, KVH, D, ps, fp8, norm, rot, interleaved, far):
    c = rope_case(T, QH, KVH, D, ps, fp8, norm, rot, interleaved, far)
    dt = torch.float8_e4m3fn if fp8 else torch.bfloat16
    ks, vs = (0.37, 1.9) if fp8 else (1.0, 1.0)
    kc, vc = L.new_cache(c["pages"], KVH, ps, D, dt)
    bits = torch.uint8 if fp8 else torch.int16
    kc.view(bits).fill_(0x55)
    vc.view(bits).fill_(0x55)
    x = torch.zeros(T, c["qkv"].shape[1] + 8, dtype=torch.bfloat16, device="cuda")[:, :c["qkv"].shape[1]]
    x.copy_(c["qkv"])
    q, k, v = (t.unflatten(1, (-1, D)) for t in x.split([QH * D, KVH * D, KVH * D], 1))
    dev = lambda t: None if t is None else t.cuda()
    out = L.lynx_qk_norm_rope(q, k, v, c["pos"].cuda(), c["slots"].cuda(), dev(c["freqs"]), kc, vc, dev(c["wq"]), dev(c["wk"]), 1e-5,
                              interleaved, ks, vs)
    qh, kh, vh = (t.unflatten(1, (-1, D)) for t in c["qkv"].split([QH * D, KVH * D, KVH * D], 1))
    # fp32: sine and cosine 2e-7 off, norm and rotation a dozen roundings of 2^-24: below 3e-6 of the pair's magnitude
    want, size = ref.norm_rope(qh, c["wq"], 1e-5, c["pos"], c["freqs"], interleaved)
    assert bool(((out.cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 3e-6 * size).all())
    want, size = ref.norm_rope(kh, c["wk"], 1e-5, c["pos"], c["freqs"], interleaved)
    wrote_k, wrote_v = torch.zeros(kc.shape, dtype=torch.bool), torch.zeros(vc.shape, dtype=torch.bool)
    kcf, vcf = kc.cpu().float().double(), vc.cpu().float().double()
    for t in range(T):
        s = int(c["slots"][t])
        if not 0 <= s < c["pages"] * ps:
            continue
        gk, gv = kcf[s // ps, :, s % ps], vcf[s // ps, :, :, s % ps]
        wrote_k[s // ps, :, s % ps], wrote_v[s // ps, :, :, s % ps] = True, True
        if fp8:
            # half a step: 2^-4 of the value, or half the least step 2^-9; what is larger than 448 scales becomes 448
            a, b = (want[t] / ks).clamp(-448, 448), (vh[t].double() / vs).clamp(-448, 448)
            assert bool(((gk - a).abs() <= 2.0 ** -4 * a.abs() + 2.0 ** -10 + 3e-6 * size[t] / ks).all())
            assert torch.equal(gv, b.float().to(dt).float().double())
        else:
            assert bool(((gk - want[t]).abs() <= 2.0 ** -8 * want[t].abs() + 3e-6 * size[t]).all())
            assert torch.equal(gv, vh[t].double())
    # every other place of the cache as it was
    assert bool((kc.view(bits).cpu()[~wrote_k] == 0x55).all()) and bool((vc.view(bits).cpu()[~wrote_v] == 0x55).all())


def test_norm_rope_in_place_and_saturating():
    T, QH, KVH, D, ps = 9, 4, 2, 64, 16
    c = rope_case(T, QH, KVH, D, ps, True, True, 64, False, 100)
    x = (c["qkv"].float() * 3).to(torch.bfloat16).cuda()
    x[2, -D:] = 3e38                                          # beyond E4M3: the largest code, not NaN
    x[2, QH * D:QH * D + KVH * D] = 0                            # a row of zeros: no division by zero
    mk = lambda t: [u.unflatten(1, (-1, D)) for u in t.split([QH * D, KVH * D, KVH * D], 1)]
    kc, vc = L.new_cache(c["pages"], KVH, ps, D, torch.float8_e4m3fn)
    q, k, v = mk(x)
    args = (c["pos"].cuda(), c["slots"].cuda(), c["freqs"].cuda(), kc, vc, c["wq"].cuda(), c["wk"].cuda())
    out = L.lynx_qk_norm_rope(q, k, v, *args)
    s = int(c["slots"][2])
    assert bool((vc[s // ps, KVH - 1, :, s % ps].float() == 448).all()) and bool((kc[s // ps, :, s % ps].float() == 0).all())
    y = x.clone()
    q2, k2, v2 = mk(y)
    r = L.lynx_qk_norm_rope(q2, k2, v2, *args, q_out=q2)
    assert r.data_ptr() == y.data_ptr() and torch.equal(q2, out) and torch.equal(y[:, QH * D:], x[:, QH * D:])


def test_a_cache_beyond_4_gib_is_addressed_in_full():
    KVH, ps, D = 8, 64, 128
    pages = 40000                                                # 128 KiB a page: slots at the end lie beyond 2^32 bytes
    kc, vc = L.new_cache(pages, KVH, ps, D)
    assert kc.numel() * 2 > 1 << 32
    slots = [pages * ps - 1, pages * ps - 64, (pages - 7) * ps + 5, 0]
    g = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn(4, h, D, generator=g).to(torch.bfloat16).cuda() for h in (8, KVH, KVH))
    L.lynx_qk_norm_rope(q, k, v, i32([0, 1, 2, 3]), i32(slots), None, kc, vc)
    for t, s in enumerate(slots):
        assert torch.equal(kc[s // ps, :, s % ps], k[t]) and torch.equal(vc[s // ps, :, :, s % ps], v[t])
    # and attention reads there: each token alone in its sequence
    table = i32([[s // ps] for s in slots])
    kc[slots[0] // ps, :, 0], vc[slots[0] // ps, :, :, 0] = k[0], v[0]
    kc[slots[2] // ps, :, 0], vc[slots[2] // ps, :, :, 0] = k[2], v[2]
    out = L.lynx_attention(q, kc, vc, table, i32([0, 1, 2, 3, 4]), i32([1, 1, 1, 1]), 1)
    want = v.clone()
    want[0] = want[1] = vc[pages - 1, :, :, 0]                       # requests 0 and 1 share the last page
    assert torch.equal(out, want)


def test_refusals_of_the_binding():
    q = torch.zeros(4, 4, 128, dtype=torch.bfloat16, device="cuda")
    kc, vc = L.new_cache(2, 2, 16, 128)
    z = i32([0, 0, 0, 0])
    k = q[:, :2]
    with pytest.raises(ValueError, match="positions"):
        L.lynx_qk_norm_rope(q, k.contiguous(), k.contiguous(), z[:3], z, None, kc, vc)
    with pytest.raises(ValueError, match="contiguous"):
        L.lynx_qk_norm_rope(q.transpose(0, 1), k, k, z, z, None, kc, vc)
    with pytest.raises(ValueError, match="shapes"):
        L.lynx_qk_norm_rope(q, q, q, z, z, None, kc, vc)
    with pytest.raises(TypeError, match="bfloat16"):
        L.lynx_qk_norm_rope(q.float(), k, k, z, z, None, kc, vc)
    with pytest.raises(L.LynxError, match="16 bytes"):
        flat = torch.zeros(4 * 512 + 8, dtype=torch.bfloat16, device="cuda")
        L.lynx_qk_norm_rope(flat[1:2049].view(4, 4, 128), k, k, z, z, None, kc, vc)
    with pytest.raises(ValueError, match="block_table"):
        L.lynx_kv_assign(z, z, 4, 16, z, z, z[:2])
    with pytest.raises(ValueError, match="ring_state"):
        L.lynx_kv_assign(z, z, 4, 16, z.view(4, 1), z, z)
    with pytest.raises(ValueError, match="workspace"):
        L.lynx_attention(q, kc, vc, z.view(4, 1), i32([0, 1, 2, 3, 4]), z, 1, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError, match="prefix_table"):
        L.lynx_attention_prefix(q, kc, vc, z.view(4, 1), i32([0, 1, 2, 3, 4]), z, 1, z, 10)
