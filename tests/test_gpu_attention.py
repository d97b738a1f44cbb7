"""lynx_attention and lynx_attention_prefix on the GPU against the host oracle in 64 bits, within bounds that follow from the roundings
(tests/attention_ref.py).  Every cache slot that no token occupies holds NaN."""
import math

import numpy as np
import pytest
import torch

import attention_ref as ref
import paper_2411_08982_amd as L

pytestmark = pytest.mark.gpu


def i32(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


class Case:
    """Requests of (tokens in the cache, new tokens), a cache of scattered pages filled with their keys and values, NaN elsewhere."""

    def __init__(self, lens, QH, KVH, D, ps, fp8=False, seed=0, prefix=0, peak=2.0, pad=3, spare=2):
        g = torch.Generator().manual_seed(seed * 1000 + len(lens) * 10 + D)
        self.B, self.QH, self.KVH, self.D, self.ps, self.fp8, self.prefix = len(lens), QH, KVH, D, ps, fp8, prefix
        self.seq = [c + n for c, n in lens]
        self.q_start = [0] + np.cumsum([n for _, n in lens]).tolist()
        self.rows = self.q_start[-1]
        self.T = self.rows + pad
        self.max_new = max(n for _, n in lens)
        dt = torch.float8_e4m3fn if fp8 else torch.bfloat16
        self.ks, self.vs = (0.5, 1.7) if fp8 else (1.0, 1.0)
        common = prefix // ps
        held = [max(ref.pages_needed(s, ps), common) for s in self.seq]
        pages = common + sum(h - common for h in held) + spare
        ids = torch.randperm(pages, generator=g).tolist()
        per_row = max(held) + 1 if held else 1
        self.table = [[-1] * per_row for _ in lens]
        kc, vc = torch.full((pages, KVH, ps, D), math.nan), torch.full((pages, KVH, D, ps), math.nan)
        shared_k = [torch.randn(KVH, D, generator=g) for _ in range(prefix)]
        shared_v = [torch.randn(KVH, D, generator=g) for _ in range(prefix)]
        at = common
        for b, h in enumerate(held):
            self.table[b][:common] = ids[:common]
            self.table[b][common:h] = ids[at:at + h - common]
            at += h - common
            for j in range(self.seq[b]):
                k, v = (shared_k[j], shared_v[j]) if j < prefix else (torch.randn(KVH, D, generator=g), torch.randn(KVH, D, generator=g))
                kc[self.table[b][j // ps], :, j % ps], vc[self.table[b][j // ps], :, :, j % ps] = k, v
        # the prefix through a table of its own; the page it ends in may be any copy of it
        self.prefix_table = ids[:common] + ([next(self.table[b][common] for b in range(self.B) if self.seq[b] >= prefix)] if prefix % ps else [])
        self.kc, self.vc = kc.to(dt).cuda(), vc.to(dt).cuda()
        self.q = (torch.randn(self.T, QH, D, generator=g) * peak).to(torch.bfloat16)

    def expect(self, scale, window=0, sinks=0):
        return ref.attention(self.q, self.kc.float().cpu(), self.vc.float().cpu(), self.table, self.q_start, self.seq, scale, window, sinks,
                             self.ks, self.vs)

    def run(self, window=0, sinks=0, scale=None, max_new=None, q=None, **kw):
        q = self.q.cuda() if q is None else q
        args = (q, self.kc, self.vc, i32(self.table), i32(self.q_start), i32(self.seq), self.max_new if max_new is None else max_new)
        if self.prefix:
            return L.lynx_attention_prefix(*args, i32(self.prefix_table), self.prefix, scale, self.ks, self.vs, **kw)
        return L.lynx_attention(*args, scale, window, sinks, self.ks, self.vs, **kw)

    def check(self, window=0, sinks=0, scale=None, **kw):
        out = torch.full((self.T, self.QH, self.D), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((self.T, self.QH), 7.0, dtype=torch.float32, device="cuda")
        self.run(window, sinks, scale, out=out, lse=lse, **kw)
        want, want_lse, tol = self.expect(self.D ** -0.5 if scale is None else scale, window, sinks)
        o, l, n = out.cpu().double(), lse.cpu().double(), self.rows
        assert bool((o[n:] == 7).all()) and bool((l[n:] == 7).all()), "rows behind the last request"
        worst = ((o[:n] - want[:n]).abs() - tol[:n]).max().item() if n else 0
        # (a length beyond what was ever cached makes a request see NaN: so do oracle and kernel)
        wild = torch.isnan(want[:n])
        assert torch.equal(wild, torch.isnan(o[:n]))
        assert bool(((o[:n] - want[:n]).abs() <= tol[:n])[~wild].all()), worst
        none, lost = torch.isinf(want_lse[:n]), torch.isnan(want_lse[:n])
        assert torch.equal(none, torch.isinf(l[:n]) & (l[:n] < 0)) and bool((o[:n][none] == 0).all())
        # scores 144 roundings of 2^-24 off at most, as in the bound of out; the logarithm a few more
        assert bool(((l[:n] - want_lse[:n])[~none & ~lost].abs() <= 2e-5 * (1 + want_lse[:n][~none & ~lost].abs())).all())
        return out, lse


EDGES = [(0, 1), (15, 1), (16, 1), (31, 1), (63, 1), (64, 1), (65, 1), (300, 1), (0, 0), (777, 1), (128, 0)]
MIXED = [(0, 1), (5, 40), (130, 3), (0, 70), (257, 1), (64, 2), (0, 0), (99, 17)]


@pytest.mark.parametrize("lens", [EDGES, MIXED], ids=["decode", "mixed"])
@pytest.mark.parametrize("QH,KVH,D,ps,fp8,window,sinks", [
    (8, 2, 128, 16, False, 0, 0),
    (4, 4, 64, 48, False, 0, 0),
    (5, 1, 128, 64, True, 0, 0),
    (32, 1, 64, 32, False, 50, 4),           # 32 rows per token, window and first tokens
    (6, 2, 128, 1024, True, 64, 70),         # first tokens longer than the window
    (16, 2, 64, 16, True, 1, 0),             # a token sees itself only
    (7, 1, 128, 16, False, 100, 1),
    (2, 2, 64, 16, True, 1000, 4),           # a window wider than most contexts
])
def test_attention_equals_the_oracle(lens, QH, KVH, D, ps, fp8, window, sinks):
    Case(lens, QH, KVH, D, ps, fp8).check(window, sinks)


@pytest.mark.parametrize("lens,QH,KVH,D,ps,fp8,window,sinks", [
    ([(0, 1)], 1, 1, 64, 16, False, 0, 0),
    ([(2999, 1)], 8, 1, 128, 16, False, 0, 0),          # one long context, cut into many parts
    ([(5000, 1)], 4, 2, 64, 64, True, 3000, 4),
    ([(4100, 3), (10, 1)], 4, 1, 128, 48, True, 0, 0),
    ([(0, 300)], 4, 2, 128, 16, False, 0, 0),           # a prompt from the start
    ([(1000, 257)], 8, 2, 64, 32, False, 200, 4),
    ([(63, 129), (64, 128), (65, 127), (1, 1)], 2, 1, 128, 64, True, 0, 0),
    ([(i * 7 % 90, 1 + i % 2) for i in range(150)], 4, 2, 64, 16, False, 0, 0),
    ([(0, 200), (700, 150)], 6, 2, 128, 16, True, 33, 3),
])
def test_attention_of_long_contexts_and_prompts(lens, QH, KVH, D, ps, fp8, window, sinks):
    Case(lens, QH, KVH, D, ps, fp8, seed=1).check(window, sinks)


def test_a_few_prompts_among_many_single_tokens():
    # both kinds of workgroups, in turns: enough of each for a CU to have one
    Case([(300 + i, 1) for i in range(40)] + [(90, 70)] + [(5, 1)] * 3, 16, 8, 64, 16, seed=19).check()
    Case([(200, 1)] * 20 + [(700, 60)] + [(0, 0)] * 20, 32, 8, 64, 32, True, seed=20).check(window=150, sinks=3)


def test_group_of_many_heads_and_a_large_batch():
    Case([(20, 2), (0, 1), (3, 0), (100, 5)], 256, 1, 64, 16, seed=2).check()
    Case([(i % 5, i % 3) for i in range(1024)], 2, 1, 64, 16, seed=3).check()


@pytest.mark.parametrize("max_new", [0, 1, 5, 1000])
def test_the_hint_of_new_tokens_changes_no_more_than_roundings(max_new):
    Case(MIXED, 8, 2, 128, 16, seed=4).check(max_new=max_new)


def test_scores_far_apart_and_a_scale():
    # weights of one token each: scores hundreds apart, and a scale that is not 1 / sqrt(D)
    Case(EDGES, 4, 2, 128, 16, seed=5, peak=60.0).check(scale=0.25)
    Case(MIXED, 4, 2, 64, 32, seed=6).check(scale=1e-4)


def test_rows_that_see_nothing_and_lengths_that_lie():
    c = Case([(40, 3), (0, 4), (10, 2)], 4, 2, 64, 16, seed=7)
    c.seq[1] = 2                       # fewer tokens than new rows: the first two are at negative positions
    c.seq[2] = 0
    c.check()
    c = Case([(40, 3), (20, 1)], 4, 2, 64, 16, seed=8)
    c.table[0] = [-1] * len(c.table[0])                # a request whose pages are nowhere: nothing to see
    c.table[1][0] = 10 ** 6
    c.check()
    c.seq[1] = 2 ** 31 - 1                          # longer than its row of the table: cut to it
    c.check()
    c = Case([(30, 1), (20, 2), (3, 1)], 4, 2, 64, 16, seed=9)
    c.q_start = [0, 1, 3, 9]                          # a last row start behind T, one that goes back: clamped, nothing out of bounds
    c.run()
    c.q_start = [-4, 2, 1, 4]
    assert bool(torch.isfinite(c.run()[:2].float()).all())
    torch.cuda.synchronize()


def test_row_ranges_that_overlap_beyond_all_bounds():
    # 512 requests that each claim all rows, a million tokens long: 2^34 blocks to read, more than 32 bits count.  Nothing is read
    B, T, pages = 1024, 4096, 1024
    q_start = i32([0, T] * (B // 2) + [0])
    cache = L.new_cache(2, 1, 1024, 64)
    q = torch.zeros(T, 8, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 7.0)
    L.lynx_attention(q, *cache, torch.zeros(B, pages, dtype=torch.int32, device="cuda"), q_start, i32([pages * 1024] * B), 1, out=out)
    assert bool((out == 7).all())


def test_more_key_heads_than_the_line_has_workgroups():
    Case([(0, 1), (70, 2), (130, 1), (0, 0)], 520, 520, 64, 16, seed=14).check()


@pytest.mark.parametrize("D,KVH,fp8", [(128, 1, False), (64, 2, True)])
def test_the_largest_step(D, KVH, fp8):
    # one prompt of 65536 tokens, the same as 1024 requests, and its second half behind the first as a shared prefix; and a few of its rows
    # by themselves.  Each result is within 2^-8 (sum of weights times |v| + |result|) of the true one, as in the oracle's bound
    T, QH, ps = 65536, 8, 256
    g = torch.Generator(device="cuda").manual_seed(32)
    kc, vc = L.new_cache(T // ps, KVH, ps, D, torch.float8_e4m3fn if fp8 else torch.bfloat16)
    for c in (kc, vc):
        c.copy_(torch.randn(c.shape, generator=g, device="cuda").to(c.dtype))
    q = torch.randn(T, QH, D, generator=g, device="cuda").to(torch.bfloat16)
    table = torch.randperm(T // ps, generator=g, device="cuda").to(torch.int32).view(1, -1)
    biggest = float(vc.view(torch.uint8).view(vc.dtype).float().abs().max())
    full = L.lynx_attention(q, kc, vc, table, i32([0, T]), i32([T]), T)

    def same(part, lo):
        want = full[lo:lo + part.shape[0]].float()
        assert bool(((part.float() - want).abs() <= 2 * 1.02 * 2.0 ** -8 * (biggest + want.abs())).all())
        # (all roundings one way would be that far off; of both signs they are 2^-8 of the result's norm at most, twice, and twice that for good measure)
        assert float((part.float() - want).norm()) <= 4 * 2.0 ** -8 * float(want.norm())

    for lo, n in ((0, 1), (0, 100), (16000, 1), (32000, 20), (65000, 536), (65535, 1), (40000, 300)):
        same(L.lynx_attention(q[lo:lo + n].contiguous(), kc, vc, table, i32([0, n]), i32([lo + n]), n), lo)
    starts, lengths = i32(list(range(0, T + 1, 64))), i32(list(range(64, T + 1, 64)))
    rows = table.expand(1024, -1).contiguous()
    same(L.lynx_attention(q, kc, vc, rows, starts, lengths, 64), 0)
    half = T // 2
    same(L.lynx_attention_prefix(q[half:], kc, vc, rows[512:].contiguous(), starts[:513], lengths[512:].contiguous(), 64, table[0, :half // ps].contiguous(), half), half)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("n", [1, 40])
def test_pages_behind_four_gib(fp8, n):
    # the last pages of caches whose offsets do not fit 32 bits: as in a small cache
    c = Case([(150, n), (70, n)], 8, 2, 128, 64, fp8, seed=15)
    want = c.run()
    far = (5 << 30) // (2 * 64 * 128 * (1 if fp8 else 2))
    small = c.kc.shape[0]
    kc, vc = L.new_cache(far, 2, 64, 128, c.kc.dtype)
    for big, cache in ((kc, c.kc), (vc, c.vc)):
        big.view(torch.uint8)[far - small:].copy_(cache.view(torch.uint8))
    c.kc, c.vc, c.table = kc, vc, [[p if p < 0 else p + far - small for p in row] for row in c.table]
    assert torch.equal(c.run()[:c.rows], want[:c.rows])
    if n == 1:
        want = L.lynx_attention_prefix(c.q.cuda(), kc, vc, i32(c.table), i32(c.q_start), i32(c.seq), 1, i32([c.table[0][0]]), 64)
        c.table[1][0] = 7                              # the prefix's own pages are not read
        got = L.lynx_attention_prefix(c.q.cuda(), kc, vc, i32(c.table), i32(c.q_start), i32(c.seq), 1, i32([c.table[0][0]]), 64)
        assert torch.equal(got[:c.rows], want[:c.rows])


def test_two_graphs_on_one_workspace():
    a, b = Case(MIXED, 8, 2, 128, 16, seed=16), Case([(200 + i, 1 + i % 2) for i in range(20)], 8, 2, 128, 16, seed=17, prefix=200)
    wants = [c.run()[:c.rows] for c in (a, b)]
    ws = torch.empty(max(L.attention_workspace_bytes(c.B, c.T, 8, 2, 128, c.prefix) for c in (a, b)), dtype=torch.uint8, device="cuda")
    graphs, outs = [], []
    for c in (a, b):
        q, out = c.q.cuda(), torch.zeros(c.T, 8, 128, dtype=torch.bfloat16, device="cuda")
        args = (q, c.kc, c.vc, i32(c.table), i32(c.q_start), i32(c.seq), c.max_new)
        extra = (i32(c.prefix_table), c.prefix) if c.prefix else ()
        call = L.lynx_attention_prefix if c.prefix else L.lynx_attention
        call(*args, *extra, out=out, workspace=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(*args, *extra, out=out, workspace=ws)
        graphs.append((g, args, extra))
        outs.append(out)
    for _ in range(4):
        for (g, *_), out, want in zip(graphs, outs, wants):
            out.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out[:want.shape[0]], want)
        ws.fill_(0x7F)


def test_strided_rows():
    c = Case(MIXED, 6, 2, 64, 16, seed=10)
    out, _ = c.check()
    wide = torch.zeros(c.T, 3, 6, 64, dtype=torch.bfloat16, device="cuda")
    wide[:, 1] = c.q.cuda()
    dst = torch.zeros(c.T, 2, 6, 64, dtype=torch.bfloat16, device="cuda")
    c.run(q=wide[:, 1], out=dst[:, 1])
    assert torch.equal(dst[:c.rows, 1], out[:c.rows]) and bool((dst[:, 0] == 0).all())


def test_another_stream_and_two_calls_at_once():
    a, b = Case(EDGES, 8, 2, 128, 16, seed=11), Case(MIXED, 8, 2, 128, 16, seed=12)
    wa, wb = a.run(), b.run()
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(s):
            ga = a.run()
        with torch.cuda.stream(t):
            gb = b.run()
        torch.cuda.synchronize()
        assert torch.equal(wa[:a.rows], ga[:a.rows]) and torch.equal(wb[:b.rows], gb[:b.rows])


def test_results_do_not_depend_on_the_workspace_or_the_call_before():
    c = Case(MIXED + EDGES, 8, 2, 128, 16, seed=13)
    want = c.run()
    ws = L.new_attention_workspace(c.B, c.T, 8, 2, 128)
    for fill in (0x00, 0xFF, 0x7F):
        ws.fill_(fill)
        assert torch.equal(c.run(workspace=ws)[:c.rows], want[:c.rows])
    assert torch.equal(c.run(workspace=ws)[:c.rows], want[:c.rows])


# ---- a shared prefix ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("prefix", [1, 16, 63, 64, 65, 300, 512])
@pytest.mark.parametrize("QH,KVH,D,ps,fp8,new", [(8, 2, 128, 16, False, 1), (4, 4, 64, 48, True, 3), (5, 1, 128, 64, True, 2),
                                                 (32, 1, 64, 32, False, 1)])
def test_prefix_equals_the_oracle(prefix, QH, KVH, D, ps, fp8, new):
    lens = [(prefix + own, n) for own, n in [(0, 1), (1, new), (15, 1), (64, new), (200, 1), (0, 0), (33, new), (7, 0)]]
    Case(lens, QH, KVH, D, ps, fp8, seed=20, prefix=prefix).check()


def test_prefix_of_large_batches_and_long_prefixes():
    Case([(2000 + i % 70, 1 + (i % 4 == 0)) for i in range(90)], 8, 2, 64, 16, seed=21, prefix=2000).check()
    Case([(3333, 1)], 4, 2, 128, 64, seed=22, prefix=3333).check()
    Case([(700 + i, 40) for i in range(3)], 4, 2, 128, 32, True, seed=23, prefix=690).check()


def test_rows_inside_the_prefix_see_what_is_up_to_them():
    # requests that are shorter than the prefix, or end in it
    c = Case([(300, 1), (100, 5), (0, 1), (299, 2), (64, 1)], 4, 2, 64, 16, seed=24, prefix=300)
    c.check()


def test_an_empty_prefix_is_plain_attention():
    c = Case(MIXED, 8, 2, 128, 16, seed=25)
    want = c.run()
    got = L.lynx_attention_prefix(c.q.cuda(), c.kc, c.vc, i32(c.table), i32(c.q_start), i32(c.seq), c.max_new, i32([]), 0)
    assert torch.equal(got[:c.rows], want[:c.rows])


def test_prefix_on_any_workspace():
    c = Case([(200 + i, 1) for i in range(20)], 8, 2, 128, 16, seed=26, prefix=200)
    want = c.run()
    ws = L.new_attention_workspace(c.B, c.T, 8, 2, 128, 200)
    for fill in (0x00, 0xFF, 0x7F):
        ws.fill_(fill)
        assert torch.equal(c.run(workspace=ws)[:c.rows], want[:c.rows])


@pytest.mark.parametrize("prefix,fp8", [(8229, False), (24600, False), (24600, True)])
def test_prefixes_long_enough_that_tiles_and_requests_take_turns(prefix, fp8):
    B, QH, KVH, D, ps, own = 128, 16, 4, 64, 64, 3
    G, common, dt = QH // KVH, prefix // ps, torch.float8_e4m3fn if fp8 else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(31)
    pages = common + B * own
    kc, vc = (torch.randn(shape, generator=g, device="cuda").to(dt) for shape in ((pages, KVH, ps, D), (pages, KVH, D, ps)))
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.cat([order[:common].expand(B, common), order[common:].view(B, own)], 1).contiguous()
    # what every request has of the page that the prefix ends in is the same
    for cache, at in ((kc, (slice(None), slice(0, prefix % ps))), (vc, (slice(None), slice(None), slice(0, prefix % ps)))):
        raw = cache.view(torch.uint8) if fp8 else cache
        raw[(table[:, common].long(),) + at] = raw[(table[0, common].long(),) + at].clone()
    seq = [prefix + 1 + 7 * b % 120 for b in range(B)]
    q = torch.randn(B, QH, D, generator=g, device="cuda").to(torch.bfloat16)
    out = L.lynx_attention_prefix(q, kc, vc, table, i32(list(range(B + 1))), i32(seq), 1, table[0, :-(-prefix // ps)].contiguous(), prefix)
    for b in range(0, B, 5):
        ids = table[b].long()
        k = kc[ids].double().transpose(0, 1).reshape(KVH, -1, D)[:, :seq[b]].contiguous()
        v = vc[ids].double().permute(1, 0, 3, 2).reshape(KVH, -1, D)[:, :seq[b]].contiguous()
        qq = q[b].double().view(KVH, G, D)
        for h in range(KVH):
            w = torch.softmax(qq[h] @ k[h].t().contiguous() * D ** -0.5, 1)
            want, size = w @ v[h], w @ v[h].abs()
            # weights and result are rounded to bf16, 2^-8 of the value each; scores are 80 fp32 roundings off at most, as in the oracle's bound
            shake = (D + 16) * 2.0 ** -24 * float((qq[h].abs() @ k[h].abs().t().contiguous()).max()) * D ** -0.5
            tol = 2.0 ** -8 * (size + want.abs()) * 1.02 + 2 * shake * size
            assert bool(((out[b, h * G:(h + 1) * G].double() - want).abs() <= tol).all()), (b, h)


# ---- all of it together ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fp8", [False, True])
def test_decode_steps_eager_and_as_a_graph(fp8):
    """Steps as an engine makes them: pages assigned, queries and keys normed, rotated and cached, attention over the cache, a MoE
    layer behind it.  One captured step replayed over changing lengths gives what eager calls give, step by step, bit for bit,
    and the first and last step's attention is checked against the oracle."""
    import workloads as wl
    B, T, QH, KVH, D, ps, per_row, steps = 6, 8, 8, 2, 64, 16, 8, 12
    cfg = wl.CONFIGS["tiny"]                                     # hidden 512 = QH * D
    d = wl.make_layer_device(cfg, T, "cuda")
    Wgu, Wdp = L.lynx_pack_weights(d["Wg"], d["Wu"], d["Wd"])
    g = torch.Generator(device="cuda").manual_seed(3)
    Wqkv = (torch.randn(cfg.H, (QH + 2 * KVH) * D, generator=g, device="cuda") / 20).to(torch.bfloat16)
    wq, wk = (1 + torch.rand(2, D, generator=g, device="cuda")).to(torch.bfloat16)
    freqs = 1e4 ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)
    xs = torch.randn(steps, T, cfg.H, generator=g, device="cuda").to(torch.bfloat16)
    dt = torch.float8_e4m3fn if fp8 else torch.bfloat16
    scales = dict(k_scale=0.5, v_scale=0.25) if fp8 else {}
    plan = [[1] * B for _ in range(steps)]
    plan[0] = [2, 1, 1, 0, 3, 1]
    plan[5] = [1, -1, 1, 1, 0, 1]
    plan[6] = [1, 2, 1, 1, 2, 1]

    class Engine:
        def __init__(self):
            self.kc, self.vc = L.new_cache(B * per_row, KVH, ps, D, dt)
            for c in (self.kc, self.vc):
                c.view(torch.uint8).fill_(0x7F)
            self.len, self.new, self.table = i32([0] * B), i32([0] * B), i32([[-1] * per_row] * B)
            self.ring, self.state = i32(list(range(B * per_row))), i32([0, B * per_row])
            self.a = dict(q_start=i32([0] * (B + 1)), seq_len=self.len, positions=i32([0] * T), slots=i32([0] * T), ring_state=self.state, status=i32([0]))
            self.x = torch.zeros(T, cfg.H, dtype=torch.bfloat16, device="cuda")
            self.qkv = torch.zeros(T, (QH + 2 * KVH) * D, dtype=torch.bfloat16, device="cuda")
            self.q, self.o = (torch.zeros(T, QH, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            self.lse, self.h = torch.zeros(T, QH, device="cuda"), torch.zeros_like(self.x)
            self.ws = L.new_attention_workspace(B, T, QH, KVH, D)
            self.buf = L.LayerBuffers(T, cfg.H, cfg.F, cfg.N, cfg.k, 2)

        def step(self):
            L.lynx_kv_assign(self.len, self.new, T, ps, self.table, self.ring, self.state, out=self.a)
            torch.mm(self.x, Wqkv, out=self.qkv)
            q, k, v = (t.unflatten(1, (-1, D)) for t in self.qkv.split([QH * D, KVH * D, KVH * D], 1))
            L.lynx_qk_norm_rope(q, k, v, self.a["positions"], self.a["slots"], freqs, self.kc, self.vc, wq, wk, q_out=self.q, **scales)
            L.lynx_attention(self.q, self.kc, self.vc, self.table, self.a["q_start"], self.len, 3, out=self.o, lse=self.lse, workspace=self.ws, **scales)
            L.lynx_moe_layer(self.o.view(T, cfg.H), d["Wr"], d["bias"], Wgu, Wdp, cfg.F, cfg.k, 2.0, 2, 1, buffers=self.buf)
            L.lynx_residual_add(self.x, self.buf.y, out=self.h)

        def load(self, i):
            self.new.copy_(i32(plan[i]))
            self.x.copy_(xs[i])

    eager, replayed = Engine(), Engine()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        replayed.step()                                        # (no new tokens yet: the warm-up changes nothing)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        replayed.step()
    for i in range(steps):
        eager.load(i)
        replayed.load(i)
        eager.step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert int(eager.a["status"]) == 0
        for e, r in ((eager.q, replayed.q), (eager.o, replayed.o), (eager.lse, replayed.lse), (eager.h, replayed.h), (eager.table, replayed.table),
                     (eager.len, replayed.len), (eager.state, replayed.state)):
            assert torch.equal(e, r), i
        if i in (0, steps - 1):
            n = int(eager.a["q_start"][-1])
            want, _, tol = ref.attention(eager.q.cpu(), eager.kc.float().cpu(), eager.vc.float().cpu(), eager.table.tolist(),
                                         eager.a["q_start"].tolist(), eager.len.tolist(), D ** -0.5, k_scale=scales.get("k_scale", 1.0),
                                         v_scale=scales.get("v_scale", 1.0))
            assert bool(((eager.o[:n].cpu().double() - want[:n]).abs() <= tol[:n]).all())


def test_the_binding_refuses_what_could_be_read_out_of_bounds():
    c = Case([(20, 1), (3, 1)], 4, 2, 64, 16, seed=18)
    q, need = c.q.cuda(), L.attention_workspace_bytes(c.B, c.T, 4, 2, 64)
    args = (q, c.kc, c.vc, i32(c.table), i32(c.q_start), i32(c.seq), 1)
    byte = torch.zeros(1, dtype=torch.uint8, device="cuda")
    for ws in (byte.expand(need), torch.zeros(need - 1, dtype=torch.uint8, device="cuda"), torch.zeros(need, dtype=torch.uint8)):
        with pytest.raises(ValueError, match="workspace"):
            L.lynx_attention(*args, workspace=ws)
    for i, bad in ((3, i32(c.table).t()), (4, i32(c.q_start)[:-1]), (5, i32(c.seq)[:1]), (5, i32(c.seq).long()), (1, c.kc.transpose(2, 3)), (0, q[:, :, :32])):
        with pytest.raises((ValueError, TypeError)):
            L.lynx_attention(*args[:i], bad, *args[i + 1:])
    with pytest.raises(ValueError, match="out"):
        L.lynx_attention(*args, out=torch.empty_like(q)[:-1])
    with pytest.raises(ValueError, match="lse"):
        L.lynx_attention(*args, lse=torch.empty(c.T * 4 - 1, device="cuda"))
    with pytest.raises(L.LynxError, match="out must not be q"):
        L.lynx_attention(*args, out=q)
    with pytest.raises(ValueError, match="prefix_table"):
        L.lynx_attention_prefix(*args, i32([0]), 17)
