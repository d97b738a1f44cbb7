"""Long prompts on the GPU against dense attention in 64 bits on the host: tiles of 128 rows over many blocks, cut and whole, with windows
whose border runs through every block of a tile, first tokens far in front of it, and single tokens in the same batch."""
import math

import pytest
import torch

import paper_2411_08982_amd as L
from test_gpu_attention import i32

pytestmark = pytest.mark.gpu


def dense(q, k, v, pos, scale, window, sinks):
    """q [n, G, D], k, v [m, D] float64 at positions pos and 0 .. m-1 -> out, lse and the bound on out's error, as attention_ref has it."""
    n, G, D = q.shape
    qq = q.reshape(n * G, D)
    z = (qq @ k.T) * scale
    i, j = pos.repeat_interleave(G)[:, None], torch.arange(k.shape[0])[None, :]
    seen = (j <= i) & ((j > i - window) | (j < sinks)) if window else j <= i
    z = z.masked_fill(~seen, -math.inf)
    w = torch.softmax(z, 1)
    out, size = w @ v, w @ v.abs()
    # weights and result rounded to bf16, 2^-8 of the value each; scores are fp32 sums over D terms with 16 more fp32 roundings
    shake = (D + 16) * 2.0 ** -24 * scale * (qq.abs() @ k.abs().T).masked_fill(~seen, 0).amax(1, keepdim=True)
    tol = 2.0 ** -8 * (size + out.abs()) * 1.02 + 2 * shake * size
    return out.view(n, G, D), z.logsumexp(1).view(n, G), tol.view(n, G, D)


@pytest.mark.parametrize("lens,QH,KVH,D,ps,fp8,window,sinks", [
    ([(0, 2100)], 8, 2, 128, 64, False, 0, 0),                     # one prompt: its last tiles are cut
    ([(0, 1500)], 4, 2, 64, 16, True, 0, 0),
    ([(5000, 700), (3, 1), (0, 1024), (900, 1)], 4, 1, 128, 32, False, 0, 0),
    ([(3001, 513), (700, 2)], 10, 2, 128, 48, True, 0, 0),
    ([(0, 1000)], 4, 2, 128, 16, False, 128, 0),                     # parts of a few blocks each
    ([(1111, 1300), (2000, 1)], 4, 2, 64, 64, False, 777, 70),
    ([(4000, 600), (100, 40)], 8, 2, 128, 128, True, 1000, 4),
    ([(i * 37, 129 + i) for i in range(12)], 16, 4, 64, 16, False, 300, 4),
])
def test_prompts_equal_dense_attention(lens, QH, KVH, D, ps, fp8, window, sinks):
    g = torch.Generator().manual_seed(len(lens) + D + window)
    G, dt = QH // KVH, torch.float8_e4m3fn if fp8 else torch.bfloat16
    ks, vs = (0.5, 1.7) if fp8 else (1.0, 1.0)
    seq = [c + n for c, n in lens]
    held = [-(-s // ps) for s in seq]
    pages = sum(held) + 2
    ids = torch.randperm(pages, generator=g)
    table, at = torch.full((len(lens), max(held) + 1), -1), 0
    kc, vc = torch.full((pages, KVH, ps, D), math.nan), torch.full((pages, KVH, D, ps), math.nan)      # places of no token hold NaN
    keys, values = [], []
    for b, s in enumerate(seq):
        table[b, :held[b]] = ids[at:at + held[b]]
        at += held[b]
        k, v = (torch.randn(s, KVH, D, generator=g).to(dt).float() for _ in range(2))
        j = torch.arange(s)
        kc[table[b, j // ps], :, j % ps], vc[table[b, j // ps], :, :, j % ps] = k, v
        keys.append(k.double() * ks)
        values.append(v.double() * vs)
    starts = [0]
    for _, n in lens:
        starts.append(starts[-1] + n)
    T = starts[-1] + 2
    q = (torch.randn(T, QH, D, generator=g) * 2).to(torch.bfloat16)
    out = torch.full((T, QH, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, QH), 7.0, device="cuda")
    L.lynx_attention(q.cuda(), kc.to(dt).cuda(), vc.to(dt).cuda(), i32(table.tolist()), i32(starts), i32(seq), max(n for _, n in lens),
                     window=window, sinks=sinks, k_scale=ks, v_scale=vs, out=out, lse=lse)
    o, l = out.cpu().double(), lse.cpu().double()
    assert bool((o[-2:] == 7).all()) and bool((l[-2:] == 7).all())
    for b, (c, n) in enumerate(lens):
        rows = slice(starts[b], starts[b + 1])
        for h in range(KVH):
            heads = slice(h * G, (h + 1) * G)
            want, want_lse, tol = dense(q[rows, heads].double(), keys[b][:, h], values[b][:, h], c + torch.arange(n), D ** -0.5, window, sinks)
            assert bool(((o[rows, heads] - want).abs() <= tol).all()), (b, h)
            # (scores 144 roundings of 2^-24 off at most, the logarithm a few more)
            assert bool(((l[rows, heads] - want_lse).abs() <= 2e-5 * (1 + want_lse.abs())).all()), (b, h)
