"""Scores of any magnitude that fits 32 bits: queries and keys of one channel that are powers of two and small whole numbers, so that every
score is exact and the softmax is the mean over the tokens of the largest one."""
import math

import pytest
import torch

import paper_2411_08982_amd as L
from test_gpu_attention import i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("power", [10, 21, 24, 30, 31, 32, 33, 40, 80, 120])
@pytest.mark.parametrize("n", [1, 4, 70])            # tiles of 16 rows, of 16 and 128, of 128
@pytest.mark.parametrize("D,fp8,prefix", [(128, False, 0), (64, True, 0), (64, False, 0), (128, True, 0), (128, False, 320), (64, True, 320)])
def test_the_largest_score_wins(D, fp8, prefix, n, power):
    B, QH, KVH, ps, m = 12, 8, 2, 16, 400
    G, scale, dt = QH // KVH, 0.5, torch.float8_e4m3fn if fp8 else torch.bfloat16
    g = torch.Generator().manual_seed(power * 100 + n)
    k = torch.zeros(m, KVH, D)
    k[:, :, 5] = torch.randint(-16, 17, (m, KVH), generator=g).float()
    k[m // 2, :, 5] = 0
    v = torch.randn(m, KVH, D, generator=g).to(dt).float()
    pages = m // ps
    table = torch.randperm(pages, generator=g)
    kc, vc = torch.zeros(pages, KVH, ps, D), torch.zeros(pages, KVH, D, ps)
    j = torch.arange(m)
    kc[table[j // ps], :, j % ps], vc[table[j // ps], :, :, j % ps] = k, v
    seq = [m - 3 * b for b in range(B)]
    T = B * n
    q = torch.zeros(T, QH, D)
    q[:, :, 5] = torch.where(torch.rand(T, QH, generator=g) < 0.5, -1.0, 1.0) * 2.0 ** (power - torch.randint(0, 3, (T, QH), generator=g))
    args = (q.to(torch.bfloat16).cuda(), kc.to(dt).cuda(), vc.to(dt).cuda(), i32(table.expand(B, -1).tolist()), i32(list(range(0, T + 1, n))), i32(seq), n)
    lse = torch.empty(T, QH, device="cuda")
    if prefix:
        out = L.lynx_attention_prefix(*args, i32(table[:prefix // ps].tolist()), prefix, scale=scale, lse=lse)
    else:
        out = L.lynx_attention(*args, scale=scale, lse=lse)
    out, lse = out.cpu().double().view(B, n, QH, D), lse.cpu().double().view(B, n, QH)
    z = scale * torch.einsum("thc,mhc->thm", q.double(), k.double().repeat_interleave(G, 1)).view(B, n, QH, m)
    pos = torch.tensor(seq)[:, None] - n + torch.arange(n)
    z = z.masked_fill(j > pos[:, :, None, None], -math.inf)
    w = torch.softmax(z, -1).transpose(1, 2).reshape(B, KVH, G * n, m)
    vv = v.double().permute(1, 0, 2)
    back = lambda x: x.reshape(B, QH, n, D).transpose(1, 2)
    want, size = back(w @ vv), back(w @ vv.abs())
    # weights and result rounded to bf16
    assert bool(((out - want).abs() <= 1.02 * 2.0 ** -8 * (size + want.abs())).all())
    top = z.logsumexp(-1)
    assert bool(((lse - top).abs() <= 2e-5 * (1 + top.abs())).all())


@pytest.mark.parametrize("n", [1, 70])
def test_the_least_scale_that_is_taken(n):
    # weights are all the same: the mean of what a row sees, and the logarithm of how many those are
    D, ps, m, QH = 64, 16, 300, 4
    g = torch.Generator().manual_seed(n)
    pages = -(-m // ps)
    k, v = torch.randn(pages, 1, ps, D, generator=g).to(torch.bfloat16), torch.randn(pages, 1, D, ps, generator=g).to(torch.bfloat16)
    q = torch.randn(n, QH, D, generator=g).to(torch.bfloat16)
    lse = torch.empty(n, QH, device="cuda")
    out = L.lynx_attention(q.cuda(), k.cuda(), v.cuda(), i32([list(range(pages))]), i32([0, n]), i32([m]), n, scale=1e-38, lse=lse)
    vv = v[:, 0].double().transpose(1, 2).reshape(-1, D)[:m]
    seen = torch.arange(m - n + 1, m + 1)
    want, size = (torch.cumsum(x, 0)[m - n:] / seen[:, None] for x in (vv, vv.abs()))
    # weights (here exact) and result rounded to bf16
    assert bool(((out.cpu().double() - want[:, None]).abs() <= 1.02 * 2.0 ** -8 * (size + want.abs())[:, None]).all())
    assert bool(((lse.cpu().double() - seen.double().log()[:, None]).abs() <= 2e-5 * (1 + seen.double().log()[:, None])).all())
