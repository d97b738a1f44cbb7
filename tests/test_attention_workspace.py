"""The workspace of the attention calls: how large it may get, and that one for the largest step serves every smaller one, also where the
smaller one reads a shared prefix apart and the larger one does not."""
import random

import pytest
import torch

import paper_2411_08982_amd as L
from test_gpu_attention import Case, i32

MIB = 1 << 20


def test_the_size_never_falls():
    rng = random.Random(5)
    heads = [(8, 8, 64), (32, 4, 128), (64, 8, 128), (64, 1, 64), (256, 1, 64), (5, 5, 128), (1024, 1024, 64), (600, 300, 128)]
    for _ in range(3000):
        QH, KVH, D = rng.choice(heads)
        size = lambda top: int(2 ** rng.uniform(0, top))
        a = [size(10), size(16), rng.choice([0, size(20)])]
        b = [max(x, rng.choice([x, size(top)])) for x, top in zip(a, (10, 16, 20))]
        small, large = (L.attention_workspace_bytes(B, T, QH, KVH, D, P) for B, T, P in (a, b))
        assert 0 < small <= large, (a, b, QH, KVH, D)


def test_a_short_prefix_or_long_prompts_take_no_gigabytes():
    plain = L.attention_workspace_bytes(1024, 65536, 64, 8, 128)
    assert plain < 80 * MIB
    # the largest step behind 64 tokens: 16 rows of each request are the most for which the prefix is read apart
    assert L.attention_workspace_bytes(1024, 65536, 64, 8, 128, 64) < plain + 140 * MIB
    # a few prompts behind a long one: 128 rows of each request
    assert L.attention_workspace_bytes(8, 65536, 64, 8, 128, 100000) < plain + 44 * MIB


@pytest.mark.gpu
@pytest.mark.parametrize("QH,KVH,D,ps,fp8", [(8, 2, 128, 16, False), (5, 1, 64, 32, True)])
def test_both_sides_of_the_rule(QH, KVH, D, ps, fp8):
    """Requests of fewer and of more rows than a prefix is read apart for: each as the oracle has it, and the latter as lynx_attention has it."""
    G = QH // KVH
    for prefix, new, apart in ((600, 127 // G, True), (600, 128 // G + 1, False), (64, 16 // G, True), (64, 16 // G + 1, False), (130, 32 // G, True),
                               (130, 33 // G + 1, False)):
        c = Case([(prefix + 20, new), (prefix, new), (prefix + 70, new)], QH, KVH, D, ps, fp8, seed=50, prefix=prefix, pad=0)
        out, lse = c.check()
        plain, plain_lse = torch.empty_like(out), torch.empty_like(lse)
        L.lynx_attention(c.q.cuda(), c.kc, c.vc, i32(c.table), i32(c.q_start), i32(c.seq), c.max_new, k_scale=c.ks, v_scale=c.vs, out=plain, lse=plain_lse)
        if apart:        # (sums in another order)
            assert not torch.equal(lse, plain_lse)
        else:
            assert torch.equal(out, plain) and torch.equal(lse, plain_lse)


@pytest.mark.gpu
@pytest.mark.parametrize("QH,KVH,D,ps,fp8", [(8, 2, 128, 16, False), (4, 4, 64, 48, True)])
def test_large_and_small_rows_behind_a_prefix_that_is_read_apart(QH, KVH, D, ps, fp8):
    # tiles of 128 rows for what requests have of their own, some cut, beside single tokens; one request inside the prefix
    lens = [(700, 60), (2500, 40), (640, 1), (650, 1), (0, 3), (900, 2), (641, 1), (699, 1), (640, 0), (1000, 1)]
    Case(lens, QH, KVH, D, ps, fp8, seed=51, prefix=640).check()


@pytest.mark.gpu
def test_a_workspace_for_the_largest_step_serves_smaller_ones():
    QH, KVH, D, ps, prefix = 8, 2, 64, 16, 640
    ws = L.new_attention_workspace(8, 400, QH, KVH, D, prefix)
    guard = torch.full((ws.numel() + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    for lens in ([(700, 390), (650, 1)], [(640, 1)] * 7, [(640, 20), (641, 3)], [(900, 90), (641, 1), (0, 0)], [(640 + i, 30) for i in range(8)]):
        c = Case(lens, QH, KVH, D, ps, seed=52, prefix=prefix)
        assert L.attention_workspace_bytes(c.B, c.T, QH, KVH, D, prefix) <= ws.numel()
        want = c.run()
        guard.fill_(0xA5)
        got = c.run(workspace=guard[:ws.numel()])
        assert torch.equal(got[:c.rows], want[:c.rows]) and bool((guard[ws.numel():] == 0xA5).all())
