"""lynx_qk_norm_rope with slots that follow one another, as a prompt's do: values go into the cache in runs of 16 bytes (8 tokens of a bf16
cache, 16 of an 8-bit one) where such a run is whole, and token by token elsewhere.  Without norm and rotation keys and values are rounded
once or not at all, so the caches have to equal the host's in every byte, those that no token occupies among them."""
import numpy as np
import pytest
import torch

import paper_2411_08982_amd as L

pytestmark = pytest.mark.gpu

BITS = {torch.bfloat16: torch.int16, torch.float8_e4m3fn: torch.uint8}


def slots_of(prompts, ps, rng, spare=3):
    """Slots of prompts of (first place, tokens), one behind the other, each from its place in a page of its own on; pages are scattered."""
    need = [-(-(first % ps + n) // ps) for first, n in prompts]
    pages = sum(need) + spare
    ids = rng.permutation(pages)
    out, at = [], 0
    for (first, n), k in zip(prompts, need):
        j = first % ps + np.arange(n)
        out.append(ids[at + j // ps] * ps + j % ps)
        at += k
    return np.concatenate(out) if out else np.zeros(0, np.int64), pages


def check(slots, pages, KVH, D, ps, fp8, seed=0):
    T, dt = len(slots), torch.float8_e4m3fn if fp8 else torch.bfloat16
    ks, vs = (0.37, 1.9) if fp8 else (1.0, 1.0)
    g = torch.Generator().manual_seed(seed)
    k, v = (torch.randn(T, KVH, D, generator=g).mul(50).to(torch.bfloat16) for _ in range(2))
    caches = L.new_cache(pages, KVH, ps, D, dt)
    for c in caches:
        c.view(BITS[dt]).fill_(0x55)
    want = [c.view(BITS[dt]).cpu() for c in caches]
    # the kernel's own steps: one division in 32 bits, saturation, one rounding
    codes = [(x.float() / torch.tensor(s, dtype=torch.float32)).clamp(-448, 448).to(dt) if fp8 else x for x, s in ((k, ks), (v, vs))]
    slots = torch.as_tensor(slots)
    keep = (slots >= 0) & (slots < pages * ps)
    at = slots[keep]
    want[0][at // ps, :, at % ps] = codes[0].view(BITS[dt])[keep]
    want[1][at // ps, :, :, at % ps] = codes[1].view(BITS[dt])[keep]
    q = torch.zeros(T, KVH, D, dtype=torch.bfloat16, device="cuda")
    L.lynx_qk_norm_rope(q, k.cuda(), v.cuda(), torch.zeros(T, dtype=torch.int32, device="cuda"), slots.int().cuda(), None, *caches,
                        k_scale=ks, v_scale=vs)
    for c, w in zip(caches, want):
        assert torch.equal(c.view(BITS[dt]).cpu(), w)


FORMS = [(64, False), (128, False), (64, True), (128, True)]


@pytest.mark.parametrize("D,fp8", FORMS)
@pytest.mark.parametrize("first", range(16))
def test_prompts_that_begin_anywhere_in_a_run(first, D, fp8):
    rng = np.random.default_rng([first, D])
    # two prompts, the second's runs at any residue of the 16 tokens that a workgroup has
    slots, pages = slots_of([(first, 41), (first + 5, 70)], 48, rng)
    check(slots, pages, 2, D, 48, fp8, first)


@pytest.mark.parametrize("D,fp8", FORMS)
@pytest.mark.parametrize("T", [1, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 129, 1023, 1024, 1025, 1055, 1057, 1500, 2049])
def test_prompts_of_any_length(T, D, fp8):
    for ps in (16, 64):
        slots, pages = slots_of([(0, T)], ps, np.random.default_rng(T))
        check(slots, pages, 3, D, ps, fp8, T)


@pytest.mark.parametrize("D,fp8", FORMS)
@pytest.mark.parametrize("first", [0, 3, 8, 13])
def test_more_than_1024_tokens_from_anywhere_in_a_run(first, D, fp8):
    rng = np.random.default_rng([first, D, 1])
    slots, pages = slots_of([(first, 611), (first + 3, 500), (first + 1, 90)], 128, rng)
    check(slots, pages, 2, D, 128, fp8, first)


@pytest.mark.parametrize("D,fp8", FORMS)
@pytest.mark.parametrize("T", [90, 1201])
def test_runs_with_holes_and_single_tokens_beside_them(T, D, fp8):
    """Prompts of all lengths, single tokens between them, tokens that are not written in the middle of runs, slots at the end of the
    cache and outside it, and runs that go backwards or skip a place."""
    for seed in range(4):
        rng = np.random.default_rng([T, seed, D])
        prompts, left = [], T
        while left > 0:
            n = min(left, int(rng.choice([1, 1, 2, 9, 16, 17, 40, 77])))
            prompts.append((int(rng.integers(0, 64)), n))
            left -= n
        ps = int(rng.choice([16, 32, 48, 64]))
        slots, pages = slots_of(prompts, ps, rng)
        for i in rng.integers(0, T, 4):
            slots[i] = rng.choice([-1, -(2 ** 31), pages * ps, 2 ** 31 - 1])
        i = int(rng.integers(0, T - 24))
        slots[i:i + 20] = slots[i:i + 20][::-1].copy()
        slots[i + 21], slots[i + 22] = slots[i + 22], slots[i + 21]
        check(slots, pages, 2, D, ps, fp8, seed)


@pytest.mark.parametrize("D,fp8", FORMS)
def test_a_prompt_that_ends_with_the_cache(D, fp8):
    # the last page's last tokens, and tokens that would follow them behind the cache
    ps, pages = 32, 5
    check(np.arange(pages * ps - 21, pages * ps + 11), pages, 2, D, ps, fp8)
    check(np.arange(-9, 40), pages, 2, D, ps, fp8)
