"""Row ranges of the attention calls other than 0 .. T in order: requests that begin behind row 0, padding that holds NaN, ranges that go
back.  Rows of requests are compared with the host oracle in 64 bits, all others have to stay as they were."""
import math

import pytest
import torch

import paper_2411_08982_amd as L
from test_gpu_attention import Case, i32

pytestmark = pytest.mark.gpu


def shifted(c, front, behind=0):
    """The case with `front` more rows in front of its first request's and `behind` behind its padding; all padding is NaN."""
    nan = lambda n: torch.full((n, c.QH, c.D), math.nan, dtype=torch.bfloat16)
    c.q = torch.cat([nan(front), c.q[:c.rows], nan(c.T - c.rows + behind)])
    c.q_start = [s + front for s in c.q_start]
    c.T += front + behind
    return c


def check_ranges(c, rows, want=None, **kw):
    """rows: those that have to equal the oracle; nothing else is written, where `kw` leaves nothing unspecified."""
    out = torch.full((c.T, c.QH, c.D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((c.T, c.QH), 7.0, dtype=torch.float32, device="cuda")
    c.run(out=out, lse=lse, **kw)
    want, want_lse, tol = c.expect(c.D ** -0.5) if want is None else want
    o, l = out.cpu().double(), lse.cpu().double()
    rows = torch.as_tensor(rows, dtype=torch.long)
    assert bool(((o - want).abs() <= tol)[rows].all())
    none = torch.isinf(want_lse[rows])
    assert torch.equal(none, torch.isinf(l[rows]))
    # (scores 144 roundings of 2^-24 off at most, and the logarithm a few more, as in Case.check)
    assert bool(((l[rows] - want_lse[rows])[~none].abs() <= 2e-5 * (1 + want_lse[rows][~none].abs())).all())
    return o, l


def untouched(c, o, l, rows):
    rows = torch.as_tensor(rows, dtype=torch.long)
    assert bool((o[rows] == 7).all()) and bool((l[rows] == 7).all())


@pytest.mark.parametrize("front", [1, 16, 100])
@pytest.mark.parametrize("lens,QH,KVH,D,ps,fp8,prefix", [
    ([(383, 1)], 1, 1, 128, 16, False, 64),                               # one row, its tile cut into two parts
    ([(384 + i * 90, 1 + i % 2) for i in range(6)], 8, 2, 64, 16, False, 300),    # short tiles, some of them cut
    ([(2000, 1), (64, 1), (10, 2)], 4, 2, 128, 64, True, 64),           # one request that is cut, one that is not, one inside the prefix
    ([(200, 60), (200, 1), (150, 9)], 8, 2, 64, 32, False, 130),         # tiles of 128 rows as well
    ([(300, 40)], 5, 1, 128, 16, True, 192),
    ([(70, 1), (0, 0), (500, 3)], 4, 4, 64, 48, False, 0),               # no prefix: lynx_attention
    ([(100, 50), (40, 1)], 8, 2, 128, 16, True, 0),
])
def test_requests_that_begin_behind_row_0(front, lens, QH, KVH, D, ps, fp8, prefix):
    c = shifted(Case(lens, QH, KVH, D, ps, fp8, seed=40, prefix=prefix), front, 5)
    end = front + c.rows
    o, l = check_ranges(c, range(front, end))
    untouched(c, o, l, list(range(front)) + list(range(end, c.T)))


@pytest.mark.parametrize("prefix", [0, 200])
def test_last_row_start_behind_the_rows(prefix):
    c = Case([(230, 1), (220, 2), (203, 3)], 4, 2, 64, 16, seed=41, prefix=prefix, pad=0)
    want = c.expect(c.D ** -0.5)
    c.q_start = [0, 1, 3, 9]                              # clamped to T = 6
    check_ranges(c, range(6), want)


@pytest.mark.parametrize("prefix", [0, 200])
def test_row_starts_that_go_back(prefix):
    c = Case([(230, 2), (220, 1), (203, 3)], 4, 2, 64, 16, seed=42, prefix=prefix, pad=3)
    c.q_start, c.seq = [0, 2, 2, 2], [232, 220, 206]
    first = c.expect(c.D ** -0.5)
    c.q_start = [1, 1, 1, 4]
    last = c.expect(c.D ** -0.5)
    want = [torch.cat([a[:1], b[1:]]) for a, b in zip(first, last)]
    c.q_start = [-4, 2, 1, 4]                             # rows 0, 1 and rows 1, 2, 3: row 1 is in both, rows from 4 on in none
    o, l = check_ranges(c, [0], want)
    untouched(c, o, l, range(4, c.T))


def test_row_ranges_that_overlap_beyond_all_bounds_behind_a_prefix():
    # as without a prefix: 2^34 blocks, more than 32 bits count, so no request's own part is read; rows in no request stay as they were
    B, T, pages = 1024, 4096, 1024
    q_start = i32([8, T - 8] * (B // 2) + [8])
    cache = L.new_cache(2, 1, 1024, 64)
    for t in cache:
        t.zero_()
    q = torch.zeros(T, 8, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 7.0)
    L.lynx_attention_prefix(q, *cache, torch.zeros(B, pages, dtype=torch.int32, device="cuda"), q_start, i32([pages * 1024] * B), 1,
                            i32([0]), 512, out=out)
    assert bool((out[:8] == 7).all()) and bool((out[T - 8:] == 7).all())
