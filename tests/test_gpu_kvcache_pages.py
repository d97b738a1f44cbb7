"""lynx_kv_assign says when pages are lost: pages of ended requests that the ring has no place for."""
import os
import re

import pytest
import torch

import paper_2411_08982_amd as L
from paper_2411_08982_amd import attention as A

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "lynx", "attention.h")


def test_the_header_and_the_binding_have_the_same_bit():
    assert int(re.search(r"#define LYNX_KV_LOST_PAGES (\d+)", open(HEADER).read()).group(1)) == A.KV_LOST_PAGES


def run(ctx, new, T, table, ring, state, shared=0):
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    t, r = i32(table), i32(ring)
    o = L.lynx_kv_assign(i32(ctx), i32(new), T, 16, t, r, i32(state), shared)
    return dict({n: o[n].tolist() for n in ("seq_len", "ring_state", "status")}, table=t.tolist(), ring=r.tolist())


@pytest.mark.gpu
def test_pages_that_the_ring_has_no_place_for():
    # four pages, three of them free by the count, and a request that ends with two: one has a place behind the free ones
    got = run([32], [-1], 1, [[0, 1]], [7, 2, 3, 9], [1, 3])
    assert got == dict(seq_len=[0], ring_state=[1, 4], status=[A.KV_LOST_PAGES], table=[[0, 1]], ring=[0, 2, 3, 9])
    # a count beyond the ring: no place at all
    got = run([16], [-1], 1, [[0]], [1, 2], [0, 2 ** 31 - 1])
    assert got == dict(seq_len=[0], ring_state=[0, 2], status=[A.KV_LOST_PAGES], table=[[0]], ring=[1, 2])
    # the same page in two rows
    got = run([16, 16], [-1, -1], 1, [[1], [1]], [0, 5], [0, 1])
    assert got["status"] == [A.KV_LOST_PAGES] and got["ring"] == [0, 1] and got["ring_state"] == [0, 2]
    # a row that holds more pages than there are
    got = run([80], [-1], 1, [[0, 1, 0, 1, 0]], [9, 9], [0, 0])
    assert got["status"] == [A.KV_LOST_PAGES] and got["ring"] == [0, 1] and got["ring_state"] == [0, 2]
    # beside another reason: no free page for the second request, whose length stays
    got = run([32, 16], [-1, 1], 4, [[0, 1], [2, -1]], [3, 3], [0, 0], 0)
    assert got["status"] == [A.KV_NO_PAGES] and got["ring_state"] == [0, 2] and got["seq_len"] == [0, 16]
    got = run([48, 16], [-1, 1], 4, [[0, 1, 0], [1, -1, -1]], [3, 3], [0, 0], 0)
    assert got["status"] == [A.KV_NO_PAGES + A.KV_LOST_PAGES]


@pytest.mark.gpu
def test_pages_that_just_fit_are_not_lost():
    # every page comes back, the ring's places go round
    got = run([32, 32], [-1, -2], 1, [[0, 1], [2, 3]], [9, 9, 9, 9], [3, 0])
    assert got == dict(seq_len=[0, 0], ring_state=[3, 4], status=[0], table=[[0, 1], [2, 3]], ring=[1, 2, 3, 0])
    # shared pages are nobody's to give back
    got = run([48, 40], [-1, -1], 1, [[5, 0, 1], [5, 2, 3]], [4, 9, 9, 9, 9, 9], [0, 1], shared=1)
    assert got["status"] == [0] and got["ring_state"] == [0, 5] and got["ring"] == [4, 0, 1, 2, 3, 9]
    # unless the call is told of fewer than there are: each row brings the shared page back
    got = run([48, 40], [-1, -1], 1, [[5, 0, 1], [5, 2, 3]], [4, 9, 9, 9, 9, 9], [0, 1], shared=0)
    assert got["status"] == [A.KV_LOST_PAGES] and got["ring_state"] == [0, 6]
