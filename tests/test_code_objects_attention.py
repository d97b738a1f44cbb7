"""The build's check of the attention kernel's waits: it passes on the library that was built and refuses what it is there for."""
import os

import pytest

from paper_2411_08982_amd import check_code
from paper_2411_08982_amd.build import LIB

LOAD, READ, OTHER = "global_load_lds_dwordx4 v[6:7], off nt", "ds_read_b128 v[8:11], v4", "scratch_load_dword v1, off, off"
NAME = "_ZN4lynx11attn_kernelILi128ELb0ELb0EEEvNS_10AttnParamsE"


def wait(n):
    return f"s_waitcnt vmcnt({n})"


def listing(body, symbol=NAME):
    """body, eight bytes an instruction from 0x9000; "-> n": the target of a branch is the n-th instruction."""
    out = [f"0000000000009000 <{symbol}>:"]
    for i, text in enumerate(body):
        op, _, target = text.partition(" -> ")
        mark = f" <{symbol}+0x{8 * int(target):x}>" if target else ""
        out.append(f"\t{op}{' 0' if target else ''}    // {0x9000 + 8 * i:012X}: DDF68000 007F0006{mark}")
    return "\n".join(out) + "\n"


def kernel(turn=None, last=None, first=None, before=(), skip=True):
    """A tile of blocks of four units of two loads: the loads ahead, a turn of the loop, the last block."""
    first = [LOAD] * 8 if first is None else first
    turn = [wait(6), READ, READ, LOAD, LOAD] * 4 if turn is None else turn
    last = sum(([wait(n), READ, READ] for n in (6, 4, 2, 0)), []) if last is None else last
    body = list(before) + first
    top = len(body) + 1
    body += [f"s_cbranch_scc1 -> {top + len(turn) + 1}" if skip else "s_nop 0"] + turn + [f"s_cbranch_scc1 -> {top}"] + last
    return listing(body + ["s_waitcnt lgkmcnt(0)", "ds_read_b32 v1, v2", "s_endpgm"])


@pytest.mark.skipif(not os.path.exists(LIB), reason="the library is not built")
def test_every_unit_of_the_built_kernels_is_waited_for():
    # a turn and a last block of each of 8 kernels: 8 units with bf16 and D = 128, 4 otherwise
    texts = [text for _, text in check_code.code_object_texts(LIB)]
    assert sum(map(check_code.check_units, texts)) == 2 * (2 * 8 + 6 * 4)
    # the tiles' barriers behind direct loads: a first one and two turns of each of the two bf16 kernels that have tiles
    tiles = [text for text in texts if "attn_kernel" in text]
    assert len(tiles) == 1 and check_code.check_waits(tiles[0]) >= 2 * 3


def test_a_kernel_as_it_should_be():
    assert check_code.check_units(kernel()) == 8
    assert check_code.check_units(kernel(before=["global_load_dword v1, v[2:3], off", wait(0), READ])) == 8
    # other memory operations behind a unit make the wait longer than it has to be
    assert check_code.check_units(kernel(turn=[wait(6), READ, READ, LOAD, OTHER, LOAD] * 4, last=sum(([wait(n), READ] for n in (6, 4, 2, 0)), []))) == 8
    assert check_code.check_units(kernel().replace("attn_kernel", "other_kernel")) == 0


@pytest.mark.parametrize("change", [
    dict(first=[LOAD] * 7),                                                     # one load less than four units
    dict(first=[LOAD] * 8 + [READ]),                                            # read before anything is waited for
    dict(turn=[wait(7), READ, READ, LOAD, LOAD] * 4),                           # a wait that is too short
    dict(turn=[wait(6), READ, READ, LOAD] + [wait(6), READ, READ, LOAD, LOAD] * 3),    # a load that has gone, or two that became one
    dict(turn=[wait(6), READ, READ, LOAD, LOAD] * 3 + [READ, READ, LOAD, LOAD]),        # a wait that has gone
    dict(turn=[wait(6), READ, READ, LOAD, LOAD] * 3 + [wait(6), READ, READ]),           # loads that have gone at a turn's end
    dict(last=sum(([wait(n), READ, READ] for n in (6, 4, 3, 0)), [])),          # the last block: a wait that is too short,
    dict(last=sum(([wait(n), READ, READ] for n in (6, 4, 2)), [])),             # and a unit that is never read
    dict(last=sum(([wait(n), READ, READ] for n in (6, 4, 2, 1)), [])),
    dict(first=[LOAD, OTHER] + [LOAD] * 7, turn=[wait(7), READ, READ, LOAD, LOAD] * 4),   # what comes in front of a unit's last load does not count
], ids=range(10))
def test_units_that_may_not_have_landed_are_refused(change):
    with pytest.raises(RuntimeError, match="attn_kernel"):
        check_code.check_units(kernel(**change))


def test_a_tile_s_barrier_without_its_wait_is_refused():
    body = ["buffer_load_dwordx4 v67, s[4:7], 0 offen lds", "s_waitcnt vmcnt(1)", "s_barrier", "s_endpgm"]
    with pytest.raises(RuntimeError, match="nothing waits"):
        check_code.check_waits(listing(body))
    body[1] = "s_waitcnt vmcnt(0) lgkmcnt(0)"
    assert check_code.check_waits(listing(body)) == 1
