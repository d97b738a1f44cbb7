"""What the expert kernel takes for granted of the compiler, checked in the AMD code objects of the library just built.

Placement: the kernel's two LDS buffers for token rows are the destination of direct-to-LDS loads, whose LDS address is 16
bits wide, so they have to lie in the first 64 KiB.  The language does not say where a __shared__ array goes.  Both are
aligned to kStageAlign and the kernel's other arrays are smaller than that together: whatever lies ahead of or between
the buffers moves the end of the segment by a whole kStageAlign, and the segment's size shows it.

The attention kernel's four LDS buffers for blocks of the cache are filled by such loads too: aligned to ATTENTION_ALIGN, which is more
than the kernel's other arrays take together.  Its tiles wait at barriers, as below.  Its waves of few rows have four units of a block on their way
and read each behind a wait that leaves as many loads outstanding as come behind that unit: check_units counts them in the machine code.

Waits: a wave reports its pieces of a chunk of token rows at a barrier, before which they must have landed.  The kernel waits
until at most as many loads are outstanding as it has issued behind them, a number that follows from its source as long as
the compiler neither drops nor merges loads.  They are counted again in the machine code, ahead of every barrier behind a
direct-to-LDS load, in the order of the listing (the kernel's loops around them are laid out straight).

Products: the wide kernel's matrix instructions are written out, so the compiler does not keep the wait states that they need: two
between a VALU instruction that writes an operand of theirs and its use, and up to 19 (for the longest of them) between a product and
any other instruction on its sums.  Their operands come from loads and their sums stay in place; that no instruction comes too
close is checked in the machine code, in the order of the listing and across every branch.
"""
from __future__ import annotations

import os
import re
import subprocess
import tempfile

LLVM = os.environ.get("ROCM_LLVM_BIN", "/opt/rocm/llvm/bin")
KERNEL = "ffn_kernel"
WIDE = "ffn_wide_kernel"
STAGE_END = 65536     # 2 * kStageBuffer
STAGE_ALIGN = 4096    # kStageAlign
ATTENTION = "attn_kernel"
ATTENTION_ALIGN = 16384    # kLdsAlign


def _run(tool, *args, cwd=None):
    return subprocess.run([os.path.join(LLVM, tool), *args], cwd=cwd, capture_output=True, text=True, check=True).stdout


def code_object_texts(lib_path: str):
    """(metadata notes, disassembly) of every gfx950 code object in the library that holds one of the kernels."""
    with tempfile.TemporaryDirectory() as d:
        os.symlink(os.path.abspath(lib_path), os.path.join(d, "lib.so"))   # (the extracted objects land beside it)
        _run("llvm-objdump", "--offloading", "lib.so", cwd=d)
        for name in sorted(os.listdir(d)):
            if not name.endswith("gfx950"):
                continue
            notes = _run("llvm-readelf", "--notes", name, cwd=d)
            if KERNEL in notes or ATTENTION in notes:
                yield notes, _run("llvm-objdump", "-d", name, cwd=d)


def check_placement(notes: str) -> int:
    """Raises if an LDS buffer of the kernel can reach past STAGE_END; the number of kernels looked at."""
    kernels = re.findall(r"\.group_segment_fixed_size:\s*(\d+)(?:(?!\.group_segment_fixed_size).)*?\.name:\s*(\S*" + KERNEL + r"\S*)",
                         notes, re.S)
    for size, name in kernels:
        if not STAGE_END <= int(size) < STAGE_END + STAGE_ALIGN:
            raise RuntimeError(f"{name}: {size} bytes of LDS: the buffers for token rows do not lie in the first {STAGE_END}")
    return len(kernels)


def check_attention_placement(notes: str) -> int:
    """Raises if a buffer of the attention kernel can reach past STAGE_END; the number of kernels looked at."""
    kernels = re.findall(r"\.group_segment_fixed_size:\s*(\d+)(?:(?!\.group_segment_fixed_size).)*?\.name:\s*(\S*" + ATTENTION + r"\S*)",
                         notes, re.S)
    for size, name in kernels:
        if int(size) >= STAGE_END + ATTENTION_ALIGN:
            raise RuntimeError(f"{name}: {size} bytes of LDS: the buffers for blocks of the cache do not lie in the first {STAGE_END}")
    return len(kernels)


def check_waits(listing: str) -> int:
    """Raises if a barrier of the kernel can be reached before the direct-to-LDS loads ahead of it have landed; the number of
    such barriers."""
    barriers = 0
    name = ""
    behind = None         # memory operations issued behind the last direct-to-LDS load, None = none to wait for
    landed = False
    for line in listing.splitlines():
        head = re.match(r"[0-9a-f]+ <(\S+)>:", line)
        if head:
            name, behind = head.group(1), None
            continue
        words = line.split("//")[0].split()
        if not words or (KERNEL not in name and ATTENTION not in name):
            continue
        op = words[0]
        if op.startswith(("buffer_", "global_", "flat_", "scratch_")):
            if words[-1] == "lds":
                behind, landed = 0, False
            elif behind is not None:
                behind += 1
        elif op == "s_waitcnt" and behind is not None:
            count = re.search(r"vmcnt\((\d+)\)", line)
            landed = landed or (count is not None and int(count.group(1)) <= behind)
        elif op == "s_barrier" and behind is not None:
            if not landed:
                raise RuntimeError(f"{name}: a barrier {behind} loads behind direct-to-LDS loads that nothing waits for")
            barriers += 1
            behind = None
    return barriers


UNITS = 4             # units of a block that a wave has on their way


def check_units(listing: str) -> int:
    """Raises if a wave of the attention kernel can read a unit of a block from LDS before all loads of it have landed; the number of
    units read.

    The loads are followed in the order of the listing: the first run of them is UNITS units, each wait that reads follow is for the
    oldest unit, and behind each unit read come the loads of another or, in a tile's last block, none.  A branch has to find as many
    loads on their way as its target does in that order, which then stands for every path."""
    read = 0
    name, start = "", 0
    unit = 0              # loads of a unit
    out = []              # memory operations on their way, oldest first; True: a load into LDS
    waited = None         # the last wait's count, None: reads have followed it
    at = {}               # address -> loads on their way there, by the listing or by a branch ahead of it

    def fail(what):
        raise RuntimeError(f"{name}: {what}")

    def whole_units():
        if sum(out) % unit:
            fail(f"{sum(out)} loads into LDS on their way, in units of {unit}")
        return sum(out) // unit

    for line in listing.splitlines():
        head = re.match(r"([0-9a-f]+) <(\S+)>:", line)
        if head:
            if out:
                fail("loads into LDS on their way at its end")
            start, name, unit, waited, at = int(head.group(1), 16), head.group(2), 0, None, {}
            continue
        words = line.split("//")[0].split()
        if not words or ATTENTION not in name:
            continue
        op, address = words[0], re.search(r"//\s*([0-9A-Fa-f]+):", line)
        if op.startswith("global_load_lds"):
            out.append(True)
        elif not out:
            continue
        elif op.startswith(("buffer_", "global_", "flat_", "scratch_")):
            out.append(False)
        elif op == "s_waitcnt" and "vmcnt" in line:
            if unit == 0:
                unit = sum(out) // UNITS
                if unit == 0 or whole_units() != UNITS:
                    fail(f"{sum(out)} loads into LDS ahead of the first wait, not {UNITS} units")
            waited = int(re.search(r"vmcnt\((\d+)\)", line).group(1))
        elif op.startswith("ds_read") and waited is not None:
            whole_units()
            oldest = [i for i, lds in enumerate(out) if lds][unit - 1]
            if waited > len(out) - 1 - oldest:
                fail(f"a unit is read with {waited} loads outstanding, {len(out) - 1 - oldest} behind it")
            del out[:oldest + 1]
            read, waited = read + 1, None
            if not any(out):
                out, unit = [], 0
        elif op.startswith("ds_read") and unit == 0:
            fail("a unit is read without a wait")
        places = [int(address.group(1), 16)] if address else []
        jump = re.search(r"<\S+?(?:\+0x([0-9a-f]+))?>\s*$", line) if op.startswith(("s_branch", "s_cbranch")) else None
        if jump:
            places.append(start + int(jump.group(1) or "0", 16))
        for place in places:
            if at.setdefault(place, sum(out)) != sum(out):
                fail(f"{sum(out)} and {at[place]} loads into LDS on their way at {place:#x}")
    if out:
        fail("loads into LDS on their way at its end")
    return read


SUM_STATES = 19       # most wait states between a product and another instruction on its sums
OPERAND_STATES = 2    # between a VALU instruction and a product that takes what it writes


def _registers(operand: str) -> set:
    m = re.fullmatch(r"-?\|?([va])(?:\[(\d+):(\d+)\]|(\d+))\|?", operand)
    if not m:
        return set()
    lo = int(m.group(2) or m.group(4))
    return {(m.group(1), i) for i in range(lo, int(m.group(3) or lo) + 1)}


class _Instruction:
    """What the products' wait states depend on, from a line of the listing."""

    def __init__(self, line: str):
        words = line.split("//")[0].replace(",", " ").split()
        self.text, op = line.strip(), words[0]
        self.product = op.startswith("v_mfma")
        self.states = int(words[1], 0) + 1 if op == "s_nop" else 1
        self.regs = set().union(*map(_registers, words[1:]))
        self.sums = _registers(words[1]) if self.product else set()
        self.writes = set()
        if op.startswith("v_") and not self.product and not op.startswith("v_cmp"):
            self.writes = _registers(words[1])
            if "swap" in op:      # (writes both operands)
                self.writes |= _registers(words[2])
        self.ends = op in ("s_branch", "s_endpgm", "s_setpc_b64")
        m = re.search(r"//\s*([0-9A-Fa-f]+):", line)
        self.address = int(m.group(1), 16) if m else None
        m = re.search(r"<\S+?(?:\+0x([0-9a-f]+))?>\s*$", line) if op.startswith(("s_branch", "s_cbranch")) else None
        self.jump = int(m.group(1) or "0", 16) if m else None     # from the start of the function


def _check_distances(ins: _Instruction, recent: list):
    states = 0
    for before in reversed(recent):
        if states >= SUM_STATES:
            return
        if ins.product and states < OPERAND_STATES and before.writes & ins.regs:
            raise RuntimeError(f"{ins.text} uses a register that was written {states} states before")
        if not ins.product and before.sums & ins.regs:
            raise RuntimeError(f"{ins.text} uses a sum of a product {states} states before")
        states += before.states


def _check_function(name: str, start: int, code: list):
    at = {ins.address: i for i, ins in enumerate(code) if ins.address is not None}
    paths = [(0, [], None)]       # where a path begins, what ran before it, how many states it is followed for (None: to the end)
    while paths:
        i, recent, left = paths.pop()
        while i < len(code) and (left is None or left > 0):
            ins = code[i]
            try:
                _check_distances(ins, recent)
            except RuntimeError as e:
                raise RuntimeError(f"{name}: {e}") from None
            recent = recent[-SUM_STATES:] + [ins]
            if left is not None:
                left -= ins.states
            if ins.jump is not None:
                if start + ins.jump not in at:
                    raise RuntimeError(f"{name}: {ins.text}: no instruction at its target")
                if left is None or left > 0:
                    paths.append((at[start + ins.jump], recent, SUM_STATES if left is None else left))
            if ins.ends:
                if left is not None:
                    break
                recent = []
            i += 1


def check_operands(listing: str) -> int:
    """Raises if an instruction of the wide kernel comes too close to a matrix instruction (see above); the number of matrix
    instructions."""
    products = 0
    name, start, code = "", 0, []

    def finish():
        nonlocal products
        if WIDE in name:
            _check_function(name, start, code)
            products += sum(ins.product for ins in code)

    for line in listing.splitlines():
        head = re.match(r"([0-9a-f]+) <(\S+)>:", line)
        if head:
            finish()
            name, start, code = head.group(2), int(head.group(1), 16), []
        elif WIDE in name and line.split("//")[0].strip():
            code.append(_Instruction(line))
    finish()
    return products


def check(lib_path: str) -> None:
    kernels = barriers = products = attention = units = 0
    for notes, listing in code_object_texts(lib_path):
        kernels += check_placement(notes)
        barriers += check_waits(listing)
        products += check_operands(listing)
        attention += check_attention_placement(notes)
        units += check_units(listing)
    if kernels == 0 or barriers < kernels or products == 0 or attention == 0 or units < attention:
        raise RuntimeError(f"{lib_path}: {kernels} kernels, {barriers} barriers, {products} products, {attention} attention kernels and {units} of their units found: the checks do not read this library")
