"""Build-time guards over what the compiler makes of the matrix-core kernels for gfx950.

scan(), over the assembly:
v_mfma ignores the execution mask.  The compiler lowers a branch on a value it cannot prove
wave-uniform to an exec-mask update, and for short blocks it drops the branch that would skip the
block when the mask is empty; a matrix instruction in such a block then runs on registers whose loads
were skipped.  The kernels keep every condition around a matrix instruction scalar; this scan checks
the result: it fails when a v_mfma sits between a saveexec that no skip branch follows and the
restore of exec.

undefined_operands(), over the machine code behind the register allocator: elements of one vector that are loop variables of their
own share a register tuple, and where a loop's exit leaves them undefined, this compiler (ROCm 7.2) notes that for the tuple's
first element alone.  The allocator then takes the others for undefined inside the loop as well, where they hold values, and
may give their registers to temporaries: wrong results in some builds and not in others.  It marks such operands "undef".  The
kernels keep such vectors whole; nothing in them reads a value that the source left undefined, so any marked vector register is a fault.
"""
from __future__ import annotations

import re
from typing import Iterable, List

_LABEL = re.compile(r"^(_Z\w+):")


def scan(asm_text: str) -> List[str]:
    """Returns one message per suspect matrix instruction."""
    out: List[str] = []
    kernel = "?"
    pending = 0   # line of a saveexec whose next instruction has not been seen yet
    masked = 0    # line of the saveexec that opened an unskipped masked block
    for ln, line in enumerate(asm_text.splitlines(), 1):
        t = line.strip()
        m = _LABEL.match(t)
        if m:
            kernel, pending, masked = m.group(1), 0, 0
            continue
        if not t or t[0] in ";.":
            continue
        fields = t.replace(",", " ").split()
        ins = fields[0]
        if pending:
            if not ins.startswith("s_cbranch_exec"):
                masked = pending
            pending = 0
        if "saveexec" in ins:
            pending = ln
            continue
        if ins in ("s_or_b64", "s_mov_b64") and len(fields) > 1 and fields[1] == "exec":
            masked = 0
        if ins.startswith("v_mfma") and masked:
            out.append(f"line {ln}: {kernel}: matrix instruction in a masked block without a skip branch "
                       f"(exec narrowed at line {masked})")
    return out


_FUNCTION = re.compile(r"^name:\s+(\S+)")
_UNDEF = re.compile(r"\bundef (?:renamable )?\$[av]gpr\d+")


def undefined_operands(mir: Iterable[str]) -> List[str]:
    """One message per instruction with a source among the vector registers that the allocator takes for undefined, from the lines of
    the machine code printed behind it."""
    out: List[str] = []
    kernel = "?"
    for line in mir:
        if "undef" in line:
            if _UNDEF.search(line.split(" = ", 1)[-1]):  # (in front of it: a result, of which only a part is written)
                out.append(f"{kernel}: operand taken for undefined: {line.strip()[:120]}")
        elif line.startswith("name:"):
            m = _FUNCTION.match(line)
            kernel = m.group(1) if m else "?"
    if kernel == "?":
        out.append("no function in what was printed: the compiler knows another name for the place behind the allocator")
    return out
