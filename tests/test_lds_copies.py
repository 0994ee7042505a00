"""Copies from global memory to LDS take their LDS address from m0, which needs
a wait state after it has been written (the compiler sees to it in its own code,
not inside inline assembly): each statement that does both has it."""

import glob
import os
import re
import struct
import subprocess

import pytest

from paper_2607_14530_amd import xhc as X

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_14530_amd", "csrc")


def statements():
    """(file, instructions) of the inline assembly that writes m0"""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.hip"))):
        for m in re.finditer(r"asm\s+volatile\s*\(((?:\s*\"(?:[^\"\\]|\\.)*\")+)", open(path).read()):
            text = "".join(re.findall(r"\"((?:[^\"\\]|\\.)*)\"", m.group(1)))
            lines = [s.strip() for s in re.split(r"\\n|;|\\t", text) if s.strip()]
            if any(re.match(r"s_\w+ m0\b", s) for s in lines):
                yield os.path.basename(path), lines


def is_copy(s):
    return re.match(r"(global_load_lds|scratch_load_lds)", s) or (s.startswith("buffer_load") and s.endswith("lds"))


def test_the_statements_are_found():
    names = [n for n, lines in statements() for s in lines if is_copy(s)]
    assert names.count("xhc_device.h") == 2 and names.count("xhc_ffn.h") == 1


@pytest.mark.parametrize("name,lines", list(statements()))
def test_m0_is_waited_for(name, lines):
    written = None
    for i, s in enumerate(lines):
        if re.match(r"s_\w+ m0\b", s):
            written = i
        if is_copy(s) and written is not None:
            between = lines[written + 1:i]
            assert between and between[0].startswith("s_nop"), (name, lines)


# ---------------------------------------------------------------- the built code

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"
OFF = 99            # further back than is looked for


def code_objects():
    """The library's device code, an ELF for each source."""
    data = open(X.LIB_PATH, "rb").read()
    at = data.find(MAGIC)
    while at >= 0:
        p = at + len(MAGIC) + 8
        for _ in range(struct.unpack_from("<Q", data, p - 8)[0]):
            off, size, n = struct.unpack_from("<QQQ", data, p)
            if data[p + 24:p + 24 + n].endswith(b"gfx950"):
                yield data[at + off:at + off + size]
            p += 24 + n
        at = data.find(MAGIC, at + 1)


def scalars(operand):
    """Scalar registers of an operand, m0 as -1"""
    if operand == "m0":
        return {-1}
    m = re.fullmatch(r"s\[(\d+):(\d+)\]|s(\d+)", operand)
    if not m:
        return set()
    return {int(m[3])} if m[3] else set(range(int(m[1]), int(m[2]) + 1))


def kernels(path):
    """(name, instructions) of the functions with a copy; an instruction is its text, or a label's"""
    text = subprocess.run([OBJDUMP, "-d", "--symbolize-operands", "--no-show-raw-insn", path], capture_output=True,
                          text=True, check=True).stdout
    for part in re.split(r"\n(?=[0-9a-f]+ <_Z)", text)[1:]:
        if " lds" in part or "_load_lds" in part:
            lines = [s.split("//")[0].strip() for s in part.split("\n")]
            yield lines[0], [re.sub(r"^[0-9a-f]+ (?=<)", "", s) for s in lines[1:] if s]


def nearest(ins, at, registers, vector):
    """Fewest wait states between instruction `at` and a write of one of the registers, by a vector (or a scalar)
    instruction, over all ways there."""
    labels = {s[1:-2]: i for i, s in enumerate(ins) if s.startswith("<")}
    jumps = {}
    for i, s in enumerate(ins):
        if s.startswith(("s_branch", "s_cbranch")):
            jumps.setdefault(labels[s.split()[-1]], []).append(i)

    def before(i):
        fall = [i - 1] if i > 0 and not ins[i - 1].startswith(("s_branch", "s_endpgm", "s_setpc")) else []
        return fall + jumps.get(i, [])

    best, seen, todo = OFF, {}, [(p, 0) for p in before(at)]
    while todo:
        i, states = todo.pop()
        if states >= 5 or seen.get(i, OFF) <= states:
            continue
        seen[i] = states
        s = ins[i]
        if s.startswith("<"):
            todo += [(p, states) for p in before(i)]
            continue
        op, *rest = s.split(None, 1)
        operands = [o.strip() for o in re.split(r",(?![^\[]*\])", rest[0])] if rest else []
        written = operands[:2] if re.match(r"v_(add_co|addc|sub_co|subb|subrev_co|div_scale|mad_u64|mad_i64)", op) \
            else operands[:1]
        if op.startswith("v_" if vector else "s_") and any(scalars(o) & registers for o in written):
            best = min(best, states)
            continue
        states += int(operands[0]) + 1 if op == "s_nop" else 1
        todo += [(p, states) for p in before(i)]
    return best


@pytest.mark.skipif(not (os.path.exists(OBJDUMP) and os.path.exists(X.LIB_PATH)),
                    reason="needs the library and llvm-objdump")
def test_the_built_copies_wait(tmp_path):
    """Every copy to LDS in the library: a wait state at least behind a scalar write of m0, five behind a vector
    write (v_readfirstlane, say) of a descriptor or an offset.  The compiler cannot look into the copies' statements,
    so what it puts in front of them is checked here."""
    found = 0
    for k, code in enumerate(code_objects()):
        path = str(tmp_path / f"{k}.o")
        open(path, "wb").write(code)
        for name, ins in kernels(path):
            for i, s in enumerate(ins):
                if not is_copy(s):
                    continue
                found += 1
                registers = set()
                for o in re.split(r"[ ,]+(?![^\[]*\])", s)[1:]:
                    registers |= scalars(o)
                assert nearest(ins, i, {-1}, False) >= 1, (name, s)
                assert not registers or nearest(ins, i, registers, True) >= 5, (name, s)
    assert found > 600, found
