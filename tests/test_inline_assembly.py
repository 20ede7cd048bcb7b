"""Wait states that the compiler does not keep for inline assembly: a vector memory instruction may read a scalar
register 5 wait states after a vector instruction wrote it, no sooner (v_readlane writes one wherever a spilled scalar
register comes back). Looked for in the sources' assembly statements and in the built library's instructions."""
import glob
import os
import re
import shutil
import subprocess

import pytest

from paper_2411_01783_amd import build

WAIT_STATES = 5
MEMORY = ("global_", "flat_", "buffer_", "scratch_")


def states(instruction):
    m = re.match(r"s_nop\s+(\w+)", instruction)
    return int(m.group(1), 0) + 1 if m else 1


def scalars(operand):
    """Numbers of the scalar registers that an operand names."""
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", operand)
    if m:
        return set(range(int(m.group(1)), int(m.group(2)) + 1))
    m = re.fullmatch(r"s(\d+)", operand)
    return {int(m.group(1))} if m else set()


def too_soon(lines):
    """Memory instructions that read a scalar register fewer than WAIT_STATES behind a vector write of it."""
    recent, found = [], []
    for line in lines:
        parts = line.split(None, 1)
        op, args = parts[0], [a.strip().split(" ")[0] for a in parts[1].split(",")] if len(parts) > 1 else []
        if op.startswith(MEMORY):
            read, gap = set().union(*[scalars(a) for a in args]) if args else set(), 0
            for written, n, what in reversed(recent):
                if gap >= WAIT_STATES:
                    break
                if written & read:
                    found.append("%s, %d behind %s" % (line, gap, what))
                    break
                gap += n
        written = set()
        if op.startswith("v_") and args:
            written = scalars(args[0]) | (scalars(args[1]) if "_co_" in op else set())
        recent = recent[-8:] + [(written, states(line), line)]
    return found


def test_the_search_finds_what_it_is_for():
    load = "global_load_lds_dwordx4 v1, s[4:5]"
    assert too_soon(["v_readlane_b32 s5, v9, 3", "s_mov_b32 m0, s2", "s_nop 0", load])
    assert not too_soon(["v_readlane_b32 s5, v9, 3", "s_mov_b32 m0, s2", "s_nop 3", load])
    assert not too_soon(["v_readlane_b32 s6, v9, 3", load])
    assert too_soon(["v_cmp_gt_i32_e64 s[4:5], v1, v2", "buffer_load_dword v1, off, s[4:7], 0"])


def test_memory_instructions_in_assembly_statements_wait_for_their_scalars():
    seen = 0
    for path in glob.glob(os.path.join(build.CSRC, "*")):
        for body in re.findall(r"asm volatile\((.*?)\);", open(path).read(), flags=re.S):
            text, _, operands = body.partition(":")
            code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', text)).replace("\\n", "\n").replace("\\t", " ")
            lines = [x.strip() for x in code.split("\n") if x.strip()]
            kinds = re.findall(r'"([^"]*)"\s*\(', operands)
            gap = 0
            for line in lines:
                named = [int(x) for x in re.findall(r"%(\d+)", line)]
                if line.startswith(MEMORY) and any(kinds[i] == "s" for i in named):
                    seen += 1
                    assert gap >= WAIT_STATES, (path, line)
                gap += states(line)
    assert seen > 0


def test_built_library_keeps_the_wait_states(tmp_path):
    objdump = "/opt/rocm/llvm/bin/llvm-objdump"
    if not os.path.exists(objdump):
        pytest.skip("no llvm-objdump")
    lib = str(tmp_path / "lib.so")
    shutil.copy(build.build(), lib)
    subprocess.run([objdump, "--offloading", lib], check=True, capture_output=True, cwd=tmp_path)
    objects = glob.glob(lib + "*gfx950*")
    assert objects
    instructions, found = 0, []
    for obj in objects:
        text = subprocess.run([objdump, "-d", "--no-show-raw-insn", "--no-leading-addr", obj], check=True,
                              capture_output=True, text=True).stdout
        lines = [x.split("//")[0].strip() for x in text.split("\n") if x.startswith((" ", "\t"))]
        lines = [x for x in lines if x]
        instructions += len(lines)
        found += too_soon(lines)
    assert instructions > 100000
    assert not found, found[:5]
