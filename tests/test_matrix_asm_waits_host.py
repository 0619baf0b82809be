"""Wait states round the matrix instructions and loads that the kernels issue as inline assembly.

The compiler puts wait states only round instructions that it knows, and it does not look inside inline assembly.  So the device code is compiled
to assembly with the library's flags, and every path to and from each such instruction is followed:

* a vector instruction that writes an operand of a matrix instruction (A, B, C or a scale) stands two wait states before it;
* what a matrix instruction writes is left alone for 20 wait states, but for a matrix instruction that adds to exactly it; nothing
  overwrites what it reads and writes in place in that time either;
* a vector instruction that writes a scalar operand of a load stands five wait states before it.

An instruction is one wait state, s_nop n is n + 1.  20 are more than any of these instructions asks for: 16 passes and 4.  These hold for the
code of one compiler and one set of flags: run this after a change of either.
"""
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2601_11589_amd import build

FILES = ["gemm.hip", "gemm_fp8.hip", "attention_rows.hip"]
VALU_TO_MATRIX, MATRIX_TO_ANY, VALU_TO_LOAD = 2, 20, 5
REG = re.compile(r"(?<![a-z0-9_.])(?:([vas])(\d+)\b|([vas])\[(\d+):(\d+)\]|(vcc|m0|exec)\b)")


class Instr:
    __slots__ = ("line", "name", "args", "asm", "states", "next", "prev", "matrix", "vector", "regs")

    def __init__(self, line, name, args, asm):
        self.line, self.name, self.args, self.asm = line, name, args, asm
        self.states = int(args[0], 0) + 1 if name == "s_nop" else 1
        self.next, self.prev = [], []
        self.matrix = name.startswith(("v_mfma", "v_smfmac"))
        self.vector = name.startswith("v_") and not self.matrix and name != "v_nop"
        self.regs = [registers(a) for a in args]

    def writes(self):
        """Registers that a vector or matrix instruction writes."""
        if not self.regs:
            return frozenset()
        if self.name.startswith("v_swap") or (self.name.startswith("v_permlane") and "swap" in self.name):
            return self.regs[0] | self.regs[1]
        out = self.regs[0]
        if "_co_" in self.name or self.name.startswith(("v_div_scale", "v_mad_u64_u32", "v_mad_i64_i32")):
            out = out | self.regs[1]
        return out

    def touches(self):
        return frozenset().union(*self.regs)

    def __str__(self):
        return f"line {self.line}: {self.name} {', '.join(self.args)}"


def registers(text):
    out = set()
    for one, at, many, lo, hi, named in REG.findall(text):
        if one:
            out.add(one + at)
        elif many:
            out.update(f"{many}{i}" for i in range(int(lo), int(hi) + 1))
        else:
            out.add(named)
    return frozenset(out)


def split(text):
    """Operands, commas in brackets apart."""
    return [a.strip() for a in re.split(r",(?![^\[]*\])", text)] if text else []


def functions(lines):
    """Lists of instructions, linked along every path, one a function."""
    code, labels, open_labels, asm, out = [], {}, [], False, []

    def link():
        for i, c in enumerate(code):
            ends = c.name in ("s_endpgm", "s_branch", "s_setpc_b64")
            to = [] if ends else code[i + 1:i + 2]
            if c.name == "s_branch" or c.name.startswith("s_cbranch"):
                assert c.args[0] in labels, c
                to = to + code[labels[c.args[0]]:labels[c.args[0]] + 1]
            c.next = to
            for t in to:
                t.prev.append(c)

    for number, line in enumerate(lines, 1):
        if "#ASMSTART" in line or "#ASMEND" in line:
            asm = "#ASMSTART" in line
            continue
        line = line.split(";")[0].strip()
        if line.startswith(".Lfunc_end"):
            link()
            out.append(code)
            code, labels = [], {}
        elif line.endswith(":"):
            labels[line[:-1]] = len(code)
        elif line and not line.startswith("."):
            name, _, rest = line.partition(" ") if " " in line else line.partition("\t")
            name, _, more = name.partition("\t")
            code.append(Instr(number, name, split((more + " " + rest).strip()), asm))
    return out


def before(start, most):
    """(instruction, wait states between it and `start`) on every path, as far as `most` allows."""
    seen, todo = {}, [(p, 0) for p in start.prev]
    while todo:
        c, gap = todo.pop()
        if gap >= most or seen.get(id(c), most) <= gap:
            continue
        seen[id(c)] = gap
        yield c, gap
        todo += [(p, gap + c.states) for p in c.prev]


def behind(start, most):
    seen, todo = {}, [(n, 0) for n in start.next]
    while todo:
        c, gap = todo.pop()
        if gap >= most or seen.get(id(c), most) <= gap:
            continue
        seen[id(c)] = gap
        yield c, gap
        todo += [(n, gap + c.states) for n in c.next]


def faults(code):
    """What breaks a rule, and how many instructions were looked at."""
    out, looked = [], 0
    for c in code:
        if c.asm and c.matrix:
            looked += 1
            reads = frozenset().union(*c.regs[1:])
            for p, gap in before(c, VALU_TO_MATRIX):
                if p.vector and p.writes() & reads:
                    out.append(f"{p} -> {gap} wait states -> {c}")
            for n, gap in behind(c, MATRIX_TO_ANY):
                same = n.matrix and n.regs[0] == n.regs[3] == c.regs[0] and not c.regs[0] & (n.regs[1] | n.regs[2])
                if not same and n.touches() & c.regs[0]:
                    out.append(f"{c} -> {gap} wait states -> {n}")
        elif c.asm and c.name.startswith("buffer_load"):
            looked += 1
            scalars = frozenset(r for r in c.touches() if r[0] == "s" or r == "vcc")
            for p, gap in before(c, VALU_TO_LOAD):
                if p.vector and p.writes() & scalars:
                    out.append(f"{p} -> {gap} wait states -> {c}")
    return out, looked


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    folder = tmp_path_factory.mktemp("asm")

    def compile_one(name):
        to = str(folder / (name + ".s"))
        cmd = [build.HIPCC] + build.COMMON + build.DEVICE_FLAGS + ["--offload-device-only", "-S", os.path.join(build.CSRC, name), "-o", to]
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        return to

    with ThreadPoolExecutor(len(FILES)) as pool:
        return dict(zip(FILES, pool.map(compile_one, FILES)))


@pytest.mark.parametrize("name", FILES)
def test_inline_matrix_instructions_have_their_wait_states(assembly, name):
    with open(assembly[name]) as f:
        found = [faults(code) for code in functions(f.readlines())]
    assert sum(looked for _, looked in found) > 50
    wrong = [text for texts, _ in found for text in texts]
    assert not wrong, f"{len(wrong)} of them:\n" + "\n".join(wrong[:20])


# The rules by hand: each listing with the number of its faults.
ACC = "v_mfma_f32_16x16x32_bf16 v[0:3], v[4:7], v[8:11], v[0:3]"
SCALED = "v_mfma_scale_f32_16x16x128_f8f6f4 a[0:3], v[8:15], v[16:23], a[0:3], v30, v31 op_sel_hi:[0,0,0]"


def inline(*lines):
    return [";;#ASMSTART", *lines, ";;#ASMEND"]


@pytest.mark.parametrize("lines, count", [
    (["v_and_b32_e32 v30, 0xff, v2", *inline(SCALED)], 1),
    (["v_and_b32_e32 v30, 0xff, v2", "s_waitcnt lgkmcnt(0)", *inline(SCALED)], 1),
    (["v_and_b32_e32 v30, 0xff, v2", *inline("s_nop 1", SCALED)], 0),
    (["v_and_b32_e32 v32, 0xff, v30", *inline(SCALED)], 0),
    (["v_and_b32_e32 v30, 0xff, v2", SCALED], 0),                                        # the compiler's own: it knows
    (["ds_read_u8 v30, v2", "s_waitcnt lgkmcnt(0)", *inline(SCALED)], 0),
    (["v_mov_b32_e32 v7, v40", *inline("s_nop 0", ACC)], 1),
    (["v_swap_b32 v40, v7", *inline(ACC)], 1),
    ([*inline(ACC), *inline(ACC)], 0),
    ([*inline(ACC), "s_nop 15", "v_mov_b32_e32 v40, v3"], 1),
    ([*inline(ACC), "s_nop 15", "s_nop 3", "v_mov_b32_e32 v40, v3"], 0),
    ([*inline(ACC), "ds_write_b32 v50, v2"], 1),
    ([*inline(ACC), *inline("v_mfma_f32_16x16x32_bf16 v[40:43], v[0:3], v[8:11], v[40:43]")], 1),
    ([*inline(ACC), *inline("v_mfma_f32_16x16x32_bf16 v[2:5], v[12:15], v[8:11], v[2:5]")], 1),
    # round a loop: the write stands behind the instruction that reads it
    ([".LBB0_1:", *inline(SCALED), "v_mov_b32_e32 v31, v60", "s_cbranch_scc1 .LBB0_1"], 1),
    ([".LBB0_1:", *inline(SCALED), "v_mov_b32_e32 v31, v60", "s_nop 0", "s_cbranch_scc1 .LBB0_1"], 0),
    (["s_branch .LBB0_2", ".LBB0_1:", "v_mov_b32_e32 v31, v60", ".LBB0_2:", *inline(SCALED)], 1),
    (["v_readlane_b32 s6, v60, 3", "s_nop 3", *inline("s_mov_b32 m0, s20", "s_nop 0", "buffer_load_dwordx4 v1, s[4:7], s9 offen lds")], 0),
    (["v_readlane_b32 s6, v60, 3", *inline("s_mov_b32 m0, s20", "s_nop 0", "buffer_load_dwordx4 v1, s[4:7], s9 offen lds")], 1),
])
def test_the_rules_by_hand(lines, count):
    (code,) = functions([*lines, "s_endpgm", ".Lfunc_end0:"])
    assert len(faults(code)[0]) == count, faults(code)
