"""The assembly that the compiler makes of csrc/linear_tiles.hip.  The kernels of 256 x 256 tiles issue their matrix instructions as inline assembly, where the compiler does not keep the distances that the
hardware asks for.  They hold by how the kernel is written, and here by looking along every path through the code: two wait states from a vector instruction that writes an operand or accumulator to the matrix
instruction that reads it, twelve from a matrix instruction to anything else that reads or writes its accumulators."""
import os
import re
import subprocess
import tempfile
from collections import defaultdict

import pytest

from paper_2602_06079_amd import build as B

OPERANDS, RESULTS = 2, 12      # wait states
_REG = re.compile(r"(?<![\w.])([va])(?:\[(\d+):(\d+)\]|(\d+))(?!\w)")


def registers(text):
    """The vector registers that an operand names."""
    return {(k, i) for k, lo, hi, one in _REG.findall(text) for i in (range(int(lo), int(hi) + 1) if lo else [int(one)])}


class Kernel:
    """Instructions of a kernel as (name, [operands]), and which of them may come before each."""

    def __init__(self, lines):
        self.code, labels, self.before = [], {}, defaultdict(list)
        for line in lines:
            line = line.split(";")[0].strip()
            if not line or line.startswith("."):
                if line.endswith(":"):
                    labels[line[:-1]] = len(self.code)
                continue
            if line.endswith(":"):
                labels[line[:-1]] = len(self.code)
                continue
            name, _, rest = line.partition(" ")
            self.code.append((name, [x.strip() for x in re.split(r",(?![^\[]*\])", rest)]))
        for i, (name, ops) in enumerate(self.code):
            if name.startswith(("s_branch", "s_cbranch")):
                self.before[labels[ops[0]]].append(i)
            if name not in ("s_branch", "s_endpgm", "s_setpc_b64"):
                self.before[i + 1].append(i)
        assert not any(n.startswith(("s_swappc", "s_setpc", "s_call")) for n, _ in self.code)

    def matrix(self, i):
        return self.code[i][0].startswith("v_mfma")

    def writes(self, i):
        """What a vector instruction (not a load) writes."""
        name, ops = self.code[i]
        if not name.startswith("v_") or name.startswith("v_cmp"):
            return set()
        if name.startswith("v_swap"):
            return registers(ops[0]) | registers(ops[1])
        return registers(ops[0])

    def all(self, i):
        return registers(", ".join(self.code[i][1]))

    def earlier(self, i, states):
        """Every instruction that some path has fewer than that many wait states before i."""
        todo, seen = [(p, 0) for p in self.before[i]], {}
        while todo:
            p, gone = todo.pop()
            if seen.get(p, states) <= gone:
                continue
            seen[p] = gone
            name, ops = self.code[p]
            gone += int(ops[0], 0) + 1 if name == "s_nop" else 1
            if gone < states:
                todo += [(q, gone) for q in self.before[p]]
        return seen

    def faults(self):
        found, matrix = [], [self.matrix(i) for i in range(len(self.code))]
        accumulators = set().union(*[self.writes(i) for i in range(len(self.code)) if matrix[i]])
        for i, (name, ops) in enumerate(self.code):
            if matrix[i]:
                need = registers(", ".join(ops[1:]))
                if ops[0] != ops[3]:
                    found.append("%d: %s of other accumulators" % (i, name))
                found += ["%d: %s %s behind %s %s" % (i, name, ops, *self.code[p]) for p in self.earlier(i, OPERANDS) if not matrix[p] and self.writes(p) & need]
            else:
                touched = self.all(i) & accumulators
                if touched:
                    found += ["%d: %s %s behind %s" % (i, name, ops, self.code[p][1][0]) for p in self.earlier(i, RESULTS) if matrix[p] and self.writes(p) & touched]
        return found


def kernels_of(text):
    found, name, lines = {}, None, []
    for line in text.splitlines():
        m = re.match(r"(_ZN\w*k_linear\w*):", line)
        if m:
            name, lines = m.group(1), []
        elif name and line.startswith(".Lfunc_end"):
            found[name] = lines
            name = None
        elif name:
            lines.append(line)
    return found


def by_hand(lines):
    return any("ASMSTART" in a and "v_mfma" in b for a, b in zip(lines, lines[1:]))


@pytest.fixture(scope="module")
def kernels():
    """Those whose matrix instructions are inline assembly."""
    with tempfile.TemporaryDirectory() as d:
        out = os.path.join(d, "linear_tiles.s")
        subprocess.run([B.HIPCC] + B.HIP_FLAGS + ["--cuda-device-only", "-S", os.path.join(B.CSRC, "linear_tiles.hip"), "-o", out], check=True, capture_output=True)
        with open(out) as f:
            found = {k: v for k, v in kernels_of(f.read()).items() if by_hand(v)}
    assert len(found) == 7       # four orientations, with and without a ragged k, but where both operands lie across it
    return found


def test_distances(kernels):
    for name, lines in kernels.items():
        assert sum("v_mfma" in x for x in lines) >= 512       # two rounds of four steps
        assert Kernel(lines).faults() == [], name


def test_planted_mistakes(kernels):
    """An operand or an accumulator moved right before its use, other accumulators, and a result read at once are all seen."""
    lines = next(iter(kernels.values()))
    at = [i for i, x in enumerate(lines) if "v_mfma" in x][100]
    ops = [x.strip() for x in re.split(r",(?![^\[]*\])", lines[at].split(None, 1)[1])]
    c, p, q = (re.sub(r"\[(\d+):.*", r"\1", x) for x in ops[:3])

    def with_line(i, text):
        return Kernel(lines[:i] + [text] + lines[i:]).faults()

    for reg in (p, q):
        assert with_line(at, "\tv_mov_b32_e32 %s, 0" % reg)
    assert with_line(at, "\tv_accvgpr_write_b32 %s, 0" % c)
    assert with_line(at + 1, "\tv_accvgpr_read_b32 v0, %s" % c)
    assert Kernel(lines[:at] + [lines[at].replace(ops[0], "a[0:3]", 1) if ops[0] != "a[0:3]" else lines[at].replace(ops[0], "a[4:7]", 1)] + lines[at + 1:]).faults()


def test_paths_through_a_loop():
    """What ends a loop comes before what begins it, and before what follows it."""
    matrix = "v_mfma_f32_16x16x32_bf16 a[0:3], v[0:3], v[4:7], a[0:3]"
    for between, operand, result in (([], True, True), (["s_nop 0"], False, True), (["s_nop 10"], False, False)):
        assert bool(Kernel([".L1:", matrix, "s_nop 15", "v_mov_b32_e32 v1, 0"] + between + ["s_cbranch_scc1 .L1", "s_endpgm"]).faults()) == operand
        assert bool(Kernel([".L1:", matrix] + between + ["s_cbranch_scc1 .L1", "v_accvgpr_read_b32 v9, a0", "s_endpgm"]).faults()) == result
