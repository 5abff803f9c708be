"""Matrix instructions written in inline asm get no wait states from the compiler.  The code of the latent attention's kernels, which have them, is read
back from the built library: a register written by a vector instruction is read by a matrix instruction two wait states later at the earliest (which is
what the compiler keeps for its own), and what a matrix instruction writes is touched by another instruction its passes and three more later, unless the
next product adds to all of it.  Needs no GPU."""
import os
import re
import subprocess

import pytest

from paper_2503_10325_amd import binding as sv
from test_kernel_resources import code_objects

OBJDUMP = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")
pytestmark = pytest.mark.skipif(not (os.path.exists(sv.LIB_PATH) and os.path.exists(OBJDUMP)), reason="libspecverify.so or llvm-objdump is not there")

LINE = re.compile(r"^\t(\S+)\s*(.*?)\s*// ([0-9A-F]+):(.*)$")
PASSES = {"v_mfma_f32_32x32x16_bf16": 8, "v_mfma_f32_16x16x32_bf16": 4}       # of four cycles


def registers(operand):
    found = set()
    for kind, first, last, one in re.findall(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+)\b)", operand):
        found.update([kind + one] if one else (kind + str(i) for i in range(int(first), int(last) + 1)))
    return found


def operands(text):
    return [x.strip() for x in re.split(r",(?![^\[]*\])", text)]


class Instruction:
    def __init__(self, op, text, target):
        self.op, self.target = op, target
        self.matrix, self.vector = op.startswith("v_mfma"), op.startswith("v_") and not op.startswith("v_mfma")
        self.states = int(text, 0) + 1 if op == "s_nop" else 1
        parts = [] if op.startswith("s_") else [registers(x) for x in operands(text)]
        everything = set().union(*parts)
        writes = parts[:1]
        if op.startswith(("v_permlane16_swap", "v_permlane32_swap", "v_swap")):
            writes = parts[:2]
        elif not (op.startswith("v_") or op.startswith("ds_read") or "_load_" in op and "lds" not in op and not re.search(r"\blds\b", text)):
            writes = []
        self.writes, self.touches = set().union(*writes), everything
        if self.matrix:
            self.a_b, self.c = parts[1] | parts[2], parts[3]
            self.touches = self.a_b | self.c


def functions(listing):
    """(name, instructions, places that control may go to from each) of every function."""
    name, start, code = None, 0, []

    def whole():
        place = {at: i for i, (at, _) in enumerate(code)}
        after = []
        for i, (_, x) in enumerate(code):
            to = [] if x.op in ("s_branch", "s_endpgm") or i + 1 == len(code) else [i + 1]
            after.append(to + ([place[start + x.target]] if x.target is not None else []))
        return name, [x for _, x in code], after

    for line in listing.splitlines():
        head = re.match(r"^([0-9a-f]+) <(.+)>:$", line)
        if head:
            if code:
                yield whole()
            name, start, code = head.group(2), int(head.group(1), 16), []
            continue
        got = LINE.match(line)
        if got and name:
            op, text, at, rest = got.groups()
            target = re.search(r"<[^>]*\+0x([0-9a-f]+)>", rest) if op == "s_branch" or op.startswith("s_cbranch") else None
            code.append((int(at, 16), Instruction(op, text, int(target.group(1), 16) if target else None)))
    if code:
        yield whole()


def follow(code, after, i, states, look):
    """look(instruction) of all that may come fewer than `states` wait states behind i, each way until it says that the register is another's."""
    best, todo = {}, [(j, 0) for j in after[i]]
    while todo:
        j, waited = todo.pop()
        if waited >= states or best.get(j, states) <= waited:
            continue
        best[j] = waited
        if not look(code[j]):
            todo += [(k, waited + code[j].states) for k in after[j]]


def too_close(code, after):
    found = []
    for i, x in enumerate(code):
        if x.vector and x.writes:
            def behind_vector(y, x=x):
                if y.matrix and x.writes & y.touches:
                    found.append((x.op, sorted(x.writes)[0], y.op))
                return x.writes <= y.writes
            follow(code, after, i, 2, behind_vector)
        if x.matrix:
            def behind_matrix(y, x=x):
                if y.matrix:
                    if x.writes & y.a_b or x.writes & y.c and x.writes != y.c:
                        found.append((x.op, sorted(x.writes)[0], y.op))
                    return x.writes <= y.writes
                hit = bool(x.writes & (y.writes | y.touches))
                if hit:
                    found.append((x.op, sorted(x.writes)[0], y.op))
                return hit
            follow(code, after, i, PASSES[x.op] + 3, behind_matrix)
    return found


def listings(tmp_path):
    with open(sv.LIB_PATH, "rb") as f:
        for elf in code_objects(f.read()):
            if b"attn_latent_kernel" in elf:
                path = tmp_path / "code"
                path.write_bytes(elf)
                yield subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", str(path)], capture_output=True, text=True, check=True).stdout


def example(*lines):
    """The function of those instructions."""
    return next(functions("0 <f>:\n" + "".join(f"\t{x} // {i:X}: 00000000\n" for i, x in enumerate(lines))))[1:]


PRODUCT = "v_mfma_f32_32x32x16_bf16 a[0:15], v[0:3], v[4:7], a[0:15]"


@pytest.mark.parametrize("lines,count", [
    (("v_accvgpr_mov_b32 a15, a40", PRODUCT, "s_endpgm"), 1),
    (("v_accvgpr_mov_b32 a15, a40", "s_nop 0", PRODUCT, "s_endpgm"), 1),
    (("v_accvgpr_mov_b32 a15, a40", "s_nop 1", PRODUCT, "s_endpgm"), 0),
    (("v_mov_b32_e32 v5, v9", PRODUCT, "s_endpgm"), 1),
    ((PRODUCT, "s_nop 9", "v_accvgpr_read_b32 v9, a3", "s_endpgm"), 1),
    ((PRODUCT, "s_nop 10", "v_accvgpr_read_b32 v9, a3", "s_endpgm"), 0),
    ((PRODUCT, PRODUCT, "s_endpgm"), 0),
])
def test_what_counts_as_too_close(lines, count):
    assert len(too_close(*example(*lines))) == count


def test_products_wait_for_their_operands_and_others_for_their_results(tmp_path):
    kernels, bad = 0, {}
    for text in listings(tmp_path):
        for name, code, after in functions(text):
            if any(x.matrix for x in code):
                kernels += 1
                close = too_close(code, after)
                if close:
                    bad[name] = (len(close), close[:3])
    assert kernels >= 32 and not bad
