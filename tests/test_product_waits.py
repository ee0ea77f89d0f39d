"""Matrix products and the vector instructions that use their results, in the built library's gfx950 code.

A product's registers are there some wait states after it is issued, and neither the hardware nor the
instruction checks that: the compiler leaves instructions or s_nop between.  It counts them along the blocks of
a function.  Where a block ends in a conditional branch followed by an unconditional one it counts the second
also on the path that takes the first, where it is never executed, and a block that it has come to over a long way
it does not look through again over a short one: such paths can be some states short.  One was (an accumulator's
last register, read at the top of a loop 11 states after the product at its end: two dims of a row were wrong).
The kernels put waits of their own where products are still under way at the end of a block; this goes along
every path, with what is executed on it, and looks whether the states are there."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2505_22654_amd import build as vbuild

OBJDUMP = os.environ.get("LLVM_OBJDUMP", "/opt/rocm/llvm/bin/llvm-objdump")

# 4-cycle passes of the products that the library uses, and the states after which a vector instruction may
# use what they write: one more than three past the last pass; for the fp32 ones two past it.
PASSES = {"v_mfma_f32_16x16x32_bf16": 4, "v_mfma_f32_16x16x32_f16": 4, "v_mfma_f32_32x32x16_bf16": 8,
          "v_mfma_f32_32x32x16_f16": 8, "v_mfma_scale_f32_32x32x64_f8f6f4": 16}
FP32_PASSES = {"v_mfma_f32_16x16x4_f32": 8, "v_mfma_f32_32x32x2_f32": 16}
STATES = {**{n: p + 4 for n, p in PASSES.items()}, **{n: p + 2 for n, p in FP32_PASSES.items()}}
VECTOR = ("v_", "ds_", "global_", "buffer_", "flat_", "scratch_")
OPERAND = re.compile(r"\b([av])(?:\[(\d+):(\d+)\]|(\d+)\b)")


def registers(text):
    out = set()
    for kind, lo, hi, one in OPERAND.findall(text):
        out.update((kind, i) for i in (range(int(lo), int(hi) + 1) if lo else (int(one),)))
    return frozenset(out)


class Instruction:
    def __init__(self, line):
        text, _, note = line.partition("//")
        self.text = text.strip()
        self.op, _, rest = self.text.partition(" ")
        self.product = self.op.startswith(("v_mfma", "v_smfmac"))
        self.vector = self.op.startswith(VECTOR)
        self.states = int(rest) + 1 if self.op == "s_nop" else 1
        self.address = int(note.split(":")[0], 16)
        target = re.search(r"<.*\+0x([0-9a-f]+)>", note) if self.op.startswith(("s_branch", "s_cbranch")) else None
        self.jump = int(target.group(1), 16) if target else None   # from the function's start
        args = re.split(r",\s*(?![^\[]*\])", rest) if self.vector else []
        self.uses = registers(rest) if self.vector else frozenset()
        if self.product:
            self.result, self.factors = registers(args[0]), registers(args[1]) | registers(args[2])


def functions(code):
    """(name, instructions) of a disassembly."""
    for part in re.split(r"\n(?=[0-9a-f]+ <)", code)[1:]:
        head, *lines = part.split("\n")
        yield head.split("<", 1)[1].rstrip(">:"), [Instruction(l) for l in lines if "//" in l]


def short_waits(instructions):
    """(product, instruction that uses it, states between, states needed) where too few are left."""
    if not instructions:
        return
    at = {i.address - instructions[0].address: n for n, i in enumerate(instructions)}
    for n, p in enumerate(instructions):
        if not p.product:
            continue
        need, seen, todo = STATES[p.op], {}, [(n + 1, 0, p.result)]
        while todo:
            i, states, live = todo.pop()
            while i < len(instructions) and states < need and live:
                x = instructions[i]
                # (fewer states left to go, or more registers, than another path that came here)
                if any(s <= states and live <= r for s, r in seen.get(i, ())):
                    break
                seen.setdefault(i, []).append((states, live))
                if x.product:
                    if x.factors & live:
                        yield p, x, states, need
                    live = live - x.result       # (accumulated in the pipe, or its own to wait for)
                elif x.vector and x.uses & live:
                    yield p, x, states, need
                    live = live - x.uses
                states += x.states
                if x.jump is not None:
                    todo.append((at[x.jump], states, live))
                if x.op in ("s_branch", "s_endpgm", "s_setpc_b64"):
                    break
                i += 1


def disassembly(tmp_path):
    copy = shutil.copy(vbuild.LIB, str(tmp_path / "lib.so"))
    subprocess.run([OBJDUMP, "--offloading", copy], check=True, capture_output=True, cwd=tmp_path)
    parts = sorted(f for f in os.listdir(tmp_path) if "gfx950" in f)
    assert parts
    for f in parts:
        yield subprocess.run([OBJDUMP, "-d", str(tmp_path / f)], check=True, capture_output=True, text=True).stdout


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler for gfx950")
def test_vector_instructions_wait_for_products(tmp_path):
    products, short = 0, []
    for code in disassembly(tmp_path):
        for name, instructions in functions(code):
            products += sum(i.product for i in instructions)
            short += [f"{name}: {p.text} | {x.text} at {x.address:x}, {states} states of {need}"
                      for p, x, states, need in short_waits(instructions)]
    assert products > 1000
    assert not short, "\n".join(short[:20]) + f"\n{len(short)} in all"


LOOP = """
0000000000000100 <f>:
	v_accvgpr_read_b32 v1, a15                                 // 000000000100: 00000000
	s_nop 3                                                    // 000000000108: 00000000
	v_mfma_f32_32x32x16_bf16 a[0:15], v[4:7], v[8:11], a[0:15] // 00000000010C: 00000000
	s_cmp_lt_i32 s0, s1                                        // 000000000114: 00000000
	s_cbranch_scc1 1                                           // 000000000118: 00000000 <f+0x20>
	s_branch 9                                                 // 00000000011C: 00000000 <f+0x28>
	s_nop {wait}                                                    // 000000000120: 00000000
	s_branch -9                                                // 000000000124: 00000000 <f+0x0>
	s_endpgm                                                   // 000000000128: 00000000
"""


@pytest.mark.parametrize("wait,short", [(7, 1), (8, 0)])
def test_a_branch_that_is_not_taken_is_no_wait(wait, short):
    """s_cmp, the taken branch, s_nop (wait + 1 states) and the branch back: wait + 4 of 12."""
    (_, instructions), = functions(LOOP.format(wait=wait))
    found = list(short_waits(instructions))
    assert len(found) == short and all(s == wait + 4 and need == 12 for _, _, s, need in found)
