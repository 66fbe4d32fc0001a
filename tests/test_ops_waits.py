"""The waits that the operators' inline assembly leaves to the order of instructions, checked in the built library's own code.

The compiler knows no hazards between inline assembly and what it puts around it.  In the kernels of the matrix products
  - a matrix instruction reads a register two states after a vector instruction wrote it, or later,
  - a load to LDS reads its descriptor five states after a vector instruction (v_readfirstlane) wrote it, or later, and m0 one state,
  - a vector instruction or store reads a sum seven states after the product that wrote it, or later.
A state is an instruction, s_nop n stands for n + 1 of them."""
import os
import re
import subprocess

import pytest

from paper_1610_02496_amd import build

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
FAR = 12   # instructions that one look back or across a branch covers


def registers(kind, text):
    out = set()
    for one, lo, hi in re.findall(r"\b%s(?:(\d+)|\[(\d+):(\d+)\])" % kind, text):
        out |= {int(one)} if one else set(range(int(lo), int(hi) + 1))
    return {(kind, r) for r in out}


def both(text):
    return registers("v", text) | registers("a", text)


class Instruction:
    def __init__(self, address, op, rest):
        args = rest.split(",")
        self.text, self.address, self.states = "%x: %s %s" % (address, op, rest), address, int(rest, 0) + 1 if op == "s_nop" else 1
        self.product, self.load = op.startswith("v_mfma"), op.startswith("buffer_load") and rest.endswith("lds")
        vector = op.startswith("v_") and not self.product
        self.target = address + 4 + 4 * ((int(rest.split()[0]) + 0x8000) % 0x10000 - 0x8000) if op.startswith(("s_cbranch", "s_branch")) else None
        self.ends = op in ("s_branch", "s_endpgm")
        pair = "swap" in op or op.startswith("v_permlane") and "swap" in op
        self.vector_writes = both(",".join(args[:2 if pair else 1])) | registers("s", args[0]) if vector else set()
        self.product_writes = both(args[0]) if self.product else set()
        self.moves_m0 = args[0].strip() == "m0"
        # (a product may read its own sum at once: the hardware hands it on)
        self.product_reads = both(",".join(args[1:3])) if self.product else set()
        self.descriptor = registers("s", args[1]) if self.load else set()
        store = op.startswith(("global_store", "buffer_store", "flat_store", "ds_write", "scratch_store"))
        self.sum_reads = both(rest if store else ",".join(args[1:])) if vector or store else set()


def too_early(path):
    """What the last instruction of a path reads too early."""
    last, states = path[-1], 0
    for i in reversed(path[:-1]):
        if states < 2 and i.vector_writes & last.product_reads or states < 5 and i.vector_writes & last.descriptor or \
                states < 1 and i.moves_m0 and last.load or states < 7 and i.product_writes & last.sum_reads:
            return "%s, after %s" % (last.text, i.text)
        states += i.states
    return None


def violations(listing):
    """Of every function of a disassembly whose name holds product_kernel."""
    found, count = [], 0
    for name, body in re.findall(r"^[0-9a-f]+ <(\S*product_kernel\S*)>:\n(.*?)(?=^\S|\Z)", listing, re.M | re.S):
        code = [Instruction(int(a, 16), op, rest.strip()) for op, rest, a in re.findall(r"^\s+(\S+)([^\n]*?)//\s*([0-9A-F]+):", body, re.M)]
        at = {i.address: k for k, i in enumerate(code)}
        count += sum(i.product for i in code)
        for k, i in enumerate(code):
            runs = [code[max(0, k - FAR):k + 1]]
            if i.target in at:   # across the branch
                runs += [code[max(0, k - FAR):k + 1] + code[at[i.target]:at[i.target] + n] for n in range(1, FAR)]
            for run in runs:
                cut = max([n + 1 for n, j in enumerate(run[:-1]) if j.ends and j is not i], default=0)
                bad = too_early(run[cut:])
                if bad:
                    found.append("%s: %s" % (name, bad))
    return found, count


def test_products_wait_for_their_operands(tmp_path):
    if not os.path.exists(OBJDUMP):
        pytest.skip("no disassembler")
    lib = os.path.join(str(tmp_path), "lib.so")
    os.symlink(build.build(force=False), lib)
    subprocess.check_output([OBJDUMP, "--offloading", lib], cwd=str(tmp_path))
    found, count = [], 0
    for f in sorted(os.listdir(str(tmp_path))):
        if "gfx950" in f:
            bad, n = violations(subprocess.check_output([OBJDUMP, "-d", "--no-show-raw-insn", f], cwd=str(tmp_path), text=True))
            found, count = found + bad, count + n
    assert count > 1000 and not found, found[:5]


@pytest.mark.parametrize("code,bad", [
    ("v_mov_b32_e32 v4, v9|v_mfma_f32_16x16x32_bf16 a[0:3], v[4:7], v[8:11], a[0:3]", True),
    ("v_mov_b32_e32 v11, v9|s_nop 0|v_mfma_f32_16x16x32_bf16 a[0:3], v[4:7], v[8:11], a[0:3]", True),
    ("v_mov_b32_e32 v4, v9|s_nop 1|v_mfma_f32_16x16x32_bf16 a[0:3], v[4:7], v[8:11], a[0:3]", False),
    ("v_mov_b32_e32 v12, v9|v_mfma_f32_16x16x32_bf16 a[0:3], v[4:7], v[8:11], a[0:3]", False),
    ("v_readfirstlane_b32 s5, v1|s_mov_b32 m0, s2|v_add_u32_e32 v3, s1, v2|buffer_load_dwordx4 v3, s[4:7], 0 offen lds", True),
    ("v_readfirstlane_b32 s5, v1|s_nop 2|s_mov_b32 m0, s2|v_add_u32_e32 v3, s1, v2|buffer_load_dwordx4 v3, s[4:7], 0 offen lds", False),
    ("s_mov_b32 m0, s2|buffer_load_dwordx4 v3, s[4:7], 0 offen lds", True),
    ("v_mfma_f32_16x16x32_f16 a[0:3], v[4:7], v[8:11], a[0:3]|s_nop 5|v_accvgpr_read_b32 v1, a2", True),
    ("v_mfma_f32_16x16x32_f16 a[0:3], v[4:7], v[8:11], a[0:3]|s_nop 6|v_accvgpr_read_b32 v1, a2", False),
    ("v_mfma_f32_16x16x32_bf16 a[0:3], v[4:7], v[8:11], a[0:3]|s_nop 7|v_mov_b32_e32 v4, v9|s_cbranch_scc1 65532", True),   # round the loop
    ("v_mfma_f32_16x16x32_bf16 a[0:3], v[4:7], v[8:11], a[0:3]|s_nop 7|v_mov_b32_e32 v4, v9|s_nop 0|s_cbranch_scc1 65531", False)])
def test_the_check_itself(code, bad):
    lines = "".join("\t%s   // %012X:\n" % (text, 4 * k) for k, text in enumerate(code.split("|")))
    assert bool(violations("0000 <product_kernel>:\n" + lines)[0]) == bad
