"""What the device code of window prompts and of drafted tokens has to look like (no GPU
needed): the wait states behind products that assembly writes into vector registers, which no
compiler counts."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2412_05693_amd import batchmax as bmx
from test_device_code import LLVM_OBJDUMP

# Wait states until an instruction other than the next accumulation may touch a product's result:
# 19 behind one of 16 passes, 11 behind one of 8, and one more for safety.
STATES = {"v_mfma_f32_32x32x16_bf16": 20, "v_mfma_f32_16x16x32_bf16": 12}


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{kernel: [(address, instruction, address that it may go to or None)]}"""
    objdump = LLVM_OBJDUMP if os.path.exists(LLVM_OBJDUMP) else shutil.which("llvm-objdump")
    assert objdump, "llvm-objdump of the ROCm toolchain not found"
    d = tmp_path_factory.mktemp("code")
    shutil.copy(bmx.LIB_PATH, d / "lib.so")
    subprocess.run([objdump, "--offloading", "lib.so"], cwd=d, check=True, capture_output=True)
    out = {}
    for f in sorted(os.listdir(d)):
        if not f.endswith("gfx950"):
            continue
        text = subprocess.run([objdump, "-d", f], cwd=d, check=True, capture_output=True, text=True).stdout
        name, start = None, 0
        for line in text.splitlines():
            m = re.match(r"([0-9a-f]+) <(\S+)>:", line)
            if m:
                start, name = int(m.group(1), 16), m.group(2)
                if "window_prompt_kernel" in name or "nodes_kernel" in name:
                    out[name] = []
            elif name in out and re.match(r"\t[a-z].*// [0-9A-F]+:", line):
                ins, _, rest = line.partition("//")
                ins = ins.strip()
                goes = re.search(r"<\S+?(?:\+0x([0-9a-f]+))?>\s*$", rest) if ins.startswith(("s_cbranch", "s_branch")) else None
                out[name].append((int(rest.split(":")[0], 16), ins, start + int(goes.group(1) or "0", 16) if goes else None))
    return out


def vector_registers(text):
    found = set()
    for one, lo, hi in re.findall(r"\bv(?:(\d+)\b|\[(\d+):(\d+)\])", text):
        found |= {int(one)} if one else set(range(int(lo), int(hi) + 1))
    return found


def states_of(ins):
    m = re.fullmatch(r"s_nop (\d+)", ins)
    return 1 + int(m.group(1)) if m else 1


def touched_too_early(code, i, need):
    """An instruction that touches the result of the product code[i] too early, or None."""
    at = {address: j for j, (address, _, _) in enumerate(code)}
    op, operands = code[i][1].split(None, 1)
    result = vector_registers(operands.split(",")[0])
    todo, seen = [(i + 1, 0)], {}
    while todo:
        j, states = todo.pop()
        while states < need and seen.get(j, need) > states:
            seen[j] = states
            ins, goes = code[j][1], code[j][2]
            name, _, rest = ins.partition(" ")
            if name.startswith("v_mfma"):
                dest, a, b, c = [vector_registers(x) for x in re.split(r",\s*(?![^\[]*\])", rest)][:4]
                # (accumulating on, or a product of its own, is the hardware's matter)
                if result & (a | b) or (result & (dest | c) and op != name):
                    return ins
                if result & dest:
                    break                    # the next one's result: looked at by itself
            elif result & vector_registers(rest):
                return ins
            states += states_of(ins)
            if goes is not None:
                todo.append((at[goes], states))
            if name in ("s_branch", "s_endpgm"):
                break
            j += 1
    return None


def test_the_walk_finds_an_early_reader():
    code = lambda *x: [(4 * i, ins, goes) for i, (ins, goes) in enumerate(x)]        # noqa: E731
    mfma = "v_mfma_f32_16x16x32_bf16 v[0:3], v[8:11], a[0:3], 0"
    end = ("s_endpgm", None)
    early = code((mfma, None), ("s_nop 9", None), ("v_max_f32_e32 v9, v3, v9", None), end)
    late = code((mfma, None), ("s_nop 11", None), ("v_max_f32_e32 v9, v3, v9", None), end)
    jump = code((mfma, None), ("s_cbranch_scc1 2", 16), ("s_nop 15", None), end, ("v_mov_b32_e32 v3, 0", None), end)
    again = code((mfma, None), ("v_mfma_f32_16x16x32_bf16 v[0:3], v[8:11], a[0:3], v[0:3]", None), end)
    operand = code((mfma, None), ("v_mfma_f32_16x16x32_bf16 a[0:3], v[2:5], a[0:3], a[0:3]", None), end)
    assert touched_too_early(early, 0, 12) and touched_too_early(jump, 0, 12) and touched_too_early(operand, 0, 12)
    assert touched_too_early(late, 0, 12) is None and touched_too_early(again, 0, 12) is None


def test_products_in_vector_registers_are_waited_for(kernels):
    products = {n: 0 for n in kernels}
    for name, code in kernels.items():
        for i, (_, ins, _) in enumerate(code):
            op = ins.split(" ")[0]
            # (the compiler's own products have their states from it)
            if op in STATES and re.match(r"\S+ v\[\S+, v\[\S+, a\[", ins):
                products[name] += 1
                bad = touched_too_early(code, i, STATES[op])
                assert bad is None, (name, ins, bad)
    # 2 head sizes x 3 groups x split, all of whose logits are such products
    prompts = [c for n, c in products.items() if "window_prompt_kernel" in n]
    assert len(prompts) == 12 and min(prompts) >= 3 * 2 * 4
    assert sum(c > 0 for n, c in products.items() if "nodes_kernel" in n) >= 3
