"""The built library's GPU code, read on the CPU (nothing is launched): on every path, a matrix product's result is
read by a vector or memory instruction only after the wait states that it takes. The hardware does not wait by itself;
the compiler puts them in, but has left a path without them where a branch right after the product skips a few
instructions that read the result too."""
import heapq
import os
import re
import subprocess

import pytest

from paper_2504_15930_amd import build, sl
from test_kernel_resources import _code_objects

STATES = 8   # v_mfma_f32_16x16x32_bf16 to a vector instruction (16x16x16 takes no more)


def _registers(operand):
    m = re.match(r"[-|]*v\[(\d+):(\d+)\]", operand)
    if m:
        return set(range(int(m[1]), int(m[2]) + 1))
    m = re.match(r"[-|]*v(\d+)\b", operand)
    return {int(m[1])} if m else set()


def early_reads(listing):
    """(product, reader) pairs of a disassembled kernel with fewer states in between on some path."""
    code = [(int(m[2], 16), m[1]) for m in re.finditer(r"^\s+(\S.*?)\s*// ([0-9A-F]+): ", listing, re.M)]
    place = {address: i for i, (address, _) in enumerate(code)}

    def after(i):
        address, text = code[i]
        op = text.split()[0]
        if op == "s_endpgm":
            return []
        follow = [i + 1] if i + 1 < len(code) else []
        if op.startswith(("s_branch", "s_cbranch")):
            offset = int(text.split()[1])
            target = place.get(address + 4 + 4 * (offset - 65536 if offset >= 32768 else offset))
            return ([] if op == "s_branch" else follow) + ([] if target is None else [target])
        return follow

    found = []
    for i, (_, text) in enumerate(code):
        if not text.startswith("v_mfma"):
            continue
        result = _registers(text.split(None, 1)[1].split(",")[0].strip())
        best, heap = {}, [(0, n) for n in after(i)]
        while heap:
            states, n = heapq.heappop(heap)
            if states >= STATES or best.get(n, STATES) <= states:
                continue
            best[n] = states
            words = code[n][1].split(None, 1)
            op, operands = words[0], [x.strip() for x in words[1].split(",")] if len(words) > 1 else []
            if op.startswith(("v_", "buffer_store", "ds_", "global_store")):
                # a product that adds to this result takes it over in the matrix unit
                read = operands[1:3] if op.startswith("v_mfma") else operands[1:] if op.startswith("v_") else operands
                if result & set().union(set(), *(_registers(x) for x in read)):
                    found.append((text, code[n][1]))
                    continue
            step = int(operands[0]) + 1 if op == "s_nop" else 4 if op.startswith("v_mfma") else 1
            for m in after(n):
                heapq.heappush(heap, (states + step, m))
    return found


def test_the_check_sees_a_branch_over_the_wait():
    """A product, a branch over the instructions that hold the wait, and the reader."""
    def listing(branch):
        return "\n".join(f"\t{text} // {4 * i:012X}: 00000000" for i, text in enumerate(
            ["v_mfma_f32_16x16x32_bf16 v[4:7], v[0:3], v[8:11], 0", branch, "s_nop 5", "v_add_f32_e32 v4, v4, v1",
             "v_add_f32_e32 v5, v5, v4", "s_endpgm"]))
    assert early_reads(listing("s_cbranch_vccnz 2"))
    assert early_reads(listing("s_nop 0"))          # 7 states
    assert not early_reads(listing("s_nop 1"))


@pytest.mark.parametrize("kernel", ["split_fp4_kernel", "prefix_fp4_kernel", "unit_fp4_kernel"])
def test_products_are_read_after_their_wait(tmp_path, kernel):
    objdump = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")
    if not os.path.exists(objdump):
        pytest.skip("no llvm-objdump under ROCm here")
    if not os.path.exists(sl.LIBRARY):
        build.build()
    seen = 0
    for i, elf in enumerate(_code_objects(open(sl.LIBRARY, "rb").read())):
        path = tmp_path / f"{i}.elf"
        path.write_bytes(elf)
        text = subprocess.run([objdump, "-d", str(path)], capture_output=True, text=True, check=True).stdout
        for name, body in re.findall(r"^[0-9a-f]+ <(\S+)>:\n(.*?)(?=^[0-9a-f]+ <|\Z)", text, re.S | re.M):
            if kernel in name:
                seen += body.count("v_mfma")
                assert not early_reads(body), name
    assert seen > 100
