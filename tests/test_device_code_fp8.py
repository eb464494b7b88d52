"""CPU-only checks of the 8-bit kernels' compiled code: what their inline assembly counts on and no result shows every time."""
import os
import re
import subprocess

import pytest

from test_device_code import LLVM, code_object, registers, unwaited_loads


def disassembly(source, tmp_path):
    return subprocess.run([os.path.join(LLVM, "llvm-objdump"), "-d", code_object(source, tmp_path)], capture_output=True, text=True, check=True).stdout


def copies_of_results(asm, wait=11):
    """Kernels in which an accumulator is read or moved fewer than `wait` wait states after a matrix instruction whose latency the compiler does not know
    (one that stands in inline assembly keeps its accumulators in the a registers)."""
    found, kernel, since = [], "", None
    for line in asm.splitlines():
        head = re.match(r"^[0-9a-f]+ <(.*)>:", line)
        if head:
            kernel, since = head.group(1), None
            continue
        ins = line.split("//")[0].strip()
        if not ins:
            continue
        if ins.startswith("v_mfma_scale"):
            since = 0
        elif since is not None:
            if ins.startswith("v_accvgpr") and since < wait:
                found.append(kernel)
            since += int(ins.split()[1]) + 1 if ins.startswith("s_nop") else 1
    return found


def test_copies_are_found():
    text = "0000 <k>:\n v_mfma_scale_f32_16x16x128_f8f6f4 a[0:3], v[0:7], v[8:15], a[0:3], v1, v2\n s_nop {}\n v_accvgpr_read_b32 v3, a0\n"
    assert copies_of_results(text.format(9)) == ["k"] and copies_of_results(text.format(10)) == []


def test_direct_loads_wait_for_their_address(tmp_path):
    loads, unwaited = unwaited_loads(disassembly("fp8_gemm_wide", tmp_path))
    assert loads > 0 and not unwaited


def test_accumulators_stay_where_they_are(tmp_path):
    asm = disassembly("fp8_gemm_wide", tmp_path)
    assert asm.count("v_mfma_scale") > 0 and not copies_of_results(asm)


@pytest.mark.parametrize("source", ["fp8_gemm", "fp8_gemm_thin", "fp8_gemm_wide", "fp8_quantize", "moe"])
def test_no_spills(source, tmp_path):
    # (the counted waits of the 256-row tiles know of no loads and stores but their own)
    assert all(spilled == 0 for _, spilled in registers(source, tmp_path).values())
    assert "scratch_" not in disassembly(source, tmp_path)


def test_outputs_leave_in_whole_pieces(tmp_path):
    # the next output's first K tile is waited for by the number of stores behind its loads
    asm = disassembly("fp8_gemm_wide", tmp_path)
    assert asm.count("global_store_dwordx4") > 0 and asm.count("global_store_dwordx3") == 0 and asm.count("global_store_dwordx2") == 0
