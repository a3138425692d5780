"""The copies from memory to the LDS are inline assembly: the compiler does not look into it for the distances that the hardware asks
for.  Built here with the products that use them, and counted in the assembly: between a vector instruction's write of a scalar
register and a copy that reads it as part of its descriptor five instructions, between the write of m0 and the copy one; and no wait for the copies
but the kernel's own."""
import os
import re
import subprocess

import pytest

import __graft_entry__ as entry

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include <hip/hip_runtime.h>
#include <algorithm>
#include "slimdp_gemm.h"
using namespace slimdp;
template __global__ void slimdp::k_gemm_tiles<__bf16, %s, %s, %d, %d, %d, 2, 2, %d, true>(GemmArgs);
"""


def registers(text):
    out = set()
    for m in re.finditer(r"\bs\[(\d+):(\d+)\]|\bs(\d+)\b", text):
        out |= {int(m.group(3))} if m.group(3) else set(range(int(m.group(1)), int(m.group(2)) + 1))
    return out


@pytest.mark.parametrize("a_rows,b_rows,epilogue,tile,blocks", [("false", "false", 0, 256, 1), ("false", "true", 1, 128, 2), ("true", "true", 2, 256, 1)])
def test_distances_in_front_of_copies(tmp_path, a_rows, b_rows, epilogue, tile, blocks):
    src = tmp_path / "tiles.hip"
    src.write_text(SOURCE % (a_rows, b_rows, epilogue, tile, tile, blocks))
    flags = [f for f in entry.HIPCC_FLAGS if f not in ("-shared", "-fPIC", "-Wall")]
    asm = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "--offload-device-only", "-S", "-o", "-", str(src)],
                         check=True, capture_output=True, text=True).stdout
    at, written, m0, copies, waits, products = 0, {}, -100, 0, 0, 0
    for line in asm.splitlines():
        text = line.split(";")[0].strip()
        if not re.match(r"^([sv]_|global_|buffer_|ds_|flat_)", text):
            continue
        op, _, operands = text.partition(" ")
        if op == "s_nop":
            at += int(operands, 0) + 1
            continue
        at += 1
        if op.startswith("v_mfma"):
            products += 1
        if op == "buffer_load_dwordx4" and operands.endswith("lds"):
            copies += 1
            assert at - m0 - 1 >= 1, text
            for reg in registers(operands.split(",", 1)[1]):
                assert at - written.get(reg, -100) - 1 >= 5, (text, reg)
        elif op.startswith("v_"):
            for reg in registers(operands.split(",")[0]):
                written[reg] = at
        elif op.startswith("s_") and not op.startswith(("s_waitcnt", "s_barrier", "s_cbranch", "s_branch", "s_cmp")):
            dest = operands.split(",")[0].strip()
            if dest == "m0":
                m0 = at
            for reg in registers(dest):
                written.pop(reg, None)
    assert copies >= 2 * tile // 64 and products >= 64 * (tile // 128) ** 2 // 4, (copies, products)
    # inside the loop (between the first and the last matrix instruction) the copies are waited for in one place
    body = asm[asm.index("v_mfma"):asm.rindex("v_mfma")]
    assert len(re.findall(r"vmcnt\(\d+\)", body)) == 1, re.findall(r"s_waitcnt[^\n]*vmcnt[^\n]*", body)
