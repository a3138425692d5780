"""The distances in front of the copies from memory to the LDS in every kernel that makes them (both types, three layouts, two tiles), in the order
of the file and over every jump back: the instructions that end a loop's body come before those that begin it."""
import os
import re
import subprocess

import pytest

import __graft_entry__ as entry
from test_copy_to_lds_cpu import registers

SOURCE = """
#include <hip/hip_runtime.h>
#include <algorithm>
#include "slimdp_gemm.h"
using namespace slimdp;
template __global__ void slimdp::k_gemm_tiles<%(type)s, %(layout)s, 256, 256, 2, 2, 1, true>(GemmArgs);
template __global__ void slimdp::k_gemm_tiles<%(type)s, %(layout)s, 128, 128, 2, 2, 2, true>(GemmArgs);
"""
REACH = 40          # instructions behind which no distance matters any more


def functions(asm):
    """Instructions of every kernel with the places that its labels mark."""
    out, name = {}, None
    for line in asm.splitlines():
        text = line.split(";")[0].strip()
        m = re.match(r"^(_Z\w+):$", text)
        if m:
            name = m.group(1)
            out[name] = ([], {})
            continue
        if name is None:
            continue
        if text.startswith(".Lfunc_end"):
            name = None
            continue
        m = re.match(r"^(\.L\w+):$", text)
        if m:
            out[name][1][m.group(1)] = len(out[name][0])
        elif re.match(r"^([sv]_|global_|buffer_|ds_|flat_|scratch_)", text):
            out[name][0].append(text)
    return out


def is_copy(text):
    return text.startswith("buffer_load_dwordx4") and text.endswith("lds")


def check(code):
    at, written, m0, copies = 0, {}, -100, 0
    for text in code:
        op, _, operands = text.partition(" ")
        if op == "s_nop":
            at += int(operands, 0) + 1
            continue
        at += 1
        if is_copy(text):
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
    return copies


@pytest.mark.parametrize("type_", ["__bf16", "_Float16"])
@pytest.mark.parametrize("layout", ["false, false, 0", "false, true, 1", "true, true, 2"])
def test_distances_in_front_of_copies_in_every_kernel(tmp_path, type_, layout):
    src = tmp_path / "tiles.hip"
    src.write_text(SOURCE % {"type": type_, "layout": layout})
    flags = [f for f in entry.HIPCC_FLAGS if f not in ("-shared", "-fPIC", "-Wall")]
    asm = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "--offload-device-only", "-S", "-o", "-", str(src)],
                         check=True, capture_output=True, text=True).stdout
    kernels = {n: v for n, v in functions(asm).items() if any(is_copy(t) for t in v[0])}
    assert len(kernels) == 2
    for code, labels in kernels.values():
        assert check(code) >= 16
        around = 0
        for i, text in enumerate(code):
            m = re.match(r"^s_c?branch\w*\s+(\.L\w+)$", text)
            if m and labels.get(m.group(1), i + 1) <= i:
                j = labels[m.group(1)]
                around += check(code[max(0, i - REACH):i + 1] + code[j:j + REACH]) > 0 or any(is_copy(t) for t in code[j:i])
        assert around, "no loop with copies in it"


def test_the_check_sees_a_distance_that_is_too_short():
    good = ["s_mov_b32 m0, s3", "s_nop 0", "buffer_load_dwordx4 v1, s[8:11], 0 offen lds"]
    late = "v_readfirstlane_b32 s9, v3"
    assert check([late] + ["v_mov_b32_e32 v9, v8"] * 3 + good) == 1
    for bad in ([late] + good, [late] + ["v_mov_b32_e32 v9, v8"] * 2 + good, [good[0], good[2]]):
        with pytest.raises(AssertionError):
            check(bad)
