"""A load straight to LDS reads its base from scalar registers and its place from m0.  Where a vector instruction
(v_readfirstlane) has written one of these, the hardware wants five wait states before a memory instruction reads it; the
compiler keeps them in front of its own instructions, but it does not look into inline assembly."""
import os
import re
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
WAIT = 5


def scalars(operand):
    pair = re.fullmatch(r"s\[(\d+):(\d+)\]", operand)
    if pair:
        return {f"s{i}" for i in range(int(pair.group(1)), int(pair.group(2)) + 1)}
    return {operand} if re.fullmatch(r"s\d+|m0", operand) else set()


def too_close(lines):
    """(wait states, writer, load) of every load to LDS that reads a register too soon behind a vector instruction's write."""
    found = []
    for i, load in enumerate(lines):
        if not load.startswith("global_load_lds"):
            continue
        needs = set().union(*(scalars(o.strip().split()[0]) for o in load.split(None, 1)[1].split(","))) | {"m0"}
        states, j = 0, i - 1
        while j >= 0 and states < WAIT:
            nop = re.fullmatch(r"s_nop (\d+)", lines[j])
            if not nop and lines[j].startswith("v_") and scalars(lines[j].split(None, 1)[1].split(",")[0].strip()) & needs:
                found.append((states, lines[j], load))
            states += int(nop.group(1)) + 1 if nop else 1
            j -= 1
    return found


def test_the_check_sees_what_it_looks_for():
    writer, load = "v_readfirstlane_b32 s5, v1", "global_load_lds_dwordx4 v2, s[4:5]"
    assert too_close([writer, "s_nop 0", load]) and too_close([writer, "v_mov_b32 v3, v4", "s_nop 2", load])
    assert not too_close([writer, "s_nop 4", load]) and not too_close(["s_mov_b32 s5, s6", "s_nop 0", load])
    assert too_close(["v_readfirstlane_b32 m0, v1", "s_nop 3", load])


def test_registers_of_a_load_to_lds_are_written_in_time(tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    out = tmp_path / "form.s"
    subprocess.run([hipcc, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                    "--cuda-device-only", "-S", "-o", str(out), os.path.join(HERE, "host", "gemm_to_lds_form.hip")],
                   check=True, capture_output=True, timeout=600)
    lines = [l.split(";")[0].strip() for l in out.read_text().splitlines()]
    lines = [l for l in lines if l and not l.startswith(".") and not l.endswith(":")]
    assert sum(l.startswith("global_load_lds") for l in lines) >= 3
    assert any(l.startswith("v_readfirstlane") for l in lines)          # the form in question is among them
    assert not too_close(lines)
