"""Wait states in front of the loads straight to LDS: of the factorisation's own form, and of every such load in the library as it
was built."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2503_04424_amd import lib_path
from test_gemm_to_lds import WAIT, too_close
from test_kernel_resources import code_objects

HERE = os.path.dirname(os.path.abspath(__file__))


def tool(name, *places):
    return next((p for p in (shutil.which(name), *places) if p and os.path.exists(p)), None)


def test_registers_of_the_factorisations_loads_are_written_in_time(tmp_path):
    hipcc = tool("hipcc", "/opt/rocm/bin/hipcc")
    if not hipcc:
        pytest.skip("hipcc not available")
    out = tmp_path / "form.s"
    subprocess.run([hipcc, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                    "--cuda-device-only", "-S", "-o", str(out), os.path.join(HERE, "host", "load_to_lds_vector_base.hip")],
                   check=True, capture_output=True, timeout=600)
    lines = [l.split(";")[0].strip() for l in out.read_text().splitlines()]
    lines = [l for l in lines if l and not l.startswith(".") and not l.endswith(":")]
    assert sum(l.startswith("global_load_lds") for l in lines) >= 12
    assert any(l.startswith("v_readfirstlane") for l in lines)          # the form in question is among them
    assert not too_close(lines)


def test_every_load_to_lds_of_the_library_waits(tmp_path):
    """The code of this library's kernels (built here from source): directly in front of each such load that is written by
    hand stand the wait states that it needs behind whatever wrote its registers, or a scalar instruction that writes them, on
    any way that leads to it.  (Loads without a scalar base are the compiler's own.)"""
    objdump = tool("llvm-objdump", "/opt/rocm/llvm/bin/llvm-objdump")
    if not objdump or not os.path.exists(lib_path()):
        pytest.skip("llvm-objdump or the library not available")
    loads, short = 0, []
    for i, elf in enumerate(code_objects(lib_path())):
        path = tmp_path / f"{i}.co"
        path.write_bytes(elf)
        before = ""
        with subprocess.Popen([objdump, "-d", "--mcpu=gfx950", "--no-show-raw-insn", str(path)], stdout=subprocess.PIPE, text=True) as p:
            for line in p.stdout:
                line = line.split("//")[0].strip()
                base = re.match(r"global_load_lds\w+ v\d+, (s\[\d+:\d+\])", line)
                if base:
                    loads += 1
                    nop = re.fullmatch(r"s_nop (\d+|0x[0-9a-f]+)", before)
                    if not (nop and int(nop.group(1), 0) + 1 >= WAIT) and not before.startswith(f"s_mov_b64 {base.group(1)},"):
                        short.append((before, line))
                before = line
        assert p.returncode == 0
    assert loads > 100
    assert not short, short[:3]
