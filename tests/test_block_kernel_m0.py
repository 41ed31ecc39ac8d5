"""M0 in the products on the matrix cores, from the instructions of the library that was built here. Their asm blocks set M0 in front of every
direct-to-LDS load and cannot declare it (the compiler reserves it, and warns of a clobber): so nothing else in these kernels may use it."""
import os
import re
import subprocess

import pytest

from test_kernel_resources import LIB, _code_objects, _metadata

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
# instructions that read M0 without naming it, the direct-to-LDS loads aside
IMPLICIT = re.compile(r"movrel|set_gpr_idx|s_sendmsg|ds_gws|v_interp|ds_ordered|addtid")


@pytest.fixture(scope="module")
def gemm_code(tmp_path_factory):
    blob = open(LIB, "rb").read()
    starts = list(_code_objects(blob)) + [len(blob)]
    found = []
    for at, end in zip(starts, starts[1:]):
        if any("linear_gemm_kernel" in k[".name"] for doc in _metadata(blob, at) for k in doc["amdhsa.kernels"]):
            path = tmp_path_factory.mktemp("code") / "object.elf"
            path.write_bytes(blob[at:end])
            found.append(subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(path)], capture_output=True, text=True, check=True).stdout)
    return found


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump")
def test_only_the_loads_of_the_asm_blocks_use_m0(gemm_code):
    assert len(gemm_code) == 5                       # linear_gemm_<tile>_<steps>
    for text in gemm_code:
        lines = [line.split("//")[0].strip() for line in text.splitlines()]
        sets = [k for k, line in enumerate(lines) if re.search(r"\bm0\b", line)]
        loads = [k for k, line in enumerate(lines) if re.match(r"(buffer|global)_load\w* .*\blds$|global_load_lds", line)]
        assert loads and all(re.match(r"s_mov_b32 m0, s\d+$", lines[k]) for k in sets), [lines[k] for k in sets if not re.match(r"s_mov_b32 m0, s\d+$", lines[k])][:5]
        # one load for every setting, an instruction between
        assert len(sets) == len(loads) and all(2 <= b - a <= 4 for a, b in zip(sets, loads)), [b - a for a, b in zip(sets, loads)][:10]
        assert not any(IMPLICIT.search(line) for line in lines)
