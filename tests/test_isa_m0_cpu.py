"""On the gfx950 machine code of the kernels that copy from global memory to LDS,
compiled and taken apart here: between each write of M0 and the copy that reads it
stands one wait state (s_nop 0), which the instruction set asks for and the compiler
adds to its own copies, but not inside inline assembly."""
import os
import subprocess

import pytest

from paper_2512_00722_amd import build as B

OBJDUMP = os.path.join(os.path.dirname(os.path.dirname(B.HIPCC)), "llvm", "bin", "llvm-objdump")

pytestmark = pytest.mark.skipif(not (os.path.exists(B.HIPCC) and os.path.exists(OBJDUMP)),
                                reason="hipcc or llvm-objdump not found")


@pytest.mark.parametrize("name", ["mla.hip", "tile_attn.hip"])
def test_a_wait_state_stands_between_m0_and_the_copy(tmp_path, name):
    src = next(s for s in B.sources() if os.path.basename(s) == name)
    obj = tmp_path / "device.o"
    r = subprocess.run([B.HIPCC, *B.flags_for(src), "-x", "hip", "--cuda-device-only",
                        "--no-gpu-bundle-output", "-c", "-o", str(obj), src],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([OBJDUMP, "-d", str(obj)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    lines = [x.split("//")[0].strip() for x in r.stdout.splitlines()]
    copies = [j for j, x in enumerate(lines) if x.startswith("global_load_lds")]
    assert copies
    for j in copies:
        assert lines[j - 2].startswith("s_mov_b32 m0,"), lines[j - 2:j + 1]
        assert lines[j - 1] == "s_nop 0", lines[j - 2:j + 1]
