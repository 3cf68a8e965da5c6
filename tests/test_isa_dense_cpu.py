"""On the gfx950 assembly of tile_attn.hip, compiled here: M0, which the inline
global-to-LDS copies name as clobbered although the compiler reserves it, is
written by those copies alone, each write directly followed by its load, and
no other instruction touches it."""
import os
import re
import subprocess

import pytest

from paper_2512_00722_amd import build as B

SOURCE = next(s for s in B.sources() if os.path.basename(s) == "tile_attn.hip")

pytestmark = pytest.mark.skipif(not os.path.exists(B.HIPCC), reason="hipcc not found")


def test_m0_only_in_the_global_to_lds_copies(tmp_path):
    out = tmp_path / "tile_attn.s"
    r = subprocess.run([B.HIPCC, *B.flags_for(SOURCE), "-x", "hip", "--cuda-device-only", "-S",
                        "-o", str(out), SOURCE], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    lines = [x.split(";")[0].strip() for x in out.read_text().splitlines()]
    ins = [x for x in lines if x and not x.startswith(".") and not x.endswith(":")]
    uses = [j for j, i in enumerate(ins) if re.search(r"\bm0\b", i)]
    assert uses
    for j in uses:
        assert re.match(r"^s_mov_b32 m0, s\d+$", ins[j]), ins[j]
        assert ins[j + 1].startswith("global_load_lds_dwordx4"), (ins[j], ins[j + 1])
    assert [j for j, i in enumerate(ins) if i.startswith("global_load_lds")] == [j + 1 for j in uses]
