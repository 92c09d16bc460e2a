"""Loads straight to LDS are written by hand (inline assembly that sets m0, the register of their LDS address), and the compiler cannot be told
that m0 changes: it is a reserved register to it, which a list of clobbers may not name.  So nothing that the compiler writes in
those files may use m0, by name or as some instructions do by themselves.  Looked at in the assembly of the sources as they are built."""
import os
import re
import subprocess

import pytest

from paper_2505_19586_amd import build

FILES = [f for f in build.SOURCES if "s_mov_b32 m0" in open(os.path.join(build.CSRC, f)).read()]
# m0 itself, and what reads it unnamed: relative moves, register indexing, messages, global wave sync, other loads to LDS, ordered LDS counters
USES = re.compile(r"\bm0\b|movrel|movrels|gpr_idx|sendmsg|_gws_|\blds\b|load_lds|ds_(append|consume|ordered|.*addtid)")


def uses_of_m0(assembly: str) -> list[str]:
    found, by_hand = [], False
    for line in assembly.splitlines():
        if ";;#ASMSTART" in line:
            by_hand = True
        elif ";;#ASMEND" in line:
            by_hand = False
        elif not by_hand and line.startswith("\t") and not line.lstrip().startswith((".", ";")) and USES.search(line.split(";")[0]):
            found.append(line.strip())
    return found


def test_what_counts_as_a_use():
    assert uses_of_m0("\ts_mov_b32 m0, s3\n\tds_append v1\n\tv_movrels_b32 v0, v1\n\tv_add_u32 v0, v1, v2\n\t.amdhsa_m0 m0\n") == \
        ["s_mov_b32 m0, s3", "ds_append v1", "v_movrels_b32 v0, v1"]
    assert uses_of_m0("\t;;#ASMSTART\n\ts_mov_b32 m0, s3\n\tbuffer_load_dwordx4 v1, s[0:3], 0 offen lds\n\t;;#ASMEND\n") == []


def test_the_files():
    assert set(FILES) == {"tkv_paged.hip", "tkv_prompt.hip", "tkv_quant_shared.hip"}


@pytest.mark.parametrize("name", FILES)
def test_the_compiler_uses_no_m0(name, tmp_path):
    out = tmp_path / "out.s"
    subprocess.run([build.hipcc(), *build.FLAGS, "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, "-S", "--offload-device-only",
                    os.path.join(build.CSRC, name), "-o", str(out)], check=True, capture_output=True)
    assembly = out.read_text()
    assert "s_mov_b32 m0" in assembly
    assert uses_of_m0(assembly) == []
