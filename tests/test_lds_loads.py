"""Loads straight to LDS are written by hand (inline assembly that sets m0, the register of their LDS address), and the compiler cannot be told
that m0 changes: it is a reserved register to it, which a list of clobbers may not name.  So nothing that the compiler writes in
those files may use m0, by name or as some instructions do by themselves.  Nor does the compiler know which waits such a load needs: a
scalar register that the vector unit has written (a descriptor by way of readfirstlane) is there for a memory instruction five wait
states later (the compiler writes s_nop 4 in front of its own).  Both are looked at in the assembly of the sources as they are built."""
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


@pytest.fixture(scope="module")
def assembly_of(tmp_path_factory):
    made = {}

    def of(name):
        if name not in made:
            out = tmp_path_factory.mktemp("assembly") / "out.s"
            subprocess.run([build.hipcc(), *build.FLAGS, "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, "-S",
                            "--offload-device-only", os.path.join(build.CSRC, name), "-o", str(out)], check=True, capture_output=True)
            made[name] = out.read_text()
        return made[name]

    return of


@pytest.mark.parametrize("name", FILES)
def test_the_compiler_uses_no_m0(name, assembly_of):
    assembly = assembly_of(name)
    assert "s_mov_b32 m0" in assembly
    assert uses_of_m0(assembly) == []


def _scalars(operand: str) -> set:
    found = {"vcc"} if "vcc" in operand else set()
    for low, high, one in re.findall(r"\bs\[(\d+):(\d+)\]|\bs(\d+)\b", operand):
        found |= {int(one)} if one else set(range(int(low), int(high) + 1))
    return found


def _written_by_vector_unit(line: str) -> set:
    op, _, rest = line.partition(" ")
    if not op.startswith("v_"):
        return set()
    operands = re.sub(r"\[(\d+):(\d+)\]", r"[\1;\2]", rest).split(",")       # (the first, and the carry's)
    dst = operands[:2] if re.search(r"_co_|addc|subb|div_scale|mad_[ui]64", op) else operands[:1]
    return _scalars(",".join(dst).replace(";", ":"))


def waits_missing(assembly: str) -> list[str]:
    """Hand-written loads that read a scalar register fewer than five wait states after the vector unit wrote it."""
    found, by_hand, before = [], False, []                                   # before: (instruction, its wait states)
    for line in assembly.splitlines():
        by_hand = ";;#ASMSTART" in line or (by_hand and ";;#ASMEND" not in line)
        line = line.split(";")[0].strip().replace("\t", " ")
        if not line or line.startswith(".") or line.endswith(":"):
            continue
        if by_hand and re.match(r"(buffer|global|flat|scratch)_", line):
            states = 0
            for other, n in reversed(before):
                if states >= 5:
                    break
                if _written_by_vector_unit(other) & _scalars(line.partition(" ")[2]):
                    found.append(f"{other} -> {line}")
                states += n
        before = before[-8:] + [(line, int(line.split()[1], 0) + 1 if line.startswith("s_nop") else 1)]
    return found


def test_what_counts_as_a_missing_wait():
    load = "\t;;#ASMSTART\n\ts_mov_b32 m0, s6\n\ts_nop {}\n\tbuffer_load_dwordx4 v81, s[16:19], 0 offen lds\n\t;;#ASMEND\n"
    for write in ("v_readfirstlane_b32 s18, v18", "v_readlane_b32 s16, v18, 0", "v_sub_co_u32_e64 v18, s[18:19], s6, 1", "v_cmp_eq_u32_e64 s[16:17], 0, v1"):
        assert len(waits_missing(f"\t{write}\n" + load.format(0))) == 1 and not waits_missing(f"\t{write}\n" + load.format(3))
        assert not waits_missing(f"\t{write}\n" + 3 * "\ts_and_b32 s1, s2, s3\n" + load.format(0))
    assert not waits_missing("\tv_cndmask_b32_e64 v18, v18, 0, s[16:17]\n" + load.format(0))
    assert not waits_missing("\ts_and_b32 s17, s17, 0xffff\n" + load.format(0))


@pytest.mark.parametrize("name", FILES)
def test_no_wait_is_missing(name, assembly_of):
    assert waits_missing(assembly_of(name)) == []
