"""How warps come to a load of the accumulator, found in the sources (no GPU needed).

tcgen05.ld.sync.aligned is executed by a whole warp at once and writes the registers of all its
lanes; these hold nothing before tcgen05.wait::ld.  The warps that load come from barriers which
their lanes poll one by one (and may give up one by one) and from branches of single lanes."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2608_14563_gb300", "csrc")


def _sources():
    for name in sorted(os.listdir(CSRC)):
        if name.endswith((".cu", ".cuh")):
            with open(os.path.join(CSRC, name)) as f:
                yield name, re.sub(r"//[^\n]*", "", f.read())


def _block(text, start):
    """The braced block that begins at the first '{' from `start` on."""
    i = text.index("{", start)
    depth, j = 1, i + 1
    while depth:
        depth += {"{": 1, "}": -1}.get(text[j], 0)
        j += 1
    return text[i:j]


def test_a_load_brings_the_warp_together_and_waits_in_one_statement():
    loads = 0
    for name, text in _sources():
        for m in re.finditer(r"tcgen05\.ld\.", text):
            loads += 1
            fn = text.rindex("__device__", 0, m.start())
            before = text[text.index("{", fn):m.start()]
            assert "__syncwarp();" in before, name
            statement = text[m.start():text.index(";\n", text.index("]", text.index(": \"=r\"", m.start())))]
            assert "tcgen05.wait::ld.sync.aligned" in statement, name
    assert loads >= 1


def test_a_warp_gives_up_on_an_accumulator_as_one():
    """Every wait for an accumulator is decided by a vote of the warp: a lane that goes on alone
    would reach warp-wide instructions that the others never do."""
    waits = 0
    for name, text in _sources():
        for m in re.finditer(r"mbar_wait\w*\(tfull_bar\(", text):
            waits += 1
            line = text[text.rindex("\n", 0, m.start()):m.start()]
            assert re.search(r"const bool in_time = $", line), (name, line)
            after = text[m.end():m.end() + 160]
            assert re.search(r"if \(!__all_sync\(0xffffffffu, in_time\)\) return false;", after), name
    assert waits >= 4


def test_a_warp_reads_the_abort_flag_as_one():
    """Outside the waits themselves (one lane's, or voted on by their callers) the flag, which any
    warp of the block may raise at any time, is read through a vote."""
    reads = 0
    for name, text in _sources():
        if not name.endswith("gemm.cuh") and not name.endswith("gemm_pair.cuh"):
            continue
        for m in re.finditer(r"\*(?:g\.)?abort_flag\b(?! = )", text):
            line = text[text.rindex("\n", 0, m.start()) + 1:text.index("\n", m.end())]
            if "volatile int*" in line:
                continue  # its declaration
            reads += 1
            in_wait = re.search(r"if \(\*g\.abort_flag\) return false;", line)
            assert in_wait or "__all_sync(0xffffffffu," in line, (name, line)
    assert reads >= 3
