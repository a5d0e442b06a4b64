"""Inline assembly in the kernels' sources, without a GPU.

A matrix instruction's result may be read only so many clocks later.  The compiler keeps that distance for instructions that it
chose itself, not for the operands of an assembly block: a vector instruction written in assembly that reads accumulators would take stale
ones as soon as another schedule brings the two close together, and nothing would say so."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_16603_amd", "csrc")
ASM = re.compile(r'\basm\s*(?:volatile\s*)?\(\s*((?:"(?:[^"\\]|\\.)*"\s*)+)')


def _instructions():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.h"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        for m in ASM.finditer(text):
            template = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', m.group(1)))
            for line in re.split(r"\\n(?:\\t)?|;", template):
                if line.strip():
                    yield os.path.basename(path), line.split()[0], m.start(), text


def test_only_matrix_instructions_read_vector_registers_in_assembly():
    found = list(_instructions())
    assert any(op.startswith("v_mfma") for _, op, _, _ in found)          # (the pattern does find them)
    assert [(f, op) for f, op, _, _ in found if op.startswith("v_") and not op.startswith("v_mfma")] == []


def test_matrix_instructions_in_assembly_are_followed_by_a_wait():
    """... of 32 clocks in the same file, before its epilogue reads what they wrote."""
    for name, op, at, text in _instructions():
        if op.startswith("v_mfma"):
            assert re.search(r's_nop 15\\n\\ts_nop 15', text[at:]), name
