"""What the stage operators' sources leave to the compiler."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2311_05827_amd", "csrc")


def inline_assembly(text):
    """The strings of every asm statement."""
    for m in re.finditer(r"\basm\b\s*(?:volatile)?\s*\(((?:\s*\"(?:[^\"\\]|\\.)*\")+)", text):
        yield "".join(re.findall(r"\"((?:[^\"\\]|\\.)*)\"", m.group(1)))


def test_the_scan_sees_statements():
    text = 'asm volatile("s_nop 1\\n\\tv_mfma_x %0"\n : "+a"(s)); asm("" : "+v"(v));'
    assert list(inline_assembly(text)) == ["s_nop 1\\n\\tv_mfma_x %0", ""]


def test_no_matrix_instruction_in_inline_assembly():
    """A matrix instruction writes its results many cycles after it was issued.  The compiler keeps that distance for the ones it knows; in
    inline assembly it may move a result on at once."""
    files = sorted(glob.glob(os.path.join(CSRC, "*.h*")))
    assert any(f.endswith("matmul.hip") for f in files)
    found = [(os.path.basename(f), s) for f in files for s in inline_assembly(open(f).read()) if "mfma" in s]
    assert found == []
