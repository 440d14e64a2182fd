"""The four-bit kernels hold no assembler statements: their MFMAs are builtins, and the compiler puts the wait states that a vector instruction needs
behind an MFMA (eight for v_mfma_f32_16x16x32_bf16) only in front of instructions that it knows, not in front of a statement that reads the result."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2504_12526_amd", "csrc")


def statements(text):
    return re.findall(r"\b(?:asm|__asm__)\b[^;\n(]*\(", re.sub(r"//[^\n]*", "", text))


def test_no_assembler_in_the_four_bit_kernels():
    files = sorted(glob.glob(os.path.join(CSRC, "mom_mx*")))
    assert len(files) == 5
    found = {os.path.basename(f): statements(open(f).read()) for f in files}
    assert not any(found.values()), found
    assert statements('x = 1;\n    asm volatile("v_max3_f32 %0, %1, %1, %2" : "=v"(r) : "v"(a), "v"(b));  // asm\n') == ["asm volatile("]
