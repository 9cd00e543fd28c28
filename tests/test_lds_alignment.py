"""Byte arrays in LDS that kernels clear by 16-byte stores and set by 32-bit atomics are declared with the alignment that these need: without it their
place is the compiler's choice, and a kernel right by chance."""
import glob
import os
import re

from conftest import ROOT


def test_byte_arrays_are_aligned():
    found = 0
    for path in sorted(glob.glob(os.path.join(ROOT, "paper_2506_03206_amd", "csrc", "*.h*"))):
        with open(path) as fh:
            for line in fh:
                if re.search(r"__shared__.*\buint8_t\s+\w+\s*\[", line):
                    found += 1
                    assert "aligned(16)" in line, (os.path.basename(path), line.strip())
    assert found
