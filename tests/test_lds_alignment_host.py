"""Dynamic LDS arrays of elements smaller than a word are read and written in 16-byte pieces, so they are declared with
that alignment: without it they begin right behind the kernel's other LDS variables."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_dynamic_lds_arrays_of_small_elements_are_aligned():
    found = 0
    for path in glob.glob(os.path.join(ROOT, "paper_2605_27255_amd", "csrc", "*.h*")):
        for decl in re.findall(r"extern\s+__shared__[^;]*;", open(path).read()):
            if re.search(r"\buint(8|16)_t\b", decl):
                found += 1
                assert "__align__(16)" in decl, (path, decl)
    assert found
