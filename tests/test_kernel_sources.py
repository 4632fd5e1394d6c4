"""What the compiler is told about inline assembly in the kernels."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_23635_amd", "csrc")


def statements():
    """(file, text) of every inline assembly statement, comments taken out."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        with open(path) as f:
            src = re.sub(r"//[^\n]*", "", f.read())
        for m in re.finditer(r"\basm\b(?:\s+volatile)?\s*\(", src):
            depth, end = 1, m.end()
            while depth:
                depth += {"(": 1, ")": -1}.get(src[end], 0)
                end += 1
            yield os.path.basename(path), src[m.start():end]


def test_assembly_declares_what_it_changes():
    """An instruction that writes m0 names it as changed, and one that writes LDS names memory."""
    found = 0
    for name, text in statements():
        strings = re.findall(r'"((?:[^"\\]|\\.)*)"', text)
        code, clobbers = strings[0], strings[1:]
        if re.search(r"_b32 m0,", code):
            assert "m0" in clobbers, (name, text)
            found += 1
        if re.search(r"\blds\b", code) or re.search(r"\bds_write", code):
            assert "memory" in clobbers, (name, text)
            found += 1
    assert found
