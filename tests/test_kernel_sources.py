"""Inline assembly of the kernels says what it writes."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2509_24859_amd", "csrc")


def _statements():
    """(file, template, what follows the template) of every asm statement."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        if not path.endswith((".hip", ".h")):
            continue
        with open(path) as f:
            text = f.read()
        for m in re.finditer(r"\basm\b\s*(?:volatile)?\s*\(((?:\s*\"(?:[^\"\\]|\\.)*\")*)([^;]*)\);", text):
            yield os.path.basename(path), m.group(1), m.group(2)


def test_m0_is_named_where_it_is_written():
    """Registers that a template names by themselves are no operands: the compiler knows of them by the list of clobbers."""
    seen = 0
    for path, template, rest in _statements():
        if re.search(r"\b(?:s_mov_b32|s_add_u32|s_lshl_b32|v_readfirstlane_b32)\s+m0\b", template):
            seen += 1
            clobbers = rest.rsplit(":", 1)[-1]
            assert '"m0"' in clobbers, (path, template)
    assert seen >= 1
