"""Assembly in the kernels' sources says which special registers it overwrites (no GPU needed)."""
import glob
import os
import re

from paper_2006_02924_amd import build as builder

CSRC = builder.CSRC


def statements():
    """(file, instructions, what is named as overwritten) of every assembly statement."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        with open(path) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        for m in re.finditer(r"asm\s+volatile\s*\((.*?)\)\s*;", text, re.S):
            code, clobbers = m.group(1), ""
            parts = code.split(":")
            if len(parts) >= 4:
                clobbers = parts[-1]
            yield os.path.basename(path), parts[0], clobbers


def test_m0_is_named_where_it_is_written():
    found = [(name, code, clobbers) for name, code, clobbers in statements() if re.search(r"\b[sv]_\w+\s+m0\s*,", code)]
    assert found, "there is assembly that writes m0"
    for name, code, clobbers in found:
        assert '"m0"' in clobbers, (name, code)
