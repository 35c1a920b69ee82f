"""Inline assembly that writes a register of its own choice tells the compiler so."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_13692_amd", "csrc")


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*"))), ids=os.path.basename)
def test_m0_is_named_where_it_is_written(path):
    with open(path) as f:
        statements = re.findall(r"\basm\b[^;]*;", f.read())
    for s in statements:
        code = s.split(":")[0]
        restored = "s_mov_b32 %0, m0" in code and code.rstrip().endswith('s_mov_b32 m0, %0"')
        if re.search(r"\bm0\s*,", code) and not restored:
            assert '"m0"' in s.rsplit(":", 1)[1], s
