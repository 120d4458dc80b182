"""What the documents and comments of a layer's operators promise beyond single results: bounds, workspaces, places, and the
rules of how the kernels' sources are written.  Tolerances as in tests/test_layer_ops.py; others are derived at their tests.
"""

import glob
import os
import re

import pytest

from paper_2506_20252_amd import build as B

gpu = pytest.mark.gpu


# ---------------------------------------------------------------------------
# On the CPU
# ---------------------------------------------------------------------------


def test_inline_assembly_names_the_m0_that_it_uses():
    """Loads into LDS take their place from m0.  The compiler keeps values of its own there, so an asm statement either takes m0
    as an operand or says that it writes it."""
    found = 0
    for path in glob.glob(os.path.join(B.CSRC, "*.h*")):
        with open(path) as f:
            text = f.read()
        for statement in re.findall(r"\basm(?:\s+volatile)?\s*\((.*?)\);", text, re.S):
            code, _, operands = statement.partition("::")
            if re.search(r"\bm0\b", code):
                assert re.search(r':\s*"(?:.*,\s*")?m0"', operands), (path, statement)
            elif "load_lds" in code:
                assert '"{m0}"(' in operands, (path, statement)
            else:
                continue
            found += 1
    assert found >= 3
