"""What the 8-bit products' source may not hold (CPU only): an instruction in inline assembly next to matrix products, whose results arrive
many cycles later."""
import os
import re

import paper_2606_01007_amd as tacg


def test_no_instruction_in_inline_assembly_next_to_the_matrix_products():
    text = open(os.path.join(os.path.dirname(tacg.__file__), "csrc", "i8.hip")).read()
    assert "mfma" in text and not re.search(r"\basm\b", text)
