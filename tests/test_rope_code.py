"""What the built rotary kernels write with: whole stores of 8 and 16 bytes."""
import os
import re

import pytest

from tests.test_product_waits import OBJDUMP, disassembly, functions


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler for gfx950")
def test_pieces_are_stored_whole(tmp_path):
    seen = 0
    for code in disassembly(tmp_path):
        for name, instructions in functions(code):
            if "rope_kernel" not in name:
                continue
            seen += 1
            stores = [i.text for i in instructions if re.match(r"(global|flat)_store", i.op)]
            # bf16 halves of an odd multiple of 8 entries go in pieces of 8 bytes, all others of 16
            size = "dwordx2" if "Li4E" in name and "bf16" in name else "dwordx4"
            assert stores and all(s.split()[0].endswith("store_" + size) for s in stores), (name, stores)
    assert seen == 5
