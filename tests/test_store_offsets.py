"""Buffer stores in the kernels' sources (no GPU needed)."""

import glob
import os
import re

from paper_2607_01408_amd import build
from tests.test_lds_limit import arguments


def test_wide_buffer_stores_have_no_scalar_offset():
    """The compiler keeps the next instruction off a wide store's data registers only where the store's scalar offset is
    zero; with another the first of them may be overwritten before it is read."""
    stores = 0
    for path in sorted(glob.glob(os.path.join(build.CSRC, "*.hip")) + glob.glob(os.path.join(build.CSRC, "*.h"))):
        text = open(path).read()
        for found in re.finditer(r"__builtin_amdgcn_raw_(?:ptr_)?buffer_store_b(?:96|128)\(", text):
            stores += 1
            assert arguments(text, found.end())[3] == "0", f"{os.path.basename(path)}:{text.count(chr(10), 0, found.start()) + 1}"
        assert not re.search(r"buffer_store_dwordx[34]", text), path
    assert stores
