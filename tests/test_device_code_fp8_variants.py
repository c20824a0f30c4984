"""Variants of the 8-bit quantization by tiles that were compiled: those that a call reaches."""
import re

import pytest

from test_device_code import LLVM, _tool, code_objects  # noqa: F401  (a fixture)

pytestmark = pytest.mark.skipif(LLVM is None, reason="no llvm-readelf")


def test_rows_alone_take_tiles_of_weights_only(code_objects):  # noqa: F811
    """(type, 0 whole, 1 weights or 2 experts' rows, by rows, by columns, past the caches): whole matrices by rows alone have a kernel of their own, tiles of fp32 and weights
    are never read past the caches."""
    found = set()
    for path in code_objects:
        for name in re.findall(r"\.name:\s+(\S*k_fp8_tiles\S*)", _tool("llvm-readelf", "--notes", path)):
            found.add(re.search(r"k_fp8_tilesI(.)LNS\S*?TilesE(\d)ELb(\d)ELb(\d)ELb(\d)E", name).groups())
    both = [("1", "1"), ("0", "1")]
    assert found == {(t, kind, r, c, "0") for t in "ft" for kind in "012" for r, c in both} | {(t, "1", "1", "0", "0") for t in "ft"} | {("t", kind, r, c, "1") for kind in "02" for r, c in both}
