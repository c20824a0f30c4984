"""The kernels of 8-bit floating point products, routing and experts' sums as they were compiled."""
import re

import pytest

from test_device_code import LLVM, _tool, code_objects  # noqa: F401  (a fixture)

pytestmark = pytest.mark.skipif(LLVM is None, reason="no llvm-readelf")


def test_kernels_keep_their_registers(code_objects):  # noqa: F811
    """No kernel keeps vector registers in memory, but for at most two between the tiles of the largest products whose rows are taken by a plan."""
    kernels, bad = 0, []
    for path in code_objects:
        for block in _tool("llvm-readelf", "--notes", path).split(".agpr_count")[1:]:
            name = re.search(r"\.name:\s+(\S+)", block)[1]
            if re.search("k_fp8_|k_route|k_plan|k_combine", name):
                kernels += 1
                spilled, scratch = (int(re.search(rf"\.{k}:\s+(\d+)", block)[1]) for k in ("vgpr_spill_count", "private_segment_fixed_size"))
                few = "k_fp8_largeILNS_2OfE1" in name
                if spilled > (2 if few else 0) or scratch > (16 if few else 0):
                    bad.append((name, spilled, scratch))
    assert kernels > 40 and not bad, bad


def test_no_scratch_between_the_products_of_the_largest_tiles(code_objects):  # noqa: F811
    """Spilled registers would count among the requests that these loops wait for by number."""
    loops = 0
    for path in code_objects:
        text = _tool("llvm-objdump", "-d", "--mcpu=gfx950", path)
        for body in re.split(r"\n\n", text):
            if "k_fp8_large" not in body.split("\n", 1)[0] and "k_fp8_large" not in body[:200]:
                continue
            lines = [l.split()[0] for l in body.split("\n") if l.startswith("\t")]
            at = [i for i, op in enumerate(lines) if op.startswith("v_mfma")]
            for a, b in zip(at, at[1:]):
                if b - a < 60:
                    assert not any(op.startswith("scratch") for op in lines[a:b])
            loops += len(at) >= 128
    assert loops >= 6
