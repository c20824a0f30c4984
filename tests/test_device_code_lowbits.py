"""The few-bit kernels as they were compiled."""
import re

import pytest

from test_device_code import LLVM, _tool, code_objects  # noqa: F401  (a fixture)

pytestmark = pytest.mark.skipif(LLVM is None, reason="no llvm-readelf")


def test_kernels_keep_their_registers(code_objects):  # noqa: F811
    kernels, bad = 0, []
    for path in code_objects:
        for block in _tool("llvm-readelf", "--notes", path).split(".agpr_count")[1:]:
            name = re.search(r"\.name:\s+(\S+)", block)[1]
            if re.search("k_mx4_|k_ckpt8_", name):
                kernels += 1
                if int(re.search(r"\.vgpr_spill_count:\s+(\d+)", block)[1]) or int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", block)[1]):
                    bad.append(name)
    assert kernels > 20 and not bad, bad


def test_written_out_reads_wait_where_they_stand(code_objects):  # noqa: F811
    """The transposing reads are inline assembly: behind the last of each group stands its wait, before anything else."""
    groups = 0
    for path in code_objects:
        lines = [l for l in _tool("llvm-objdump", "-d", "--mcpu=gfx950", path).splitlines() if re.match(r"\t[a-z]", l)]
        for i, l in enumerate(lines[:-1]):
            if "ds_read_b64_tr_b16" in l and "ds_read_b64_tr_b16" not in lines[i + 1]:
                groups += 1
                assert re.search(r"s_waitcnt lgkmcnt\(0\)", lines[i + 1]), (l, lines[i + 1])
    assert groups >= 16
