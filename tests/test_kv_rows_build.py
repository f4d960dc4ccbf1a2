"""The kernel of windows on many rows, read from the gfx950 assembly of the build (no GPU needed): nothing in scratch memory."""
import os
import re

from paper_2110_08919_amd import build as lpq_build


def test_many_rows_keep_nothing_in_scratch():
    lpq_build.build()
    text = open(lpq_build.device_asm(os.path.join(lpq_build.CSRC, "kv_attend.hip"))).read()
    found = re.findall(r"\.name: +(\S*kv_rows_kernel\S*)\n(?:.*\n)*?.*\.private_segment_fixed_size: (\d+)", text)
    assert len(found) == 24
    assert [f for f in found if f[1] != "0"] == []
