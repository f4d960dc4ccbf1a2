"""The built key-value cache kernels, read from the gfx950 assembly of the build (no GPU needed): no read of a matrix result sooner
than the wait states it needs, on every fall-through path, and nothing of the attention kernels in scratch memory."""
import os
import re

import pytest

import test_kernel_schedule as schedule
from paper_2110_08919_amd import build as lpq_build

NEED = 9      # issue slots the compiler leaves between a 16x16 product and a read of it that follow each other


@pytest.fixture(scope="module")
def asm():
    lpq_build.build()
    return {s: lpq_build.device_asm(os.path.join(lpq_build.CSRC, s)) for s in ("kv_attend.hip", "kv_select.hip")}


@pytest.mark.parametrize("source", ["kv_attend.hip", "kv_select.hip"])
def test_no_read_of_a_matrix_result_too_soon(asm, source, monkeypatch):
    assert os.path.exists(asm[source]), f"the build keeps the device assembly of {source}"
    monkeypatch.setattr(schedule, "NEED", NEED)
    bad = schedule._closest_reads(asm[source])
    assert not bad, f"{len(bad)} reads of matrix results within {NEED} issue slots, e.g. {sorted(bad, key=lambda b: b[1])[:3]}"


def test_attention_keeps_nothing_in_scratch(asm):
    text = open(asm["kv_attend.hip"]).read()
    found = re.findall(r"\.name: +(\S*kv_attend_kernel\S*)\n(?:.*\n)*?.*\.private_segment_fixed_size: (\d+)", text)
    assert len(found) >= 24
    assert [f for f in found if f[1] != "0"] == []
