"""The few-rows kernel of a cache leaves it to the buffer descriptors that nothing
behind a sample's slots is read. By the builtins' contract that check covers a
load's vector offset and its constant one, not its scalar offset. So no load of that
kernel has one: a second half of a step, 16 slots further on by a scalar offset,
could pass as if it were the first, and read past the end of a full cache. Read
from the compiler's own listing of cache_one.hip, on the CPU."""
import os
import re
import subprocess

import pytest

from paper_2609_23169_amd import _build


def _scalar_offsets(lines):
    """(number of buffer loads, those with a scalar offset other than 0)."""
    found, bad = 0, []
    for line in lines:
        text = line.split(";")[0].strip()
        if not text.startswith("buffer_load"):
            continue
        found += 1
        m = re.search(r"s\[\d+:\d+\], (\S+)", text)   # the descriptor, then the scalar offset
        if not m or m.group(1) != "0":
            bad.append(text)
    return found, bad


def test_checker_finds_a_planted_offset():
    good = ["buffer_load_dwordx4 v[4:7], v1, s[8:11], 0 offen nt", "buffer_load_dwordx4 v2, s[0:3], 0 offen lds",
            "buffer_load_dwordx4 v[4:7], v1, s[8:11], 0 offen offset:64"]
    assert _scalar_offsets(good) == (3, [])
    for bad in ("buffer_load_dwordx4 v[4:7], v1, s[8:11], s5 offen nt", "buffer_load_dwordx4 v2, s[0:3], s4 offen lds"):
        assert _scalar_offsets(good + [bad]) == (4, [bad])


def test_no_load_of_the_few_rows_kernel_passes_the_check_by_a_scalar_offset(tmp_path):
    if not os.path.exists(_build.HIPCC):
        pytest.skip("no hipcc")
    out = str(tmp_path / "one.s")
    cmd = [_build.HIPCC, *_build.FLAGS, "-x", "hip", "--cuda-device-only", "-S",
           os.path.join(_build.CSRC, "cache_one.hip"), "-o", out]
    subprocess.run(cmd, check=True, capture_output=True)
    with open(out) as f:
        found, bad = _scalar_offsets(f)
    assert found > 50
    assert not bad, bad[:3]
