"""Reads across lanes that are written as text in the rotation of rows stand two wait states behind what they read."""
import os
import subprocess

import pytest

from paper_2406_11235_amd import build
from test_wait_states import HIPCC, too_early


def test_reads_across_lanes_in_the_rows_kernels(tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("no hipcc")
    out = tmp_path / "rows.s"
    flags = [f for f in build.FLAGS if f not in ("-shared", "-pthread")]
    subprocess.run([HIPCC] + flags + ["-S", "--cuda-device-only", "-x", "hip", os.path.join(build.CSRC, "qtip_rows.hip"), "-o", str(out)],
                   check=True, capture_output=True)
    reads, found = too_early(out.read_text().splitlines())
    assert reads >= 16 * 64  # the lanes' stages of the kernels that rotate
    assert not found, found[:4]
