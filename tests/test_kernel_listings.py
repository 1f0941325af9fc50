"""What the compiler makes of kernels whose source avoids an instruction."""

import os
import re
import subprocess

import pytest

from paper_2608_09703_amd import build_lib


@pytest.mark.parametrize("source", ["mls_attn.hip", "mls_cache.hip", "mls_tree.hip"])
def test_no_64_bit_shift_by_a_vector_register(source, tmp_path):
    """With its count in the last vector register that a kernel is given, such a shift has used register 0."""
    out = str(tmp_path / "listing.s")
    cmd = [build_lib.hipcc(), "-x", "hip", "-S", "--cuda-device-only", "-o", out,
           os.path.join(build_lib.CSRC, source)] + build_lib.common_flags()
    res = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr
    kernels, shifts = 0, []
    for line in open(out):
        kernels += ".amdhsa_kernel" in line
        if re.search(r"\bv_(lshlrev_b64|lshrrev_b64|ashrrev_i64)(_e64)? v\[\d+:\d+\], v\d+,", line):
            shifts.append(line.strip())
    assert kernels > 0 and not shifts, shifts[:3]
