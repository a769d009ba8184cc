"""What the compiler reports of a kernel: the joining of many ranges keeps those it has asked for in registers.  (An array of which some elements are left
unwritten lay in scratch memory, each load waited for before the next.)"""
import os
import re
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_ranges_to_be_joined_wait_in_registers(tmp_path):
    sys.path.insert(0, ROOT)
    import __graft_entry__ as entry
    if not os.path.exists(os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")):
        pytest.skip("no compiler")
    listing = str(tmp_path / "kernels_q8.s")
    entry._run(entry._compile("kernels_q8.hip", listing, ["-S", "--cuda-device-only"]))
    found = re.findall(r"\.name:\s+(\S*merge_long_kernel\S*)\n(?:.*\n)*?\s+\.private_segment_fixed_size:\s+(\d+)", open(listing).read())
    assert len(found) == 4 and all(int(n) == 0 for _, n in found), found
