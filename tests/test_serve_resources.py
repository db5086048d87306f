"""The kernels of a serving step keep their registers: no scratch memory, the occupancy they are written for, and no scratch access in the loops over the keys.
CPU only: hipcc cross-compiles."""
import re
import shutil

import pytest

from tests.test_build_resources import _resources

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not on PATH")


@pytest.mark.parametrize("src,pattern,count,waves", [
    ("ragged.hip", r"ragged_few_kernelILi(64|128)ELi1E", 2, 3), ("ragged.hip", r"ragged_few_kernelILi(64|128)ELi2E", 2, 2), ("ragged.hip", r"ragged_wide_kernel", 2, 2),
    ("ragged.hip", r"ragged_merge_kernel", 4, 4), ("serve.hip", r"append_kernel", 2, 8), ("serve.hip", r"read_kernel", 2, 8), ("serve.hip", r"plan_(one|scan|fill)_kernel", 3, 4)])
def test_no_scratch_and_occupancy(src, pattern, count, waves):
    hit = {k: v for k, v in _resources(src).items() if re.search(pattern, k)}
    assert len(hit) == count, sorted(hit)
    for name, r in hit.items():
        assert r["VGPRs Spill"] == 0 and r["ScratchSize [bytes/lane]"] == 0, (name, r)      # (scalar registers parked in lanes cost no memory access)
        assert r["Occupancy [waves/SIMD]"] >= waves, (name, r)
