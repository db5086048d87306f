"""The kernels of rotary positions and of attention over chosen pages keep their registers: no scratch memory and the occupancy they are written for.
CPU only: hipcc cross-compiles."""
import re
import shutil

import pytest

from tests.test_build_resources import _resources

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not on PATH")


@pytest.mark.parametrize("src,pattern,count,waves", [
    ("rope.hip", r"\drope_kernel", 4, 5), ("rope.hip", r"append_rope_kernel", 4, 5), ("sparse.hip", r"summarize_kernel", 2, 3), ("sparse.hip", r"select_kernel", 10, 4),
    ("sparse.hip", r"\dsparse_kernel", 6, 4), ("sparse.hip", r"sparse_merge_kernel", 2, 5)])
def test_no_scratch_and_occupancy(src, pattern, count, waves):
    hit = {k: v for k, v in _resources(src).items() if re.search(pattern, k)}
    assert len(hit) == count, sorted(hit)
    for name, r in hit.items():
        assert r["VGPRs Spill"] == 0 and r["ScratchSize [bytes/lane]"] == 0, (name, r)
        assert r["Occupancy [waves/SIMD]"] >= waves, (name, r)
