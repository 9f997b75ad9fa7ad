"""What the compiler made of the kernels of the 4-bit cache and of eviction, checked without a GPU: no scratch
memory, and registers for the workgroups that a compute unit is meant to hold."""
import shutil

import pytest

from test_kernel_resources import HIPCC, kernel_metadata

pytestmark = pytest.mark.skipif(shutil.which(HIPCC) is None, reason="hipcc not found")


@pytest.mark.parametrize("source", ["hetis_chunks.hip", "hetis_kv4.hip", "hetis_evict.hip"])
def test_no_kernel_uses_scratch_memory(source):
    meta = kernel_metadata(source)
    assert meta
    for name, f in meta.items():
        assert int(f["private_segment_fixed_size"]) == 0 and int(f.get("vgpr_spill_count", 0)) == 0, name
        assert int(f["vgpr_count"]) + int(f.get("agpr_count", 0)) <= 256, name
