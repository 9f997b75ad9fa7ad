"""What the compiler made of the kernels of the 4-bit cache and of eviction, checked without a GPU: no scratch
memory, and registers for the workgroups that a compute unit is meant to hold."""
import re
import shutil

import pytest

from test_kernel_resources import HIPCC, assembly, kernel_metadata

pytestmark = pytest.mark.skipif(shutil.which(HIPCC) is None, reason="hipcc not found")


@pytest.mark.parametrize("source", ["hetis_chunks.hip", "hetis_kv4.hip", "hetis_evict.hip"])
def test_no_kernel_uses_scratch_memory(source):
    meta = kernel_metadata(source)
    assert meta
    for name, f in meta.items():
        assert int(f["private_segment_fixed_size"]) == 0 and int(f.get("vgpr_spill_count", 0)) == 0, name
        assert int(f["vgpr_count"]) + int(f.get("agpr_count", 0)) <= 256, name


def resources(source):
    """Registers of a lane, bytes of LDS and threads of every kernel."""
    text, out = assembly(source), {}
    for block in re.findall(r"^  - \.agpr_count:.*?(?=^  - \.agpr_count|^amdhsa)", text, re.S | re.M):
        name = re.search(r"^    \.name:\s+(\S+)", block, re.M).group(1)
        number = lambda field: int(re.search(rf"\.{field}:\s+(\d+)", block).group(1))
        out[name] = number("vgpr_count"), number("group_segment_fixed_size"), number("max_flat_workgroup_size")
    return out


def residents(name):
    """Workgroups that a compute unit is meant to hold at the same time."""
    m = re.search(r"chunk_kernelILi(\d+)ELb([01])E", name)
    if m:                                                    # chunk_residents()
        return {("64", "1"): 4, ("64", "0"): 3, ("128", "1"): 3, ("128", "0"): 2}[m.groups()]
    if "chunk_combine" in name or "chunk_weights" in name:
        return 7
    if "evict_kernel" in name:
        return 1
    assert "kv4_rows_kernel" in name or "kv_move_rows_kernel" in name, name
    return 8


@pytest.mark.parametrize("source,kernels", [("hetis_chunks.hip", 6 + 8 + 8), ("hetis_kv4.hip", 4), ("hetis_evict.hip", 4 + 4)])
def test_a_compute_unit_holds_the_workgroups_it_is_meant_to(source, kernels):
    """512 registers a lane and SIMD, given out in eights, four SIMDs, 160 KB of LDS."""
    found = resources(source)
    assert len(found) == kernels, sorted(found)
    for name, (registers, lds, threads) in found.items():
        waves = 512 // (-(-registers // 8) * 8)              # of a SIMD
        assert 4 * waves * 64 >= residents(name) * threads, (name, registers)
        assert residents(name) * lds <= 160 << 10, (name, lds)
