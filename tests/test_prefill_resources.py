"""What the compiler made of the kernels of prefill Attention, rotary positions and the choice of pages, checked
without a GPU: no scratch memory, and registers and LDS for the workgroups that a compute unit is meant to hold."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2509_08309_amd import build
from test_chunk_resources import resources
from test_kernel_resources import HIPCC, kernel_metadata

pytestmark = pytest.mark.skipif(shutil.which(HIPCC) is None, reason="hipcc not found")

SOURCES = [("hetis_prefill.hip", 2 + 2), ("hetis_rope.hip", 8), ("hetis_select.hip", 4 + 2 + 3)]


@pytest.mark.parametrize("source,kernels", SOURCES)
def test_no_kernel_uses_scratch_memory(source, kernels):
    meta = kernel_metadata(source)
    assert len(meta) == kernels, sorted(meta)
    for name, f in meta.items():
        assert int(f["private_segment_fixed_size"]) == 0 and int(f.get("vgpr_spill_count", 0)) == 0, name


def residents(name):
    """Workgroups that a compute unit is meant to hold at the same time."""
    m = re.search(r"rope_kernelILi\d+ELb[01]ELi(\d)E", name)
    if m:
        return 3 if m.group(1) == "4" else 5         # (256 threads)
    if "bounds_kernel" in name or "score_kernel" in name:
        return 4                                     # (256 threads)
    if "select_kernel" in name:
        return 2                                     # (1024 threads)
    assert "prefill_kernel" in name or "prefill_direct_kernel" in name, name
    return 2                                         # (256 threads, and close to half of the LDS at head_dim 128)


@pytest.mark.parametrize("source,kernels", SOURCES)
def test_a_compute_unit_holds_the_workgroups_it_is_meant_to(source, kernels):
    """512 registers a lane and SIMD, given out in eights, four SIMDs, 160 KB of LDS."""
    found = resources(source)
    assert len(found) == kernels, sorted(found)
    for name, (registers, lds, threads) in found.items():
        waves = min(512 // (-(-registers // 8) * 8), 8)      # of a SIMD
        assert 4 * waves * 64 >= residents(name) * threads, (name, registers)
        assert residents(name) * lds <= 160 << 10, (name, lds)


def test_the_compiler_knows_what_loads_into_lds_change():
    """M0 is set by hand for them, in inline assembly that names it among the registers that it changes."""
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    ir = subprocess.run([HIPCC, *flags, "--cuda-device-only", "-S", "-emit-llvm", "-o", "-",
                         os.path.join(build.CSRC, "hetis_prefill.hip")], capture_output=True, text=True, check=True).stdout
    found = [line for line in ir.splitlines() if " asm " in line and "s_mov_b32 m0" in line]
    assert len(found) >= 4, "two head dims, two kernels"
    for line in found:
        assert "~{m0}" in line, line.strip()
