"""The flags that every source is compiled with."""
import subprocess

import pytest

SOURCE = """
#include <hip/hip_runtime.h>
__device__ __noinline__ void wide() { asm volatile("" ::: "v200"); }
__global__ __launch_bounds__(512, BOUND) void kernel() { wide(); }
"""


@pytest.mark.parametrize("bound,fine", [(2, True), (4, False)])
def test_a_kernel_that_misses_its_occupancy_does_not_build(tmp_path, bound, fine):
    """A function that a kernel calls has registers of its own, which count for the kernel: 201 leave two waves per SIMD, not four."""
    from paper_2407_15452_amd import build
    (tmp_path / "k.hip").write_text(SOURCE)
    r = subprocess.run([build.hipcc(), *build.HIPCC_FLAGS, f"-DBOUND={bound}", "-c", str(tmp_path / "k.hip"), "-o", str(tmp_path / "k.o")],
                       capture_output=True, text=True)
    assert (r.returncode == 0) == fine, r.stderr
    assert fine or "occupancy" in r.stderr
