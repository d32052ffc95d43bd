"""Code of the loads that go from memory to LDS: the instruction set asks for a wait state between a scalar write of M0 and the load that takes
its LDS address from there.  The compiler puts one in by itself, but not for asm.  Compiled for gfx950 and read; nothing is run."""
import os
import re
import subprocess

import pytest

from paper_2505_06641_amd import build

PROBE = """
#include "sp_ops_quantized.h"
__global__ void probe(const int8_t* from, int8_t* out, uint32_t n) {
  __shared__ int8_t lds[4096];
  const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) int8_t*)lds;
  for (uint32_t i = 0; i < n; ++i) sp::load_to_lds(at + i * 1024, from + i * 1024, threadIdx.x * 16);
  sp::wait_loads();
  sp::meet();
  out[threadIdx.x] = lds[threadIdx.x];
}
"""


def test_a_write_of_m0_and_the_load_that_reads_it_are_apart(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no compiler here")
    source, listing = tmp_path / "probe.hip", tmp_path / "probe.s"
    source.write_text(PROBE)
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([hipcc, *flags, "--cuda-device-only", "-S", str(source), "-o", str(listing)], check=True, stderr=subprocess.DEVNULL)
    code = [line.split(";")[0].strip() for line in listing.read_text().splitlines()]
    code = [line for line in code if re.match(r"[sv]_|global_|ds_|buffer_", line)]
    loads = [i for i, line in enumerate(code) if line.startswith("global_load_lds")]
    assert loads
    for i in loads:
        assert not re.match(r"[sv]_\w+ m0,", code[i - 1]), code[i - 1:i + 1]
