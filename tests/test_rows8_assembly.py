"""The loads to LDS that csrc/ops/product8_kernels.h writes in assembly, beside code of the compiler's own that uses the same register: compiled
for the device, never run."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

SOURCE = """
#include "product8_kernels.h"
using namespace cams_ops;
#define LOAD(at) __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)a, 4, threadIdx.x * 4 + at, 0, 0, 0)
__global__ void among_others(const int8_t *x, float *y, unsigned n)
{
    __shared__ __attribute__((aligned(1024))) int8_t a[1024], b[1024];
    __shared__ float c[64];
    __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void *)x, 0, n, 0x20000);
    LOAD(0);
    to_lds(raw_buffer(x, n), threadIdx.x * 16, b);
    LOAD(256);
    words_to_lds(raw_buffer(x, n), threadIdx.x * 4, c);
    LOAD(512);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    y[threadIdx.x] = a[threadIdx.x] + b[threadIdx.x] + c[threadIdx.x];
}
"""


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="no hipcc")
def test_the_compiler_knows_that_m0_is_written(tmp_path):
    """All five loads take their place in LDS from m0; the compiler's own ones go to one place, so it sets m0 once if it takes m0 for kept."""
    from paper_2111_00705_amd import build as B
    src, out = tmp_path / "m0.hip", tmp_path / "m0.s"
    src.write_text(SOURCE)
    flags = [f for f in B.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([HIPCC, *flags, "--cuda-device-only", "-S", "-I", B.OPS, "-o", str(out), str(src)], check=True, stdout=subprocess.DEVNULL,
                   stderr=subprocess.DEVNULL)
    body = re.search(r"^_Z12among_others.*?s_endpgm", out.read_text(), re.S | re.M).group(0)
    steps = re.findall(r"s_mov\w* m0|buffer_load_dword\S* [^\n]* lds", body)
    assert len(steps) == 10 and all(s.startswith("s_mov") == (k % 2 == 0) for k, s in enumerate(steps)), steps
