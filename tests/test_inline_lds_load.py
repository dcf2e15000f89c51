"""The loads straight to LDS of the attention kernels are inline assembly that writes m0, the register with the address in LDS.  Between two of the compiler's own such loads
to one place, which need m0 once: compiled to assembly, it has to be written again behind the inline one."""
import re
import subprocess

from paper_2303_11257_amd import build

SOURCE = """
#include "us_flash.h"
using namespace us;
extern "C" __global__ void k(const void* p, uint8_t* out, uint32_t bytes) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const v4i res = buffer_words(p, bytes);
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, bytes, 0x00027000);
  auto known = [&](uint32_t at) { __builtin_amdgcn_raw_ptr_buffer_load_lds(r, US_LDS_AT(void, lds + 4096), 4, threadIdx.x * 4 + at, 0, 0, 0); };
  known(0);
  load_to_lds(res, lds, threadIdx.x * 16);
  known(256);
  __syncthreads();
  out[threadIdx.x] = lds[threadIdx.x] + lds[4096 + threadIdx.x];
}
"""


def test_address_register_is_written_again(tmp_path):
    src, asm = tmp_path / "k.hip", tmp_path / "k.s"
    src.write_text(SOURCE)
    subprocess.run([build.HIPCC, *build.FLAGS, "-I", build.CSRC, "--offload-device-only", "-S", str(src), "-o", str(asm)], check=True)
    lines = [re.sub(r"[;/].*", "", line).strip() for line in asm.read_text().splitlines()]
    loads = [i for i, t in enumerate(lines) if re.match(r"buffer_load_.* lds$", t)]
    assert len(loads) == 3
    for first, last in zip([0] + loads, loads):
        assert any(re.match(r"s_\w+ m0,", t) for t in lines[first:last]), lines[first:last + 1]
