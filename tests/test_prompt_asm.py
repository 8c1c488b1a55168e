"""What the compiler knows of the loads to LDS that attention of packed prompts issues by itself: compiled for gfx950, read as assembly, no GPU."""
import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_07503_amd", "csrc")
_BETWEEN = r"""
#include "kernels_prompt.hip.h"

// the compiler's own load to LDS, with M0 its target, on either side of prompt_to_lds
__global__ void between(const char *p, float *out) {
    __shared__ __attribute__((aligned(16))) unsigned char lds[4096];
    __builtin_amdgcn_global_load_lds((prompt_glb_t *)(p + threadIdx.x * 16), (prompt_lds_t *)lds, 16, 0, 0);
    prompt_to_lds(p, threadIdx.x * 16u, lds + 1024);
    __builtin_amdgcn_global_load_lds((prompt_glb_t *)(p + 8192 + threadIdx.x * 16), (prompt_lds_t *)lds, 16, 2048, 0);
    prompt_barrier();
    out[threadIdx.x] = lds[threadIdx.x * 16];
}
"""


def test_m0_is_set_again_behind_a_load_to_lds(tmp_path):
    (tmp_path / "between.hip").write_text(_BETWEEN)
    r = subprocess.run(["hipcc", "--offload-arch=gfx950", "-O3", "-std=c++17", "-Wall", "-Wno-unused-function", "-I", CSRC, "-S", "--cuda-device-only", str(tmp_path / "between.hip"), "-o",
                        str(tmp_path / "between.s")], capture_output=True, text=True)
    assert r.returncode == 0 and "inline-asm" not in r.stderr, r.stderr
    found = re.findall(r"(s_mov_b32 m0|global_load_lds)", (tmp_path / "between.s").read_text())
    assert found == ["s_mov_b32 m0", "global_load_lds"] * 3, found
