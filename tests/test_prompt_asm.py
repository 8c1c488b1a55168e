"""What the compiler makes of attention of packed prompts, read without a GPU: the loads to LDS that it issues by itself, the registers that its kernels take."""
import os
import re
import subprocess

import pytest

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


_RESIDENT = r"""
#include <cstdio>
#include <initializer_list>
#include "prompt_layout.h"
int main() {
    for (int size : {2, 4})
        for (int hd : {32, 64, 96, 128, 192, 256}) printf("%d %d %d\n", size, hd, prompt_resident(size, hd));
}
"""
OBJECT = os.path.join(os.path.dirname(CSRC), "_build", "prompt_ops.o")
LLVM = "/opt/rocm/llvm/bin/"


@pytest.mark.skipif(not os.path.exists(OBJECT), reason="the library's objects are not here")
def test_workgroups_a_cu_holds(tmp_path):
    """A workgroup is a wavefront on each of a CU's four SIMDs, which have 512 registers, given out 8 at a time, for at most 8 of them; the CU has 160 KiB of LDS."""
    run = lambda *cmd: subprocess.run([str(c) for c in cmd], check=True, capture_output=True, text=True).stdout
    run(LLVM + "llvm-objcopy", "--dump-section", f".hip_fatbin={tmp_path / 'bundle'}", OBJECT, tmp_path / "copy.o")
    run(LLVM + "clang-offload-bundler", "--unbundle", "--type=o", f"--input={tmp_path / 'bundle'}", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", f"--output={tmp_path / 'code'}")
    have = {}
    for kernel in run(LLVM + "llvm-readelf", "--notes", tmp_path / "code").split(".group_segment_fixed_size:")[1:]:
        m = re.search(r"\.name: +_Z25prompt_attention(16|32)_kernelILi(\d+)ELb1EE", kernel)
        if m:
            lds, registers = int(kernel.split()[0]), int(re.search(r"\.vgpr_count: +(\d+)", kernel)[1])
            have[int(m[1]) // 8, int(m[2])] = min(8, 512 // ((registers + 7) // 8 * 8), 160 * 1024 // lds)
    (tmp_path / "main.cpp").write_text(_RESIDENT)
    run("g++", "-std=c++17", "-I", CSRC, tmp_path / "main.cpp", "-o", tmp_path / "main")
    said = {(int(size), int(hd)): int(n) for size, hd, n in (line.split() for line in run(tmp_path / "main").splitlines())}
    assert len(have) == 12 and have == said
