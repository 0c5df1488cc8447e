"""A bounded wait that runs out is the same for all lanes of a warp: one that gave up alone would leave the others to barriers and shuffles
of the whole warp, which then wait for good."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_14507_b200", "csrc")

SHIM = r"""
#include <cuda_runtime.h>
#include "ptx.cuh"
using namespace ipkvi;
// bar[0] completes its phase, nothing ever arrives at bar[1]; half of the lanes wait for either
__global__ void waits(int* out, uint64_t limit_ns) {
    __shared__ uint64_t bar[2];
    const int lane = threadIdx.x;
    if (lane == 0) {
        ptx::mbar_init(ptx::smem_addr(&bar[0]), 1);
        ptx::mbar_init(ptx::smem_addr(&bar[1]), 1);
        ptx::mbar_fence_init();
        ptx::mbar_arrive(ptx::smem_addr(&bar[0]));
    }
    __syncwarp();
    const uint32_t mine = ptx::smem_addr(&bar[lane & 1]);
    out[lane] = ptx::mbar_wait(mine, 0, limit_ns);
    __syncwarp();
    out[32 + lane] = ptx::mbar_wait_warp(mine, 0, limit_ns);
    out[64 + lane] = ptx::mbar_wait_warp(ptx::smem_addr(&bar[0]), 0, limit_ns);
    out[96 + lane] = ptx::warp_agrees(lane != 7);
}
extern "C" int run_waits(int* out) {
    waits<<<1, 32>>>(out, 1000000);
    return cudaDeviceSynchronize();
}
"""


def test_the_waits_of_the_attention_are_the_warps():
    """By reading: in the attention's kernel a wait is voted on by the warp (mbar_wait_warp, warp_agrees), or one lane's alone, whose
    outcome goes to the status word and nowhere else."""
    lines = open(os.path.join(CSRC, "paged_attend.cu")).read().split("__global__")[1].splitlines()
    found = 0
    for i, line in enumerate(lines):
        if re.search(r"\b(mbar_wait|wait_tag)\(", line):
            found += 1
            alone = "or_status(p.status" in line and any("if (lane == 0)" in x for x in lines[i - 2:i])
            assert "warp_agrees(" in line or alone, line
        found += "mbar_wait_warp(" in line
    assert found >= 4
    # and barriers of whole warps come behind a point where the warp's lanes meet
    for i, line in enumerate(lines):
        if "bar.sync" in line:
            assert "__syncwarp();" in lines[i - 1], line
    ptx = open(os.path.join(CSRC, "ptx.cuh")).read()
    for m in re.finditer(r"barrier\.cluster\.(arrive|wait)\S*\.aligned", ptx):
        assert "__syncwarp();" in ptx[:m.start()].splitlines()[-2]


@pytest.mark.gpu
def test_a_warp_gives_up_as_one(tmp_path):
    """Half of the lanes wait for a barrier that nothing completes, one millisecond; nothing waits without a limit."""
    torch = pytest.importorskip("torch")
    src, so = tmp_path / "waits.cu", tmp_path / "libwaits.so"
    src.write_text(SHIM)
    subprocess.run([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-std=c++17", "-O3", "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-Xcompiler", "-fPIC",
                    "-I", CSRC, "-o", str(so), str(src)], check=True)
    out = torch.full((128,), -1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    assert ctypes.CDLL(str(so)).run_waits(ctypes.c_void_p(out.data_ptr())) == 0
    got = out.cpu().view(4, 32).tolist()
    assert got[0] == [1, 0] * 16                         # a lane's own wait is its own
    assert got[1] == [0] * 32 and got[2] == [1] * 32 and got[3] == [0] * 32
