"""The products' waits: a warp's threads all get the same answer, and what is reported when one runs out."""

import ctypes as C
import subprocess

import pytest

from paper_2608_19659_gb300 import _build

pytestmark = pytest.mark.gpu

# Of one warp, threads with an odd lane ask for the phase before the barrier's first, which counts as complete; the others for
# the first, which nothing completes: their wait runs out (after 2 s).
HARNESS = r"""
#include "fs_mm.cuh"
__global__ void k(int split, unsigned* answer, uint32_t* status) {
  __shared__ uint64_t bar;
  if (threadIdx.x == 0) fs::mbar_init(&bar, 1);
  __syncthreads();
  answer[threadIdx.x] = fs::mm_wait(&bar, split ? threadIdx.x & 1 : 1, status);
}
extern "C" int run(int split, unsigned* answer, uint32_t* status) {
  k<<<1, 32>>>(split, answer, status);
  return cudaDeviceSynchronize();
}
"""


def test_a_warp_has_one_answer(fsb, cuda, tmp_path):
    torch = cuda
    src, so = tmp_path / "wait.cu", tmp_path / "wait.so"
    src.write_text(HARNESS)
    subprocess.run([_build.nvcc(), *_build.ARCH, *_build.NVCC_FLAGS, "-shared", "-I", _build.CSRC, str(src), "-o", str(so)], check=True)
    run = C.CDLL(str(so)).run
    answer, work = torch.full((32,), 7, dtype=torch.int32, device="cuda"), fsb.MmWorkspace(1, 1, 1)
    call = lambda split: run(split, C.c_void_p(answer.data_ptr()), C.c_void_p(work.address))  # noqa: E731
    assert call(0) == 0 and answer.tolist() == [1] * 32
    fsb.fs_mm_check(work)
    assert call(1) == 0 and answer.tolist() == [0] * 32
    with pytest.raises(fsb.FleetSieveError) as e:
        fsb.fs_mm_check(work)
    assert e.value.code == fsb.FS_ETIMEOUT
    fsb.fs_mm_check(work)  # (said once)
