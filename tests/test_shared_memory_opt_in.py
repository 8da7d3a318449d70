"""The record of how much shared memory a kernel may take, under two threads that ask for different sizes.

On the CPU the two CUDA calls are stand-ins: the one that sets the larger size returns only after the smaller one has been set too,
or after half a second where that cannot happen meanwhile."""
import os
import shutil
import subprocess
import threading

import pytest
import torch

import paper_2302_07475_b200 as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <atomic>
#include <chrono>
#include <cstdio>
#include <thread>
#include "s3gd_opt_in.h"

static std::atomic<int> attribute{0}, larger_set{0}, smaller_set{0};
static void wait_for(std::atomic<int>& flag) {
  for (int i = 0; i < 500 && flag.load() == 0; ++i) std::this_thread::sleep_for(std::chrono::milliseconds(1));
}
extern "C" cudaError_t cudaGetDevice(int* dev) { *dev = 1; return cudaSuccess; }
extern "C" cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int bytes) {
  attribute = bytes;
  if (bytes == 200) {
    larger_set = 1;
    wait_for(smaller_set);
    if (smaller_set) std::this_thread::sleep_for(std::chrono::milliseconds(100));   // the smaller one's record comes first
  } else {
    smaller_set = 1;
  }
  return cudaSuccess;
}
int main() {
  static int done[4];
  std::thread larger([] { s3gd::raise_dynamic_smem(nullptr, 200, done, 4); });
  std::thread smaller([] { wait_for(larger_set); s3gd::raise_dynamic_smem(nullptr, 66, done, 4); });
  larger.join();
  smaller.join();
  s3gd::raise_dynamic_smem(nullptr, 200, done, 4);
  std::printf("%d %d\n", attribute.load(), done[1]);
}
"""


def test_a_smaller_size_does_not_undo_a_larger_one(tmp_path):
    include = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")
    if not os.path.isdir(include) or shutil.which("g++") is None:
        pytest.skip("no compiler or no CUDA headers")
    (tmp_path / "p.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-pthread", "-I", include, "-I", os.path.join(ROOT, "paper_2302_07475_b200", "csrc"),
                    str(tmp_path / "p.cpp"), "-o", str(tmp_path / "p")], check=True)
    out = subprocess.run([str(tmp_path / "p")], check=True, capture_output=True, text=True, timeout=60).stdout.split()
    assert out == ["200", "200"]


@pytest.mark.gpu
def test_host_threads_with_small_matrices_of_different_sizes():
    shapes = [(16, 16), (128, 256), (64, 128), (200, 100), (30, 250), (128, 128)]
    g = [torch.randn(s, generator=torch.Generator("cuda").manual_seed(i), device="cuda") for i, s in enumerate(shapes)]
    out, errors = [[] for _ in shapes], []
    start = threading.Barrier(len(shapes))
    torch.cuda.synchronize()

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                ws = S.alloc_ortho_workspace(1, *shapes[i])
                start.wait()
                for _ in range(20):
                    out[i].append(torch.empty_like(g[i]))
                    S.s3gd_orthogonalise(g[i], out[i][-1], ws)
                S.s3gd_device_status(ws)
        except Exception as e:  # noqa: BLE001 -- shown by the main thread
            errors.append((shapes[i], e))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(shapes))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    torch.cuda.synchronize()
    for i, s in enumerate(shapes):
        want = torch.empty_like(g[i])
        S.s3gd_orthogonalise(g[i], want, S.alloc_ortho_workspace(1, *s))
        assert all(torch.equal(o, want) for o in out[i])
