"""Kernels that walk a layer's entries by the whole grid, at the largest number of entries that there can be: their text is compiled for the host, and the
thread whose counter goes furthest past the end walks over arrays that take address space but hardly any memory."""
import os
import re
import subprocess

import pytest

from tests.routes import ROOT

HOST = r"""
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <sys/mman.h>
#define __global__
#define __launch_bounds__(n)
#define BLOCK_THREADS 256
#define WAVES_PER_BLOCK 4
using std::min;
struct { unsigned x, y, z; } blockIdx, threadIdx, gridDim;
struct LayerDev { int32_t nnz, n_out; float *vals_t; const float *vals; const int32_t *t_perm; };
static double bias_gradient(const LayerDev &, int, int, int, int) { return 0.0; }
KERNEL
int main()
{
    const int n = 0x7fffffff;
    auto room = [](size_t bytes) { return mmap(nullptr, bytes, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0); };
    const float *g = (const float *)room(4 * (size_t)n);
    int32_t *perm = (int32_t *)room(4 * (size_t)n);
    float *out = (float *)room(4 * (size_t)n);
    if (g == MAP_FAILED || perm == MAP_FAILED || out == MAP_FAILED) return 77;
    const LayerDev layer = {n, 0, out, g, perm};
    (void)layer;
    gridDim = {4096, 1, 1};
    CALL;
    puts("walked");
}
"""
CALLS = {"k_sum_parts": "k_sum_parts(g, nullptr, perm, out, n)", "k_refresh_vals_t": "k_refresh_vals_t(&layer)",
         "k_hand_out": "k_hand_out(&layer, 4, 4, nullptr, 0, g, nullptr, perm, out, n)"}


@pytest.mark.parametrize("kernel", CALLS)
def test_counters_of_entries_do_not_wrap(kernel, tmp_path):
    source = open(os.path.join(ROOT, "paper_2104_11805_amd", "csrc", "sdnn.hip")).read()
    text = re.search(r"^__global__ [^;{]*\b" + kernel + r"\(.*?^}\n", source, re.M | re.S).group(0)
    (tmp_path / "walk.cpp").write_text(HOST.replace("KERNEL", text).replace("CALL", CALLS[kernel]))
    subprocess.run(["g++", "-std=c++17", "-O1", "-fwrapv", "-w", str(tmp_path / "walk.cpp"), "-o", str(tmp_path / "walk")], check=True)
    out = subprocess.run([str(tmp_path / "walk")], capture_output=True, text=True, timeout=60)
    if out.returncode == 77:
        pytest.skip("no 24 GiB of address space")
    assert out.returncode == 0 and out.stdout == "walked\n", out.returncode
