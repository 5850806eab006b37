"""Host side of the split products: no plan counts its tiles' parts outside the counters, and the grid barrier of the orthogonalised
update has a word that nothing else uses.  Compiles the planner as it is for 148 SMs; needs no GPU."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include "orthogonalize.cu"
#include "tc_gemm16.cu"
#include <stdio.h>
namespace pcl { int device_sm_count() { return 148; } }
using namespace pcl;

static long full, wrong;
static void check(int count, int M, int N) {
    const OrthoLayout l = ortho_layout(count, M, N);
    const size_t words = l.counters / 4, barrier = l.barrier / 4;
    // the regions in front of the counters do not reach into one another, and the barrier is one of them
    const size_t x = size_t(count) * M * l.ld * 2, a = size_t(count) * l.d * l.ldd * 2;
    const size_t at[] = {l.part, l.xl, l.xh[0], l.xh[1], l.a, l.b, l.barrier, l.counters, l.total};
    const size_t bytes[] = {size_t(count) * kMaxNormBlocks * 8, x, x, x, a, a, 4};
    for (int i = 0; i < 7; ++i) wrong += at[i] + bytes[i] > at[i + 1];
    for (const Gemm16Args& g : {gram_args(count, M, N, l.form), square_args(count, M, N, l.form), apply_args(count, M, N, l.form)}) {
        const Plan16 p = plan16(g);
        if (p.splits < 2) continue;
        const long rest = p.tiles - p.full_tiles, slots = p.pair ? 16 : 8;
        // part_done() counts at split_tile * slots + warp_slot
        const size_t first = words, last = words + size_t(rest * slots) - 1;
        wrong += rest * slots * 4 > long(kGemm16CounterBytes);
        wrong += barrier >= first && barrier <= last;
        wrong += l.counters + kGemm16CounterBytes + size_t(rest) * p.splits * (p.pair ? 256 * 256 : 128 * 128) * 4 > l.total;
        full += rest * slots * 4 == long(kGemm16CounterBytes);
    }
}

int main() {
    const int named[][3] = {{1, 5824, 22016}, {1, 5504, 16128}, {1, 8576, 14336}, {1, 7040, 7808}, {1, 4592, 10172},
                            {1, 6913, 7761}, {1, 7073, 7809}, {2, 4183, 4850}, {8, 256, 512}, {1, 2048, 2048}, {1, 8200, 4100}};
    for (auto& s : named) check(s[0], s[1], s[2]);
    for (int M = 65; M <= 16384; M += 283)
        for (int N = 65; N <= 32768; N += 401) check(1, M, N);
    for (int count = 2; count <= 40; count += 3)
        for (int M = 80; M <= 5000; M += 164)
            for (int N = 80; N <= 5000; N += 166) check(count, M, N);
    printf("%ld %ld\n", full, wrong);
}
"""


@pytest.mark.skipif(not os.path.exists(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")), reason="needs nvcc")
def test_barrier_and_counters_of_the_orthogonalised_update(tmp_path):
    from paper_1602_06709_b200 import build
    src, exe = tmp_path / "plans.cu", tmp_path / "plans"
    src.write_text(SOURCE)
    # (the device code is compiled but never run; what it and the launches refer to elsewhere stays unresolved)
    r = subprocess.run([build.NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-O1", "-Xptxas", "-O0", "-w", "-I", build.CSRC,
                        "-Xlinker", "--unresolved-symbols=ignore-all", "-o", str(exe), str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr
    full, wrong = map(int, out.stdout.split())
    assert full > 50            # the sizes reach the plans that use every counter
    assert wrong == 0
