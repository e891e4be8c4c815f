"""Where the products with 4-bit weights read the rows of `a` on their way through LDS (host code of csrc/launch_w4.h), on
the CPU: every copy of every tile lies within the matrix, and what is used is read from its own place."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include "launch_w4.h"

static void fail(const char* what, int64_t rows, int K, int64_t stride, int k, int run, int lane) {
    std::printf("%s: %lld rows of %d at %lld, tile %d, copy %d, lane %d\n", what, (long long)rows, K, (long long)stride, k, run, lane);
    std::exit(1);
}

// A tile whose first row is followed by `rows` - 1 more.
template <int TM, int WAVES>
static void check(int64_t rows, int K, int64_t stride) {
    constexpr int COPIES = TM / 4 / WAVES;
    const int64_t end = ((rows - 1) * stride + K) * 2;
    for (int wave = 0; wave < WAVES; ++wave)
        for (int lane = 0; lane < 64; ++lane) {
            lsh::W4RowCopies<TM, COPIES> from(lane, wave * COPIES, rows - 1, (uint32_t)(stride * 2));
            for (int k = 0; 128 * k < K; ++k) {
                if (128 * k + 128 > K) from.shorten((uint32_t)(K - 128 * k) * 2);
                for (int j = 0; j < COPIES; ++j) {
                    const int run = wave * COPIES + j, row = 8 * (run % (TM / 8)) + lane / 8;
                    const int input = 64 * (run / (TM / 8)) + 8 * ((lane % 8) ^ (row % 8));  // of the tile
                    const int64_t v = from.at[j], at = v + 256 * (int64_t)k;
                    if (at < 0 || at + 16 > end || at >= (int64_t)1 << 32) fail("outside the matrix", rows, K, stride, k, run, lane);
                    if (v % 16 != 0 || at / 2 % stride + 8 > K) fail("between two rows", rows, K, stride, k, run, lane);
                    if (row < rows && 128 * k + input < K && at != (row * stride + 128 * k + input) * 2)
                        fail("another place", rows, K, stride, k, run, lane);
                }
            }
        }
}

int main() {
    for (int K : {32, 64, 96, 128, 160, 224, 256, 416, 1056})
        for (int64_t stride : {(int64_t)K, (int64_t)K + 8, (int64_t)1 << 20, ((int64_t)1 << 24) - 8})
            for (int64_t rows : {1, 2, 7, 8, 9, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 100000}) {
                check<32, 4>(rows, K, stride);  // tiles of the four kernels
                check<64, 4>(rows, K, stride);
                check<64, 8>(rows, K, stride);
                check<128, 8>(rows, K, stride);
            }
    std::puts("ok");
}
"""


def test_copies_stay_in_the_matrix(tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc is missing")
    src, exe = str(tmp_path / "rows.cpp"), str(tmp_path / "rows")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.check_call([hipcc, "-O1", "-std=c++17", "--offload-arch=gfx950", "-I", os.path.join(ROOT, "include"),
                           "-I", os.path.join(ROOT, "paper_2001_04451_amd", "csrc"), src, "-o", exe])
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and res.stdout.endswith("ok\n"), res.stdout + res.stderr
