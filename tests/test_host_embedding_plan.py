"""How the gradient of learnt rows is cut into launches, compiled for the host: every launch of every size that the call allows is one that the GPU
takes, and lists with wide rows, which are sorted however short they are, give what others do."""
import os
import subprocess

import pytest

from test_host_embedding import CLANG, CSRC, HERE, PROGRAM, program  # noqa: F401  (a fixture)

LAUNCHES = PROGRAM[:PROGRAM.index('#include "embedding.hip"')] + r"""
#undef hipLaunchKernelGGL
static uint64_t most_threads = 0;
static long launches = 0;
static bool empty = false;
#define hipLaunchKernelGGL(kernel, grid, block, lds, stream, ...) record(grid, block)
static void record(dim3 grid, dim3 block) {
    const uint64_t threads = static_cast<uint64_t>(grid.x) * block.x;
    if (threads > most_threads) most_threads = threads;
    empty = empty || threads == 0;
    ++launches;
}
#include "embedding.hip"
using namespace helios;

int main() {
    const int64_t rows[] = {0, 1, 7, 8, 9, 100, 300, 999, 1000, 2048, 4000, 4095, 4096, 4097, 70000, 1 << 20, (1ll << 31) - 1025};
    const int64_t widths[] = {1, 7, 256, 257, 512, 513, 8192, 70001, 1 << 18, 1 << 20, (1 << 22) + 3, (1 << 24) - 1, 1 << 24};
    const int64_t tables[] = {0, 1, 300, 100000, (1ll << 31) - 1025};
    const int types[][2] = {{kF32, kF32}, {kF32, kF16}, {kF16, kF16}, {kBF16, kBF16}};
    static int64_t n_distinct;
    for (int64_t n : rows)
        for (int64_t width : widths)
            for (int64_t n_table : tables)
                for (const auto& t : types)
                    for (int dense = 0; dense < 2; ++dense) {
                        if (dense && n_table == 0) continue;              // (nothing to write)
                        const EmbeddingGradJob job{Count{nullptr, n}, static_cast<int32_t>(width), t[0], t[1], 1.0f, n_table, nullptr, nullptr, 0,
                                                   nullptr, width, nullptr, dense ? nullptr : &n_distinct, nullptr};
                        most_threads = 0, launches = 0, empty = false;
                        if (embedding_grad_scratch_bytes(job) > 0 && n == 0) return 3;
                        if (launch_embedding_grad(nullptr, job, nullptr) != hipSuccess) return 2;
                        if (launches == 0 || empty || most_threads >= 1ull << 32) {
                            printf("n %ld width %ld table %ld types %d %d dense %d: %ld launches, %lu threads\n", static_cast<long>(n), static_cast<long>(width),
                                   static_cast<long>(n_table), t[0], t[1], dense, launches, static_cast<unsigned long>(most_threads));
                            return 1;
                        }
                    }
    printf("ok\n");
    return 0;
}
"""


def test_every_launch_is_one_that_the_gpu_takes(tmp_path):
    """At least one launch, none of them empty, and fewer than 2^32 threads in each."""
    (tmp_path / "main.cpp").write_text(LAUNCHES)
    subprocess.run([CLANG, "-std=c++17", "-O1", "-w", "-U_FORTIFY_SOURCE", "-I", os.path.join(HERE, "hip_on_the_host"), "-I", CSRC,
                    str(tmp_path / "main.cpp"), "-o", str(tmp_path / "main")], check=True, timeout=100)
    r = subprocess.run([str(tmp_path / "main")], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout == "ok\n", (r.returncode, r.stdout[-500:], r.stderr[-500:])


@pytest.mark.parametrize("n,n_table,width,ids,count", [
    (1, 3, 1_100_000, "any", -1), (31, 7, 300_000, "skewed", -1), (33, 2, 300_000, "one", 32), (100, 1000, 100_000, "any", 0), (1000, 12, 5000, "bad", -1),
    (2048, 2000, 1300, "any", 2047), (4096, 3, 520, "few", -1), (4096, 5000, 260, "skewed", 4095), (4095, 9, 300, "none", -1),
    # ... and tables that are cleared by a launch of their own
    (1000, 1_000_000, 1, "any", -1), (4096, 120_000, 5, "skewed", 4000), (3, 1_200_000, 2, "any", 0)])
def test_gradient_of_short_lists_with_wide_rows_and_of_large_tables(program, n, n_table, width, ids, count):  # noqa: F811
    r = subprocess.run([program, str(n), str(n_table), str(width), ids, str(count)], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout == "ok\n", (r.returncode, r.stdout[-500:], r.stderr[-500:])
