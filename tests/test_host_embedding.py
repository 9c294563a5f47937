"""The gradient of learnt rows compiled for the host: its results and its scratch.  Every buffer lies between pages that cannot be
touched, so an access out of bounds ends the program; what the sums leave alone has to stay as it was."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2310_00837_amd", "csrc")
CLANG = "/opt/rocm/llvm/bin/clang++"
PROGRAM = r"""
#include <hip/hip_runtime.h>
#include <math.h>
#undef __builtin_amdgcn_readfirstlane
#define __builtin_amdgcn_readfirstlane(v) on_host_readlane(v, 0)
// what layer_dev.hpp names and the gradient does not use
template <class... T> int on_host_none(T...) { abort(); }
#define __builtin_amdgcn_permlane16_swap(...) (long long)(on_host_none(__VA_ARGS__))
#define __builtin_amdgcn_permlane32_swap(...) (long long)(on_host_none(__VA_ARGS__))
#define __builtin_amdgcn_mov_dpp(...) on_host_none(__VA_ARGS__)
#define __builtin_amdgcn_rcpf(x) (1.0f / (x))
#define __builtin_amdgcn_fmed3f(x, lo, hi) fminf(fmaxf(x, lo), hi)
#define __builtin_amdgcn_cvt_pk_fp8_f32(...) on_host_none(__VA_ARGS__)
#define __expf expf
template <class T>
T __shfl(T v, unsigned from, int width) {
    uint64_t lanes;
    const unsigned lane = on_host::now % on_host::kLanes;
    return static_cast<T>(on_host::exchange(v, &lanes)[lane / width * width + from % width]);
}
#include "embedding.hip"
#include <sys/mman.h>
#include <algorithm>
#include <map>
#include <string>
using namespace helios;

// n elements that end where a page that cannot be touched begins, with 32 GiB of such pages on either side
template <class T>
T* guarded(size_t n) {
    const size_t guard = size_t{32} << 30, bytes = (n * sizeof(T) + 4095) / 4096 * 4096;
    char* p = static_cast<char*>(mmap(nullptr, guard + bytes + guard, PROT_NONE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0));
    if (p == MAP_FAILED || (bytes && mprotect(p + guard, bytes, PROT_READ | PROT_WRITE) != 0)) abort();
    memset(p + guard, 0x5a, bytes);
    return reinterpret_cast<T*>(p + guard + bytes - n * sizeof(T));
}
uint32_t next_random() {
    static uint64_t x = 88172645463325252ull;
    x ^= x << 13, x ^= x >> 7, x ^= x << 17;
    return static_cast<uint32_t>(x >> 16);
}
void check(bool ok, const char* what) {
    if (ok) return;
    printf("wrong: %s\n", what);
    exit(1);
}

int main(int argc, char** argv) {
    const int64_t n = std::stol(argv[1]), n_table = std::stol(argv[2]), counted = std::stol(argv[5]);
    const int32_t width = std::stoi(argv[3]);
    const std::string ids_of = argv[4];
    const float scale = 0.5f;
    int32_t *ids = guarded<int32_t>(n), *err = guarded<int32_t>(2);
    float* dy = guarded<float>(n * width);
    int64_t* count = guarded<int64_t>(1);
    *count = counted;
    const int64_t live = counted < 0 ? n : counted;
    bool bad = false;
    for (int64_t i = 0; i < n; ++i) {
        uint32_t id = next_random() % n_table;
        if (ids_of == "one") id = static_cast<uint32_t>(n_table - 1);
        if (ids_of == "few") id = id % std::min<int64_t>(n_table, 5);
        if (ids_of == "skewed" && next_random() % 2) id = static_cast<uint32_t>(n_table / 2);
        ids[i] = static_cast<int32_t>(id);
        if (ids_of == "none" || (ids_of == "skewed" && next_random() % 9 == 0)) ids[i] = -1;
        if (ids_of == "bad" && next_random() % 7 == 0) {
            const int32_t wrong[4] = {-2, INT32_MIN, INT32_MAX, static_cast<int32_t>(n_table)};
            ids[i] = wrong[next_random() % 4];
            bad = bad || i < live;
        }
        for (int32_t c = 0; c < width; ++c) dy[i * width + c] = static_cast<float>(static_cast<int>(next_random() % 17) - 8);       // (sums of these are exact)
    }
    std::map<int32_t, std::vector<float>> want;
    for (int64_t i = 0; i < live; ++i) {
        if (ids[i] < 0 || ids[i] >= n_table) continue;
        std::vector<float>& w = want[ids[i]];
        w.resize(width);
        for (int32_t c = 0; c < width; ++c) w[c] += dy[i * width + c];
    }
    const int64_t rows = std::min(n, n_table);
    float *drow = guarded<float>(rows * width), *dtable = guarded<float>(n_table * width);
    int32_t* row_id = guarded<int32_t>(rows);
    int64_t* n_distinct = guarded<int64_t>(1);
    for (int call = 0; call < 4; ++call) {               // (calls 2 and 3 find the scratch as 0 and 1 have left it)
        const bool dense = call % 2;
        EmbeddingGradJob job{Count{counted < 0 ? nullptr : count, n}, width, kF32, kF32, scale, n_table, ids, dy, width,
                             dense ? dtable : drow, width, dense ? nullptr : row_id, dense ? nullptr : n_distinct, err};
        static unsigned char* scratch[2];
        if (!scratch[dense]) scratch[dense] = guarded<unsigned char>((embedding_grad_scratch_bytes(job) + 255) / 256 * 256);
        err[0] = 0;
        float mark;
        memset(&mark, 0x5a, 4);
        std::fill(drow, drow + rows * width, mark);
        if (launch_embedding_grad(nullptr, job, scratch[dense]) != hipSuccess) return 2;
        check(err[0] == (bad ? kErrData : 0), "error");
        if (dense) {
            for (int64_t k = 0; k < n_table; ++k)
                for (int32_t c = 0; c < width; ++c) check(dtable[k * width + c] == (want.count(k) ? scale * want[k][c] : 0.0f), "dtable");
            continue;
        }
        check(*n_distinct == static_cast<int64_t>(want.size()), "n_distinct");
        int64_t j = 0;
        for (const auto& [id, w] : want) {
            check(row_id[j] == id, "row_id");
            for (int32_t c = 0; c < width; ++c) check(drow[j * width + c] == scale * w[c], "drow");
            ++j;
        }
        for (int64_t q = j * width; q < rows * width; ++q) check(drow[q] == mark, "rows behind the last");
    }
    printf("ok\n");
    return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("embedding")
    (d / "main.cpp").write_text(PROGRAM)
    subprocess.run([CLANG, "-std=c++17", "-O1", "-w", "-U_FORTIFY_SOURCE", "-I", os.path.join(HERE, "hip_on_the_host"), "-I", CSRC,
                    str(d / "main.cpp"), "-o", str(d / "main")], check=True, timeout=100)
    return str(d / "main")


@pytest.mark.parametrize("n,n_table,width,ids,count", [
    (1, 1, 1, "any", -1), (1, 7, 9, "none", -1), (2, 2, 8, "one", -1), (15, 4, 3, "few", -1), (16, 100, 16, "any", -1), (17, 3, 40, "one", -1),
    (100, 10, 130, "few", -1), (777, 1000, 24, "skewed", -1), (1000, 12, 300, "skewed", 0), (1000, 12, 20, "skewed", 333), (2048, 2048, 8, "any", -1),
    (2048, 5, 17, "one", -1), (2048, 3000, 8, "bad", 2047), (2049, 3, 8, "few", -1), (2049, 100_000, 9, "any", 2048), (4097, 2, 12, "one", -1),
    (9000, 70_000, 5, "skewed", -1), (9000, 400, 8, "bad", -1), (12_289, 2_000_000, 2, "any", 12_288), (5000, 260, 136, "few", 1),
    (20_000, 20, 1, "skewed", -1), (5000, 30, 4, "none", -1), (4096, 9000, 4, "any", -1), (4096, 3, 4, "one", 4095),
    (4097, 9000, 4, "any", 4096), (3000, 2, 9, "bad", -1), (100, 5, 8, "few", 0)])
def test_gradient_of_learnt_rows(program, n, n_table, width, ids, count):
    r = subprocess.run([program, str(n), str(n_table), str(width), ids, str(count)], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout == "ok\n", (r.returncode, r.stdout[-500:], r.stderr[-500:])
