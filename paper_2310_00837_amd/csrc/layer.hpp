// Launchers of the operators of a model's layer on a prepared mini-batch (linear.hip, norm.hip, neighbours.hip).
// Every launcher enqueues on `stream` and returns the hipError_t of the launch.
#pragma once
#include "common.hpp"

namespace helios {

// ---- linear.hip
struct LinearJob {
    Count rows;                                   // of x; rows.host is the most
    int32_t n_in, n_out;
    int act, x_type, out_type;
    const void* x;
    int64_t x_ld;
    const float* x_scale;
    const void* w;
    int64_t w_ld;
    const float* w_scale;
    const void* bias;                             // from here on elements of out_type, nullable but y
    const void* residual;
    int64_t residual_ld;
    void* pre;
    int64_t pre_ld;
    void* y;
    int64_t y_ld;
};
hipError_t launch_linear(hipStream_t stream, const LinearJob& job);

struct LinearGradJob {
    Count rows;
    int32_t n_in, n_out;
    int act, x_type, out_type;
    const void* x;
    int64_t x_ld;
    const void* w;
    int64_t w_ld;
    const void* dy;
    int64_t dy_ld;
    const void* pre;
    int64_t pre_ld;
    void* dx;                                     // x_type, nullable
    int64_t dx_ld;
    void* dw;                                     // x_type, nullable
    int64_t dw_ld;
    void* dbias;                                  // out_type, nullable
};
size_t linear_grad_scratch_bytes(const LinearGradJob& job);
hipError_t launch_linear_grad(hipStream_t stream, const LinearGradJob& job, void* scratch);

// ---- norm.hip
struct NormJob {
    Count rows;
    int32_t width;
    int x_type, y_type;                           // y_type: x_type or kE4M3
    bool normalise;                               // false: the rows go to 8 bits as they are
    float eps;
    const void* x;
    int64_t x_ld;
    const void* residual;
    int64_t residual_ld;
    const void* gain;
    void* total;
    int64_t total_ld;
    void* y;
    int64_t y_ld;
    float* y_scale;
    float* inv_rms;
};
hipError_t launch_norm(hipStream_t stream, const NormJob& job);

struct NormGradJob {
    Count rows;
    int32_t width;
    int type;
    float eps;
    const void* total;
    int64_t total_ld;
    const void* gain;
    const float* inv_rms;
    const void* dy;
    int64_t dy_ld;
    const void* dtotal;
    int64_t dtotal_ld;
    void* dx;
    int64_t dx_ld;
    void* dgain;
};
size_t norm_grad_scratch_bytes(const NormGradJob& job);
hipError_t launch_norm_grad(hipStream_t stream, const NormGradJob& job, void* scratch);

// ---- neighbours.hip
constexpr uint32_t kLayerCounters = 512;
struct MeanJob {
    Count rows;
    int32_t width, type;
    const void* x;
    int64_t x_ld;
    int64_t n_src;
    const int64_t* indptr;
    const int32_t* col;
    int64_t n_col;                                // entries that col has room for
    const int32_t* row;                           // nullable: row i's own source is i
    void* mean;
    int64_t mean_ld;
    void* own;                                    // nullable
    int64_t own_ld;
    int32_t* err;
};
hipError_t launch_block_mean(hipStream_t stream, const MeanJob& job);

struct TransposeJob {
    Count rows;
    const int64_t* indptr;
    const int32_t* col;
    int64_t n_col;
    const int32_t* row;                           // nullable: no entries for the rows' own sources
    int64_t n_src;
    int32_t *src_indptr, *src_entry;
    int32_t* err;
};
size_t block_transpose_scratch_bytes(const TransposeJob& job);
hipError_t launch_block_transpose(hipStream_t stream, const TransposeJob& job, void* scratch);

struct MeanGradJob {
    int64_t n_rows, n_src, n_entries;             // the most that the lists can hold
    int32_t width, type;
    const int64_t* indptr;
    const int32_t *src_indptr, *src_entry;
    const void* dmean;
    int64_t dmean_ld;
    const void* down;                             // nullable
    int64_t down_ld;
    void* dx;
    int64_t dx_ld;
    int32_t* err;
};
// counters: uint32[kLayerCounters], zero, and left so
size_t block_mean_grad_scratch_bytes(const MeanGradJob& job);
hipError_t launch_block_mean_grad(hipStream_t stream, const MeanGradJob& job, uint32_t* counters, void* scratch);

}  // namespace helios
