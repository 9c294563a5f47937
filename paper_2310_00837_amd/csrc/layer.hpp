// Launchers of the operators of a model's layer on a prepared mini-batch (linear.hip, norm.hip, neighbours.hip,
// embedding.hip, join.hip, join_grad.hip).
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

// ---- embedding.hip
struct EmbeddingJob {
    Count rows;
    int32_t width;
    int table_type, y_type;
    float scale;
    int64_t n_table;
    const void* table;
    int64_t table_ld;
    const int32_t* ids;
    const void* add;                              // nullable
    int64_t add_ld;
    void* y;
    int64_t y_ld;
    int32_t* err;
};
hipError_t launch_embedding(hipStream_t stream, const EmbeddingJob& job);

struct EmbeddingGradJob {
    Count rows;
    int32_t width;
    int table_type, y_type;
    float scale;
    int64_t n_table;
    const int32_t* ids;
    const void* dy;
    int64_t dy_ld;
    void* out;                                    // dtable, or drow where n_distinct is not null
    int64_t out_ld;
    int32_t* row_id;
    int64_t* n_distinct;
    int32_t* err;
};
size_t embedding_grad_scratch_bytes(const EmbeddingGradJob& job);
hipError_t launch_embedding_grad(hipStream_t stream, const EmbeddingGradJob& job, void* scratch);

// ---- join.hip, join_grad.hip
struct Drop {
    uint64_t seed;
    const uint64_t* seed_dev;                     // nullable: read in place of seed
    uint32_t site;
    uint32_t threshold;                           // elements whose 16 bits are less are dropped; 0: none are
    float scale;                                  // of what is kept
};
struct DropoutJob {
    Count rows;
    int32_t width;
    int type;
    Drop drop;
    const void* x;
    int64_t x_ld;
    void* y;
    int64_t y_ld;
};
hipError_t launch_dropout(hipStream_t stream, const DropoutJob& job);

struct JoinJob {
    Count rows;
    int32_t width;
    int x_type;
    bool norm_x;
    float eps, residual_scale;
    Drop drop;
    const void* x;
    int64_t x_ld;
    const void* gain_x;
    const void* gate;
    int64_t gate_ld;                              // 0: one row for all
    const void* residual;
    int64_t residual_ld;
    const void* gain;
    void* total;
    int64_t total_ld;
    void* y;
    int64_t y_ld;
    float* y_scale;                               // not null: y is of kE4M3
    float *inv_rms_x, *inv_rms;
};
hipError_t launch_join(hipStream_t stream, const JoinJob& job);

struct JoinGradJob {
    Count rows;
    int32_t width;
    int type;
    bool norm_x;
    float eps, residual_scale;
    Drop drop;
    const void* x;
    int64_t x_ld;
    const void* gain_x;
    const void* gate;
    int64_t gate_ld;
    const void* gain;
    const void* total;
    int64_t total_ld;
    const void* dy;
    int64_t dy_ld;
    const void* dtotal;
    int64_t dtotal_ld;
    const float *inv_rms_x, *inv_rms;
    void* dx;
    int64_t dx_ld;
    void* dresidual;
    int64_t dresidual_ld;
    void* dgate;
    int64_t dgate_ld;
    void *dgain_x, *dgain;
};
size_t join_grad_scratch_bytes(const JoinGradJob& job);
hipError_t launch_join_grad(hipStream_t stream, const JoinGradJob& job, void* scratch);

}  // namespace helios
