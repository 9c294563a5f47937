// Dropout, and the join of a layer's output with the rows that went around the layer.
//
//   u = x * gain_x / sqrt(mean(x^2) + eps);  total = r * residual + gate * drop(u);  y = total * gain / sqrt(mean(total^2) + eps)
//   gradient, with q and qx the reciprocal roots, a = dy * gain and m = 1 / (1 - p) or 0:
//   dt = dtotal + q (a - total q^2 mean(a total));  dresidual = r dt;  dgate = m dt x qx gain_x;  w = m dt gate
//   dx = qx (w gain_x - x qx^2 mean(w gain_x x));  dgain_x = sum over rows of w x qx;  dgain = sum of dy total q
//
// A row is held in the registers of the lanes that share it, in 32 bits, as in the norm: both norms, the dropped elements and
// the 8-bit output are one pass over what has to be read and written, with two sums over the row, the second of which needs the first.
#include "drop_dev.hpp"

#include <algorithm>

namespace helios {

namespace {

constexpr int64_t kMostBlocks = 1 << 21;            // of a launch
constexpr int kItems = 2;                           // of a thread of the dropout kernel, in flight together

// An item is eight neighbouring columns of a row; items are numbered along the rows.
template <int TYPE>
__global__ __launch_bounds__(kBlock) void dropout_kernel(DropoutJob p) {
    const uint32_t blocks = static_cast<uint32_t>(p.width + 7) / 8;
    const int64_t items = p.rows.get() * blocks, step = static_cast<int64_t>(gridDim.x) * kBlock * kItems;
    const uint64_t seed = drop_seed(p.drop);
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * kBlock * kItems; base < items; base += step) {
        const ItemPlaces places(base, blocks);
        Raw8<TYPE> raw[kItems];
        int64_t row[kItems];
        int32_t col[kItems], valid[kItems];
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            const uint32_t i = k * kBlock + threadIdx.x;
            places.get(i, &row[k], &col[k]);
            valid[k] = base + i < items ? p.width - col[k] : 0;
            raw[k].load(p.x, row[k] * p.x_ld + col[k], valid[k]);
        }
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            float v[8];
            const uint32_t kept = p.drop.threshold ? kept_8(p.drop, seed, row[k], col[k]) : 0xffu;
            widen_8<TYPE>(raw[k].v, v);
            drop_8(kept, p.drop.scale, v);
            store_8_of<TYPE>(p.y, row[k] * p.y_ld + col[k], valid[k], v);
        }
    }
}

// ---- forward

template <int TYPE, int LANES, int CHUNKS>
__device__ __forceinline__ void join_row(const JoinJob& p, uint64_t seed, int64_t row, int lane, float* s) {
    constexpr bool kAhead = LANES <= kBlock;            // everything is asked for at once; 1024 threads have no registers for that
    float t[CHUNKS][8];
    Raw8<TYPE> residual[CHUNKS], gate[CHUNKS];
    const auto load_rest = [&](int c) {
        const int col = (c * LANES + lane) * 8, valid = p.width - col;
        if (p.residual) residual[c].load(p.residual, row * p.residual_ld + col, valid);
        if (p.gate) gate[c].load(p.gate, row * p.gate_ld + col, valid);
    };
    float sum = 0;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int col = (c * LANES + lane) * 8;
        load_8_of<TYPE>(p.x, row * p.x_ld + col, p.width - col, t[c]);
        if (kAhead) load_rest(c);
    }
    if (p.norm_x) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += t[c][e] * t[c][e];
        const float q = 1.0f / sqrtf(row_sum<LANES>(sum, s) / p.width + p.eps);
        if (p.inv_rms_x && lane == 0) p.inv_rms_x[row] = q;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int col = (c * LANES + lane) * 8;
            float g[8] = {1, 1, 1, 1, 1, 1, 1, 1};
            if (p.gain_x) load_8_of<TYPE>(p.gain_x, col, p.width - col, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) t[c][e] *= q * g[e];
        }
    }
    sum = 0;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int col = (c * LANES + lane) * 8, valid = p.width - col;
        if (!kAhead) load_rest(c);
        if (p.drop.threshold) drop_8(kept_8(p.drop, seed, row, col), p.drop.scale, t[c]);
        float v[8];
        if (p.gate) {
            widen_8<TYPE>(gate[c].v, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) t[c][e] *= v[e];
        }
        if (p.residual) {
            widen_8<TYPE>(residual[c].v, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) t[c][e] += p.residual_scale * v[e];
        }
        if (p.total) store_8_of<TYPE>(p.total, row * p.total_ld + col, valid, t[c]);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += t[c][e] * t[c][e];
    }
    if (!p.y) return;
    const float q = 1.0f / sqrtf(row_sum<LANES>(sum, s) / p.width + p.eps);
    if (p.inv_rms && lane == 0) p.inv_rms[row] = q;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int col = (c * LANES + lane) * 8;
        float g[8] = {1, 1, 1, 1, 1, 1, 1, 1};
        if (p.gain) load_8_of<TYPE>(p.gain, col, p.width - col, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) t[c][e] *= q * g[e];
    }
    finish_row<TYPE, LANES, CHUNKS>(t, p.width, lane, s, p.y, row * p.y_ld, p.y_scale ? p.y_scale + row : nullptr);
}

template <int TYPE, int LANES, int CHUNKS>
__global__ __launch_bounds__(RowShape<LANES>::kThreads) void join_kernel(JoinJob p) {
    constexpr int kThreads = RowShape<LANES>::kThreads, kRows = RowShape<LANES>::kRows;
    __shared__ float s[kThreads / kWave];
    const int64_t count = p.rows.get();
    const uint64_t seed = drop_seed(p.drop);
    const int lane = threadIdx.x % LANES;
    for (int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / LANES; row < count; row += static_cast<int64_t>(gridDim.x) * kRows)
        join_row<TYPE, LANES, CHUNKS>(p, seed, row, lane, s);
}

// ---- gradient

// The sums over the rows: dgain_x, dgain and that of a gate of one row.  Every workgroup has one row of parts for each that is asked for,
// at part + (which * workgroups + workgroup) * width; join_sum_kernel adds them up.
enum Summed { kSumGainX = 0, kSumGain = 1, kSumGate = 2, kSums = 3 };
struct SumPlaces {
    void* to[kSums];                              // null: not asked for
    int at[kSums];                                // its number among those that are
    int n;
};
SumPlaces sums_of(const JoinGradJob& p) {
    SumPlaces s{{p.dgain_x, p.dgain, p.gate_ld == 0 ? p.dgate : nullptr}, {0, 0, 0}, 0};
    for (int k = 0; k < kSums; ++k)
        if (s.to[k]) s.at[k] = s.n++;
    return s;
}

// What the sums over a row leave for its elements.
struct RowFactors {
    float q, f;                                   // 1 / rms of total, and q^2 times the mean of a total
    float qx;
};
// dt, and drop(dt) with its factors, of eight elements.
struct GradOf8 {
    float dt[8], w[8], slope[8];                  // slope: drop(dt) x qx gain_x, the gate's gradient
};
__device__ __forceinline__ GradOf8 grad_of_8(const JoinGradJob& p, const RowFactors& r, uint32_t kept, const float (&t)[8], const float (&dy)[8],
                                             const float (&dtotal)[8], const float (&x)[8], const float (&gain)[8], const float (&gain_x)[8],
                                             const float (&gate)[8]) {
    GradOf8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o.dt[e] = dtotal[e];
    if (p.dy)
#pragma unroll
        for (int e = 0; e < 8; ++e) o.dt[e] += r.q * (dy[e] * gain[e] - t[e] * r.f);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const bool is_kept = (kept >> e) & 1u;
        const float v = o.dt[e] * p.drop.scale;
        o.slope[e] = is_kept ? v * (x[e] * r.qx * gain_x[e]) : 0.0f;
        o.w[e] = is_kept ? v * gate[e] : 0.0f;
    }
    return o;
}

template <int LANES, int CHUNKS>
struct JoinGradShape {
    static constexpr int kThreads = LANES <= kWave && CHUNKS == 1 ? 512 : RowShape<LANES>::kThreads, kRows = kThreads / LANES;
    static constexpr int kMostBlocks = kThreads == kBlock ? 1024 : 512;
};
// Every workgroup goes through rows blockIdx.x * kRows + ..., asks for a row while the one before it is worked on (rows of up to
// eight elements a lane), and keeps its lanes' sums until the end.
template <int TYPE, int LANES, int CHUNKS>
__global__ __launch_bounds__((JoinGradShape<LANES, CHUNKS>::kThreads)) void join_grad_kernel(JoinGradJob p, SumPlaces places, float* part) {
    constexpr int kThreads = JoinGradShape<LANES, CHUNKS>::kThreads, kRows = JoinGradShape<LANES, CHUNKS>::kRows, kWidth = LANES * CHUNKS * 8;
    constexpr bool kPipeline = CHUNKS == 1 && LANES <= kBlock;
    __shared__ float s[kThreads / kWave];
    __shared__ float s_sum[kRows > 1 ? kRows : 1][kRows > 1 ? kWidth : 1];
    const int64_t count = p.rows.get(), stride = static_cast<int64_t>(gridDim.x) * kRows;
    const uint64_t seed = drop_seed(p.drop);
    const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES;
    float sums[kSums][CHUNKS][8];
#pragma unroll
    for (int k = 0; k < kSums; ++k)
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) sums[k][c][e] = 0;
    Raw8<TYPE> t_raw[CHUNKS], d_raw[CHUNKS], r_raw[CHUNKS], x_raw[CHUNKS], g_raw[CHUNKS];
    const auto load = [&](int64_t row) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int col = (c * LANES + lane) * 8, valid = p.width - col;
            if (p.dy) {
                t_raw[c].load(p.total, row * p.total_ld + col, valid);
                d_raw[c].load(p.dy, row * p.dy_ld + col, valid);
            }
            if (p.dtotal) r_raw[c].load(p.dtotal, row * p.dtotal_ld + col, valid);
            x_raw[c].load(p.x, row * p.x_ld + col, valid);
            if (p.gate && p.gate_ld) g_raw[c].load(p.gate, row * p.gate_ld + col, valid);
        }
    };
    // (what is the same for all rows stays in registers where a lane has one chunk)
    const auto vector_of = [&](const void* v, int c, float (&g)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = 1;
        if (v) load_8_of<TYPE>(v, (c * LANES + lane) * 8, p.width - (c * LANES + lane) * 8, g);
    };
    float gain_of[8], gain_x_of[8], gate_of[8];
    if (CHUNKS == 1) {
        vector_of(p.gain, 0, gain_of);
        vector_of(p.gain_x, 0, gain_x_of);
        vector_of(p.gate_ld == 0 ? p.gate : nullptr, 0, gate_of);
    }
    // (where a row takes the whole workgroup the rows in turn are the same for all of its threads)
    int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + sub;
    if (kPipeline && row < count) load(row);
    for (; row < count; row += stride) {
        float t[CHUNKS][8], d[CHUNKS][8], r[CHUNKS][8], x[CHUNKS][8], g[CHUNKS][8];
        if (!kPipeline) load(row);
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
#pragma unroll
            for (int e = 0; e < 8; ++e) r[c][e] = t[c][e] = d[c][e] = 0;
            if (p.dy) {
                widen_8<TYPE>(t_raw[c].v, t[c]);
                widen_8<TYPE>(d_raw[c].v, d[c]);
            }
            if (p.dtotal) widen_8<TYPE>(r_raw[c].v, r[c]);
            widen_8<TYPE>(x_raw[c].v, x[c]);
            if (p.gate && p.gate_ld) widen_8<TYPE>(g_raw[c].v, g[c]);
            else if (CHUNKS > 1) vector_of(p.gate, c, g[c]);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) g[c][e] = gate_of[e];
        }
        if (kPipeline && row + stride < count) load(row + stride);
        float square = 0, dot = 0, square_x = 0;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            if (CHUNKS > 1) vector_of(p.gain, c, gain_of);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                square += t[c][e] * t[c][e];
                dot += t[c][e] * (d[c][e] * gain_of[e]);
                square_x += x[c][e] * x[c][e];
            }
        }
        RowFactors f{0, 0, 1};
        if (p.dy) {
            f.q = p.inv_rms ? p.inv_rms[row] : 1.0f / sqrtf(row_sum<LANES>(square, s) / p.width + p.eps);
            f.f = f.q * f.q * row_sum<LANES>(dot, s) / p.width;
        }
        if (p.norm_x) f.qx = p.inv_rms_x ? p.inv_rms_x[row] : 1.0f / sqrtf(row_sum<LANES>(square_x, s) / p.width + p.eps);
        float dot_x = 0;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int col = (c * LANES + lane) * 8, valid = p.width - col;
            if (CHUNKS > 1) {
                vector_of(p.gain, c, gain_of);
                vector_of(p.gain_x, c, gain_x_of);
            }
            const uint32_t kept = p.drop.threshold ? kept_8(p.drop, seed, row, col) : 0xffu;
            const GradOf8 o = grad_of_8(p, f, kept, t[c], d[c], r[c], x[c], gain_of, gain_x_of, g[c]);
            if (p.dresidual) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = p.residual_scale * o.dt[e];
                store_8_of<TYPE>(p.dresidual, row * p.dresidual_ld + col, valid, v);
            }
            if (p.dgate && p.gate_ld) store_8_of<TYPE>(p.dgate, row * p.dgate_ld + col, valid, o.slope);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sums[kSumGain][c][e] += d[c][e] * t[c][e] * f.q;
                sums[kSumGate][c][e] += o.slope[e];
                d[c][e] = o.w[e];
                if (p.norm_x) {
                    sums[kSumGainX][c][e] += o.w[e] * x[c][e] * f.qx;
                    d[c][e] *= gain_x_of[e];
                    dot_x += d[c][e] * x[c][e];
                }
            }
        }
        const float fx = p.norm_x ? f.qx * f.qx * row_sum<LANES>(dot_x, s) / p.width : 0.0f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int col = (c * LANES + lane) * 8;
            if (p.norm_x)
#pragma unroll
                for (int e = 0; e < 8; ++e) d[c][e] = f.qx * (d[c][e] - x[c][e] * fx);
            store_8_of<TYPE>(p.dx, row * p.dx_ld + col, p.width - col, d[c]);
        }
    }
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        if (!places.to[k]) continue;
        float* to = part + (static_cast<int64_t>(places.at[k]) * gridDim.x + blockIdx.x) * p.width;
        if (kRows == 1) {
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const int col = (c * LANES + lane) * 8;
                store_8_of<kF32>(to, col, p.width - col, sums[k][c]);
            }
            continue;
        }
        __syncthreads();
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) s_sum[sub][(c * LANES + lane) * 8 + e] = sums[k][c][e];
        __syncthreads();
        for (int col = threadIdx.x; col < p.width; col += kThreads) {
            float v = 0;
            for (int j = 0; j < kRows; ++j) v += s_sum[j][col];
            to[col] = v;
        }
    }
}

// Rows that are too wide for a workgroup's registers: it goes through a row three times, for the sums that need nothing, for the one
// that needs these, and for the results, and adds to its parts in memory.
constexpr int kWideThreads = 1024, kWideBlocks = 256;
template <int TYPE>
__global__ __launch_bounds__(kWideThreads) void join_grad_wide_kernel(JoinGradJob p, SumPlaces places, float* part) {
    __shared__ float s[kWideThreads / kWave];
    const int64_t count = p.rows.get();
    const uint64_t seed = drop_seed(p.drop);
    const auto part_of = [&](int k) { return part + (static_cast<int64_t>(places.at[k]) * gridDim.x + blockIdx.x) * p.width; };
    float zeros[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int k = 0; k < kSums; ++k)
        if (places.to[k])
            for (int col = threadIdx.x * 8; col < p.width; col += kWideThreads * 8) store_8_of<kF32>(part_of(k), col, p.width - col, zeros);
    const auto vector_of = [&](const void* v, int64_t at, int valid, float otherwise, float (&g)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = otherwise;
        if (v) load_8_of<TYPE>(v, at, valid, g);
    };
    for (int64_t row = blockIdx.x; row < count; row += gridDim.x) {
        float square = 0, dot = 0, square_x = 0;
        for (int col = threadIdx.x * 8; col < p.width; col += kWideThreads * 8) {
            const int valid = p.width - col;
            float t[8], d[8], x[8], gain[8];
            vector_of(p.dy ? p.total : nullptr, row * p.total_ld + col, valid, 0, t);
            vector_of(p.dy, row * p.dy_ld + col, valid, 0, d);
            vector_of(p.gain, col, valid, 1, gain);
            vector_of(p.x, row * p.x_ld + col, valid, 0, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                square += t[e] * t[e];
                dot += t[e] * (d[e] * gain[e]);
                square_x += x[e] * x[e];
            }
        }
        RowFactors f{0, 0, 1};
        if (p.dy) {
            f.q = p.inv_rms ? p.inv_rms[row] : 1.0f / sqrtf(row_sum<kWideThreads>(square, s) / p.width + p.eps);
            f.f = f.q * f.q * row_sum<kWideThreads>(dot, s) / p.width;
        }
        if (p.norm_x) f.qx = p.inv_rms_x ? p.inv_rms_x[row] : 1.0f / sqrtf(row_sum<kWideThreads>(square_x, s) / p.width + p.eps);
        float dot_x = 0, fx = 0;
        for (int pass = p.norm_x ? 0 : 1; pass < 2; ++pass) {
            for (int col = threadIdx.x * 8; col < p.width; col += kWideThreads * 8) {
                const int valid = p.width - col;
                float t[8], d[8], r[8], x[8], gain[8], gain_x[8], gate[8];
                vector_of(p.dy ? p.total : nullptr, row * p.total_ld + col, valid, 0, t);
                vector_of(p.dy, row * p.dy_ld + col, valid, 0, d);
                vector_of(p.dtotal, row * p.dtotal_ld + col, valid, 0, r);
                vector_of(p.x, row * p.x_ld + col, valid, 0, x);
                vector_of(p.gain, col, valid, 1, gain);
                vector_of(p.gain_x, col, valid, 1, gain_x);
                vector_of(p.gate, row * p.gate_ld + col, valid, 1, gate);
                const uint32_t kept = p.drop.threshold ? kept_8(p.drop, seed, row, col) : 0xffu;
                const GradOf8 o = grad_of_8(p, f, kept, t, d, r, x, gain, gain_x, gate);
                float out[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) out[e] = p.norm_x ? o.w[e] * gain_x[e] : o.w[e];
                if (pass == 0) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) dot_x += out[e] * x[e];
                    continue;
                }
                float sum[kSums][8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    sum[kSumGainX][e] = o.w[e] * x[e] * f.qx;
                    sum[kSumGain][e] = d[e] * t[e] * f.q;
                    sum[kSumGate][e] = o.slope[e];
                }
#pragma unroll
                for (int k = 0; k < kSums; ++k) {
                    if (!places.to[k]) continue;
                    float before[8];
                    load_8_of<kF32>(part_of(k), col, valid, before);
#pragma unroll
                    for (int e = 0; e < 8; ++e) before[e] += sum[k][e];
                    store_8_of<kF32>(part_of(k), col, valid, before);
                }
                if (p.dgate && p.gate_ld) store_8_of<TYPE>(p.dgate, row * p.dgate_ld + col, valid, o.slope);
                if (p.dresidual) {
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = p.residual_scale * o.dt[e];
                    store_8_of<TYPE>(p.dresidual, row * p.dresidual_ld + col, valid, v);
                }
                if (p.norm_x)
#pragma unroll
                    for (int e = 0; e < 8; ++e) out[e] = f.qx * (out[e] - x[e] * fx);
                store_8_of<TYPE>(p.dx, row * p.dx_ld + col, valid, out);
            }
            if (pass == 0) fx = f.qx * f.qx * row_sum<kWideThreads>(dot_x, s) / p.width;
        }
    }
}

__global__ __launch_bounds__(kBlock) void join_sum_kernel(SumPlaces places, const float* part, int n_parts, int32_t width, int type) {
    const int64_t each = static_cast<int64_t>(n_parts) * width;
    int k = 0;
    while (!places.to[k] || places.at[k] != static_cast<int>(blockIdx.y)) ++k;
    sum_columns(part + places.at[k] * each, n_parts, width, blockIdx.x * kSumColumns, places.to[k], type);
}

// The lanes and chunks for a row of `width` elements, as in the norm; in the gradient a lane has one chunk as long as it can, since it holds
// five rows and three sums of it.
template <int TYPE, class RUN>
auto join_by_width(int32_t width, RUN run) {
    if (width <= 128) return run.template go<TYPE, 16, 1>();
    if (width <= 512) return run.template go<TYPE, 64, 1>();
    if (width <= 1024) return run.template go<TYPE, 64, 2>();
    if (width <= 2048) return run.template go<TYPE, 256, 1>();
    if (width <= 8192) return run.template go<TYPE, 256, 4>();
    return run.template go<TYPE, 1024, 4>();
}
constexpr int32_t kMostInRegisters = 8192;
template <int TYPE, class RUN>
auto grad_by_width(int32_t width, RUN run) {
    if (width <= 128) return run.template go<TYPE, 16, 1>();
    if (width <= 512) return run.template go<TYPE, 64, 1>();
    if (width <= 1024) return run.template go<TYPE, 64, 2>();
    if (width <= 2048) return run.template go<TYPE, 256, 1>();
    if (width <= kMostInRegisters) return run.template go<TYPE, 1024, 1>();
    return run.template wide<TYPE>();
}

struct RunJoin {
    hipStream_t stream;
    JoinJob job;
    template <int TYPE, int LANES, int CHUNKS>
    hipError_t go() const {
        typedef RowShape<LANES> Shape;
        const unsigned blocks = static_cast<unsigned>(std::min<int64_t>((job.rows.host + Shape::kRows - 1) / Shape::kRows, kMostBlocks));
        hipLaunchKernelGGL((join_kernel<TYPE, LANES, CHUNKS>), dim3(blocks), dim3(Shape::kThreads), 0, stream, job);
        return hipGetLastError();
    }
};
struct JoinGradBlocks {                           // workgroups of the gradient
    int64_t rows;
    template <int TYPE, int LANES, int CHUNKS>
    unsigned go() const {
        typedef JoinGradShape<LANES, CHUNKS> Shape;
        return static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>((rows + Shape::kRows - 1) / Shape::kRows, Shape::kMostBlocks)));
    }
    template <int TYPE>
    unsigned wide() const {
        return static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>(rows, kWideBlocks)));
    }
};
unsigned join_grad_blocks(const JoinGradJob& job) { return grad_by_width<kF32>(job.width, JoinGradBlocks{job.rows.host}); }
struct RunJoinGrad {
    hipStream_t stream;
    JoinGradJob job;
    SumPlaces places;
    float* part;
    template <int TYPE, int LANES, int CHUNKS>
    hipError_t go() const {
        hipLaunchKernelGGL((join_grad_kernel<TYPE, LANES, CHUNKS>), dim3(join_grad_blocks(job)), dim3(JoinGradShape<LANES, CHUNKS>::kThreads), 0, stream, job,
                           places, part);
        return hipGetLastError();
    }
    template <int TYPE>
    hipError_t wide() const {
        hipLaunchKernelGGL((join_grad_wide_kernel<TYPE>), dim3(join_grad_blocks(job)), dim3(kWideThreads), 0, stream, job, places, part);
        return hipGetLastError();
    }
};

}  // namespace

hipError_t launch_dropout(hipStream_t stream, const DropoutJob& job) {
    if (job.rows.host < 1) return hipSuccess;
    const int64_t items = job.rows.host * ((job.width + 7) / 8);
    const unsigned blocks = static_cast<unsigned>(std::min<int64_t>((items + kBlock * kItems - 1) / (kBlock * kItems), kMostBlocks));
    if (job.type == kF32) hipLaunchKernelGGL(dropout_kernel<kF32>, dim3(blocks), dim3(kBlock), 0, stream, job);
    else if (job.type == kF16) hipLaunchKernelGGL(dropout_kernel<kF16>, dim3(blocks), dim3(kBlock), 0, stream, job);
    else hipLaunchKernelGGL(dropout_kernel<kBF16>, dim3(blocks), dim3(kBlock), 0, stream, job);
    return hipGetLastError();
}

hipError_t launch_join(hipStream_t stream, const JoinJob& job) {
    if (job.rows.host < 1) return hipSuccess;
    const RunJoin run{stream, job};
    if (job.x_type == kF32) return join_by_width<kF32>(job.width, run);
    if (job.x_type == kF16) return join_by_width<kF16>(job.width, run);
    return join_by_width<kBF16>(job.width, run);
}

size_t join_grad_scratch_bytes(const JoinGradJob& job) {
    return sizeof(float) * sums_of(job).n * join_grad_blocks(job) * static_cast<size_t>(job.width);
}

hipError_t launch_join_grad(hipStream_t stream, const JoinGradJob& job, void* scratch) {
    const SumPlaces places = sums_of(job);
    const RunJoinGrad run{stream, job, places, static_cast<float*>(scratch)};
    hipError_t e = job.type == kF32   ? grad_by_width<kF32>(job.width, run)
                   : job.type == kF16 ? grad_by_width<kF16>(job.width, run)
                                      : grad_by_width<kBF16>(job.width, run);
    if (e == hipSuccess && places.n > 0) {
        const unsigned columns = static_cast<unsigned>((job.width + kSumColumns - 1) / kSumColumns);
        hipLaunchKernelGGL(join_sum_kernel, dim3(columns, static_cast<unsigned>(places.n)), dim3(kBlock), 0, stream, places, run.part,
                           static_cast<int>(join_grad_blocks(job)), job.width, job.type);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace helios
