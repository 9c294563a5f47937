// Root-mean-square norm of rows, with the addition of a residual in front of it and, for the products in 8 bits behind it,
// an output in e4m3 with a scale for every row; and its gradient.
//
//   t = x + residual;  y = t * gain / sqrt(mean(t^2) + eps)
//   8 bits: scale = max(max|y| / 448, 2^-126), y8 = e4m3(y / scale)
//   gradient, with q = 1 / sqrt(mean(t^2) + eps) and u = dy * gain:
//   dx = dtotal + q (u - t q^2 mean(u t));  dgain = sum over rows of dy t q
//
// A row is held in the registers of the lanes that share it, in 32 bits, so that it is read once and every output is made
// from the unrounded sums.  What bounds it is memory: one pass over what has to be read and written.  100 003 x 1024 in half
// precision with residual, sum and 8-bit output: 128 us for 717 MB, 5.6 TB/s (a plain copy reaches 6.4); the gradient of
// 26 624 x 512 in bfloat16 with dtotal and dgain: 26 us for 109 MB, of which the join of dgain's parts is 5; 1024 x 256 in single
// precision 4 us of kernel, a launch and a trip to memory.
#include "layer.hpp"
#include "layer_dev.hpp"

#include <algorithm>

namespace helios {

namespace {

constexpr int64_t kMostBlocks = 1 << 21;            // of a launch
constexpr float kE4M3Max = 448.0f, kMinScale = 0x1p-126f;

// Lanes that share a row: LANES (a power of two), each with CHUNKS times eight elements; up to a wave several rows to a workgroup, else
// the workgroup has one.
template <int LANES>
struct RowShape {
    static constexpr int kThreads = LANES > kBlock ? LANES : kBlock;
    static constexpr int kRows = kThreads / LANES;
};
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float* s) {
    v = group_sum<(LANES < kWave ? LANES : kWave)>(v);
    if (LANES > kWave) {
        constexpr int kWaves = LANES / kWave;
        __syncthreads();
        if (lane_id() == 0) s[wave_id()] = v;
        __syncthreads();
        v = 0;
        const int first = wave_id() / kWaves * kWaves;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v += s[first + w];
    }
    return v;
}
template <int LANES>
__device__ __forceinline__ float row_max(float v, float* s) {
    v = group_max<(LANES < kWave ? LANES : kWave)>(v);
    if (LANES > kWave) {
        constexpr int kWaves = LANES / kWave;
        __syncthreads();
        if (lane_id() == 0) s[wave_id()] = v;
        __syncthreads();
        const int first = wave_id() / kWaves * kWaves;
        v = s[first];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) {
            const float o = s[first + w];
            v = o > v || o != o ? o : v;
        }
    }
    return v;
}

__device__ __forceinline__ void store_8_of_e4m3(void* base, int64_t at, int valid, const float (&v)[8]) {
    typedef int32_t i32x2_any __attribute__((ext_vector_type(2), aligned(1)));
    int32_t w[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        w[k] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * k], v[4 * k + 1], 0, false);
        w[k] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * k + 2], v[4 * k + 3], w[k], true);
    }
    uint8_t* p = static_cast<uint8_t*>(base) + at;
    if (valid >= 8) {
        *reinterpret_cast<i32x2_any*>(p) = i32x2_any{w[0], w[1]};
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < valid) p[e] = static_cast<uint8_t>(static_cast<uint32_t>(w[e / 4]) >> (8 * (e % 4)));
}

template <int TYPE, int LANES, int CHUNKS>
__device__ __forceinline__ void norm_row(const NormJob& p, int64_t row, int lane, float* s) {
    float t[CHUNKS][8];
    float sum = 0;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int col = (c * LANES + lane) * 8, valid = p.width - col;
        load_8_of<TYPE>(p.x, row * p.x_ld + col, valid, t[c]);
        if (p.residual) {
            float r[8];
            load_8_of<TYPE>(p.residual, row * p.residual_ld + col, valid, r);
#pragma unroll
            for (int e = 0; e < 8; ++e) t[c][e] += r[e];
        }
        if (p.total) store_8_of<TYPE>(p.total, row * p.total_ld + col, valid, t[c]);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += t[c][e] * t[c][e];
    }
    if (p.normalise) {
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
    }
    if (!p.y_scale) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int col = (c * LANES + lane) * 8;
            store_8_of<TYPE>(p.y, row * p.y_ld + col, p.width - col, t[c]);
        }
        return;
    }
    float most = 0;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float a = fabsf(t[c][e]);
            most = a > most || a != a ? a : most;
        }
    most = row_max<LANES>(most, s) / kE4M3Max;
    // (y / scale, correctly rounded, by way of the reciprocal and one step of Newton's: by the reciprocal alone a quotient can fall to the wrong
    // side of the middle between two values of 8 bits.  An infinite scale leaves 0 of what is finite.)
    const float scale = most < kMinScale ? kMinScale : most, inv = 1.0f / scale;
    if (lane == 0) p.y_scale[row] = scale;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int col = (c * LANES + lane) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float near = t[c][e] * inv;     // t / scale, but for its last bit
            t[c][e] = inv > 0.0f ? __builtin_fmaf(__builtin_fmaf(-near, scale, t[c][e]), inv, near) : near;
        }
        store_8_of_e4m3(p.y, row * p.y_ld + col, p.width - col, t[c]);
    }
}

template <int TYPE, int LANES, int CHUNKS>
__global__ __launch_bounds__(RowShape<LANES>::kThreads) void norm_kernel(NormJob p) {
    constexpr int kThreads = RowShape<LANES>::kThreads, kRows = RowShape<LANES>::kRows;
    __shared__ float s[kThreads / kWave];
    const int64_t count = p.rows.get();
    const int lane = threadIdx.x % LANES;
    for (int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / LANES; row < count; row += static_cast<int64_t>(gridDim.x) * kRows)
        norm_row<TYPE, LANES, CHUNKS>(p, row, lane, s);
}

// A workgroup of the gradient: with one chunk to a lane, as many rows at a time as fit 1024 threads, so that there are few sums of
// dgain to be added up.
template <int LANES, int CHUNKS>
struct GradShape {
    static constexpr int kThreads = LANES <= kWave && CHUNKS == 1 ? 1024 : RowShape<LANES>::kThreads, kRows = kThreads / LANES;
    static constexpr int kMostBlocks = kThreads == 1024 ? 256 : 1024;
};
// Every workgroup goes through rows blockIdx.x * kRows + ..., asks for a row while the one before it is worked on (rows of up to
// eight elements a lane: more would not fit the registers), and keeps its lanes' sums for dgain until the end.
template <int TYPE, int LANES, int CHUNKS>
__global__ __launch_bounds__((GradShape<LANES, CHUNKS>::kThreads)) void norm_grad_kernel(NormGradJob p, float* part) {
    constexpr int kThreads = GradShape<LANES, CHUNKS>::kThreads, kRows = GradShape<LANES, CHUNKS>::kRows, kWidth = LANES * CHUNKS * 8;
    constexpr bool kPipeline = CHUNKS == 1;
    __shared__ float s[kThreads / kWave];
    __shared__ float s_gain[kRows > 1 ? kRows : 1][kRows > 1 ? kWidth : 1];
    const int64_t count = p.rows.get(), stride = static_cast<int64_t>(gridDim.x) * kRows;
    const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES;
    float dg[CHUNKS][8];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) dg[c][e] = 0;
    Raw8<TYPE> t_raw[CHUNKS], d_raw[CHUNKS], r_raw[CHUNKS];
    const auto load = [&](int64_t row) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int col = (c * LANES + lane) * 8, valid = p.width - col;
            t_raw[c].load(p.total, row * p.total_ld + col, valid);
            d_raw[c].load(p.dy, row * p.dy_ld + col, valid);
            if (kPipeline && p.dtotal) r_raw[c].load(p.dtotal, row * p.dtotal_ld + col, valid);
        }
    };
    float gain[8] = {1, 1, 1, 1, 1, 1, 1, 1};
    if (kPipeline && p.gain) load_8_of<TYPE>(p.gain, lane * 8, p.width - lane * 8, gain);
    const auto gain_of = [&](int c, float (&g)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = gain[e];
        if (!kPipeline && p.gain) load_8_of<TYPE>(p.gain, (c * LANES + lane) * 8, p.width - (c * LANES + lane) * 8, g);
    };
    // (where a row takes the whole workgroup the rows in turn are the same for all of its threads)
    int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + sub;
    if (kPipeline && row < count) load(row);
    for (; row < count; row += stride) {
        float t[CHUNKS][8], d[CHUNKS][8], r[8];
        if (!kPipeline) load(row);
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            widen_8<TYPE>(t_raw[c].v, t[c]);
            widen_8<TYPE>(d_raw[c].v, d[c]);
            if (kPipeline && p.dtotal) widen_8<TYPE>(r_raw[c].v, r);
        }
        if (kPipeline && row + stride < count) load(row + stride);
        float square = 0, dot = 0;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            float g[8];
            gain_of(c, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) square += t[c][e] * t[c][e], dot += t[c][e] * d[c][e] * g[e];
        }
        dot = row_sum<LANES>(dot, s);
        const float q = p.inv_rms ? p.inv_rms[row] : 1.0f / sqrtf(row_sum<LANES>(square, s) / p.width + p.eps);
        const float f = q * q * dot / p.width;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int col = (c * LANES + lane) * 8, valid = p.width - col;
            float g[8], out[8];
            gain_of(c, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dg[c][e] += d[c][e] * t[c][e] * q;
                out[e] = q * (d[c][e] * g[e] - t[c][e] * f);
            }
            if (p.dtotal) {
                if (!kPipeline) load_8_of<TYPE>(p.dtotal, row * p.dtotal_ld + col, valid, r);
#pragma unroll
                for (int e = 0; e < 8; ++e) out[e] += r[e];
            }
            store_8_of<TYPE>(p.dx, row * p.dx_ld + col, valid, out);
        }
    }
    if (!p.dgain) return;
    float* to = part + static_cast<int64_t>(blockIdx.x) * p.width;
    if (kRows == 1) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int col = (c * LANES + lane) * 8;
            store_8_of<kF32>(to, col, p.width - col, dg[c]);
        }
        return;
    }
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) s_gain[sub][(c * LANES + lane) * 8 + e] = dg[c][e];
    __syncthreads();
    for (int col = threadIdx.x; col < p.width; col += kThreads) {
        float v = 0;
        for (int k = 0; k < kRows; ++k) v += s_gain[k][col];
        to[col] = v;
    }
}

__global__ __launch_bounds__(kBlock) void gain_sum_kernel(const float* part, int n_parts, int32_t width, void* out, int type) {
    sum_columns(part, n_parts, width, blockIdx.x * kSumColumns, out, type);
}

// The lanes and chunks for a row of `width` elements: sixteen lanes or a wave, whose sums need no LDS, while a lane has at most two chunks, then a
// workgroup.  Widths far below a shape's most leave lanes idle (of 256 elements half the wave, of 1032 half the workgroup), which
// short rows hide behind the launch and long lists behind memory.
template <int TYPE, class RUN>
auto by_width(int32_t width, RUN run) {
    if (width <= 128) return run.template go<TYPE, 16, 1>();
    if (width <= 512) return run.template go<TYPE, 64, 1>();
    if (width <= 1024) return run.template go<TYPE, 64, 2>();
    if (width <= 2048) return run.template go<TYPE, 256, 1>();
    if (width <= 8192) return run.template go<TYPE, 256, 4>();
    return run.template go<TYPE, 1024, 4>();
}
template <class RUN>
hipError_t by_type(int type, int32_t width, RUN run) {
    if (type == kF32) return by_width<kF32>(width, run);
    if (type == kF16) return by_width<kF16>(width, run);
    return by_width<kBF16>(width, run);
}

struct RunNorm {
    hipStream_t stream;
    NormJob job;
    template <int TYPE, int LANES, int CHUNKS>
    hipError_t go() const {
        typedef RowShape<LANES> Shape;
        const unsigned blocks = static_cast<unsigned>(std::min<int64_t>((job.rows.host + Shape::kRows - 1) / Shape::kRows, kMostBlocks));
        hipLaunchKernelGGL((norm_kernel<TYPE, LANES, CHUNKS>), dim3(blocks), dim3(Shape::kThreads), 0, stream, job);
        return hipGetLastError();
    }
};
struct GradBlocks {                               // workgroups of the gradient
    int64_t rows;
    template <int TYPE, int LANES, int CHUNKS>
    unsigned go() const {
        typedef GradShape<LANES, CHUNKS> Shape;
        return static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>((rows + Shape::kRows - 1) / Shape::kRows, Shape::kMostBlocks)));
    }
};
struct RunGrad {
    hipStream_t stream;
    NormGradJob job;
    float* part;
    template <int TYPE, int LANES, int CHUNKS>
    hipError_t go() const {
        const unsigned blocks = GradBlocks{job.rows.host}.go<TYPE, LANES, CHUNKS>();
        hipLaunchKernelGGL((norm_grad_kernel<TYPE, LANES, CHUNKS>), dim3(blocks), dim3(GradShape<LANES, CHUNKS>::kThreads), 0, stream, job, part);
        return hipGetLastError();
    }
};

}  // namespace

hipError_t launch_norm(hipStream_t stream, const NormJob& job) {
    if (job.rows.host < 1) return hipSuccess;
    return by_type(job.x_type, job.width, RunNorm{stream, job});
}

size_t norm_grad_scratch_bytes(const NormGradJob& job) {
    return job.dgain ? sizeof(float) * by_width<kF32>(job.width, GradBlocks{job.rows.host}) * static_cast<size_t>(job.width) : 0;
}

hipError_t launch_norm_grad(hipStream_t stream, const NormGradJob& job, void* scratch) {
    float* part = static_cast<float*>(scratch);
    hipError_t e = by_type(job.type, job.width, RunGrad{stream, job, part});
    if (e == hipSuccess && job.dgain) {
        const unsigned blocks = static_cast<unsigned>((job.width + kSumColumns - 1) / kSumColumns);
        hipLaunchKernelGGL(gain_sum_kernel, dim3(blocks), dim3(kBlock), 0, stream, part, static_cast<int>(by_width<kF32>(job.width, GradBlocks{job.rows.host})), job.width, job.dgain, job.type);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace helios
