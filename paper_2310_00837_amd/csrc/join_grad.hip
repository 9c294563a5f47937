// Gradient of the join of a layer's output with the rows that went around the layer (join.hip).
//
//   with q and qx the reciprocal roots, a = dy * gain, and k = 1 where an element is kept, else 0, s = 1 / (1 - p):
//   dt = dtotal + q (a - total q^2 mean(a total));  dresidual = r dt;  dgate = s k dt x qx gain_x;  w = s k dt gate
//   dx = qx (w gain_x - x qx^2 mean(w gain_x x));  dgain_x = sum over rows of w x qx;  dgain = sum of dy total q
//
// (k = 0 selects: an element that is dropped adds 0 to these whatever is multiplied there.)
// With a gate of one row, dgate and dgain_x are one sum, S = sum over rows of k dt x qx: dgate = s gain_x S, dgain_x = s gate S.
// A row is held in registers in 32 bits and read once; lanes go through rows and keep their sums of columns until the end; a second launch adds the
// workgroups' sums.  26 624 rows of 512 in bfloat16 with a gate for all: 35 us, 31 and 4 for the second launch; 11 264 of 256 in single precision with
// a gate each: 24, of which 18 and 4.  In the first of these the main launch moves 5.3 TB/s, 0.83 of a copy's rate, and its vector instructions (376 for eight elements of a
// wave, of which the generator is a quarter) fill about half of its time: what is left is that a row's loads, two sums and stores follow one another.
// Registers are kept for a second workgroup on a CU and not for the next row (asked for ahead it took 24.7 us in place of 23.4 for
// 11 264 x 256 in single precision, 73.6 in place of 70 for 6000 x 4096 in bfloat16).  1024 threads, for 4097 to 8192 columns, have too few: 4 to 69 of
// them go to memory and back, and 2048 x 8192 takes 112 us in single precision, 62 in bfloat16, for 63 and 32 us of bytes.
#include "drop_dev.hpp"

#include <algorithm>

namespace helios {

namespace {

// What the sums over the rows are for: S (times gate_ld's matrix, if there is one) and that of dy total q.  Every workgroup has a row of parts for each
// that is asked for, at part + (its number * workgroups + workgroup) * width; join_sum_kernel adds them up.
enum Summed { kSumS = 0, kSumGain = 1, kSums = 2 };
struct SumPlaces {
    bool asked[kSums];
    int at[kSums];                                // its number among those that are asked for
    int n;
};
SumPlaces sums_of(const JoinGradJob& p) {
    SumPlaces s{{p.dgain_x || (p.dgate && p.gate_ld == 0), p.dgain != nullptr}, {0, 0}, 0};
    for (int k = 0; k < kSums; ++k)
        if (s.asked[k]) s.at[k] = s.n++;
    return s;
}

// What the sums over a row leave for its elements.
struct RowFactors {
    float q, f;                                   // 1 / rms of total, and q^2 times the mean of a total
    float qx;
};
// What becomes of eight elements before the sum over the row that dx needs.
struct GradOf8 {
    float dt[8];
    float w[8];                                   // w gain_x
};
// front: gain_x times s times the gate
__device__ __forceinline__ GradOf8 grad_of_8(const RowFactors& r, const Kept8& kept, const float (&t)[8], const float (&dy)[8], const float (&dtotal)[8],
                                             const float (&x)[8], const float (&gain)[8], const float (&front)[8]) {
    GradOf8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        o.dt[e] = __builtin_fmaf(r.q, __builtin_fmaf(-t[e], r.f, dy[e] * gain[e]), dtotal[e]);
        o.w[e] = kept.on[e] ? o.dt[e] * front[e] : 0.0f;
    }
    return o;
}

// Threads and rows of a workgroup: up to a wave several rows, else the workgroup has one.
template <int LANES>
struct GradShape {
    static constexpr int kThreads = LANES <= kWave ? 512 : LANES;
    static constexpr int kRows = kThreads / LANES;
    static constexpr int kMostBlocks = 256 * 1024 / kThreads;             // (about four waves for a SIMD)
};
// A lane beyond the last chunk loads what is there, too, and adds nothing to the sums over a row.
// WITH: what there is, where that is known: branches for it cost copies of what is loaded, and registers for a gate's rows that there are none of
// (26 624 x 512 in bfloat16, without the second launch: 43 us with them, 35 without, before its rows were streamed).
enum With { kWithAny = 0, kWithOneGate = 1, kWithGates = 2 };       // any; dy, dtotal, and a gate of one row or none; dy, dtotal and a gate for every row
template <int TYPE, int LANES, int ROWS, int WITH>
__global__ __launch_bounds__(GradShape<LANES>::kThreads) void join_grad_kernel(JoinGradJob p, SumPlaces places, float* part) {
    constexpr int kThreads = GradShape<LANES>::kThreads, kRows = GradShape<LANES>::kRows, kWidth = LANES * 8;
    constexpr bool kBoth = WITH != kWithAny;
    // Where a row's columns are added up, which decides what 1024 threads have no registers for: both sums after everything else, 2048 rows of 8191 in bfloat16 77 us,
    // that for dgain before the last sum over the row, 86; the other types and widths the other way about (8191 in single precision 125 and 116, 8192 in
    // bfloat16 without dtotal 116 and 100).
    constexpr bool kGainLast = TYPE == kBF16 && ROWS == kRowsWithRest;
    const bool gates = WITH == kWithGates || (WITH == kWithAny && p.gate_ld != 0);
    __shared__ float s3[2][3][RowSums<LANES, 3>::kWaves], s1[2][1][RowSums<LANES, 1>::kWaves];
    __shared__ float s_sum[kRows > 1 ? kRows : 1][kRows > 1 ? kWidth : 1];
    RowSums<LANES, 3> first_sums{s3};
    RowSums<LANES, 1> last_sum{s1};
    const int64_t count = p.rows.get(), stride = static_cast<int64_t>(gridDim.x) * kRows;
    const uint64_t seed = drop_seed(p.drop);
    const float per = 1.0f / static_cast<float>(p.width);
    const int lane = threadIdx.x % LANES, sub = row_of_lanes<LANES>();
    const int32_t col = lane * 8;
    const bool in = col < p.width;
    const auto load = [&](Raw8<TYPE>& to, const void* base, int64_t at) { to.template load_row<ROWS>(base, at, col, p.width); };
    const auto widen = [&](Raw8<TYPE>& raw, float (&v)[8]) {
        raw.template align<ROWS>(col, p.width);
        widen_8<TYPE>(raw.v, v);
    };
    Raw8<TYPE> t_raw, d_raw, r_raw, x_raw, g_raw;
    if (!kBoth) t_raw.clear(), d_raw.clear(), r_raw.clear();
    const auto load_row = [&](int64_t row) {
        load(x_raw, p.x, row * p.x_ld);
        if (kBoth || p.dy) {
            load(t_raw, p.total, row * p.total_ld);
            load(d_raw, p.dy, row * p.dy_ld);
        }
        if (kBoth || p.dtotal) load(r_raw, p.dtotal, row * p.dtotal_ld);
        if (gates) load(g_raw, p.gate, row * p.gate_ld);
    };
    const auto load_vector = [&](const void* v, float (&to)[8]) {
        if (!v) return;
        Raw8<TYPE> raw;
        float f[8];
        load(raw, v, 0);
        widen(raw, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) to[e] *= f[e];
    };
    float gain[8], front[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) gain[e] = 1, front[e] = p.drop.scale;
    load_vector(p.gain, gain);
    load_vector(p.gain_x, front);
    if (!gates) load_vector(p.gate, front);
    float sum_s[8] = {0, 0, 0, 0, 0, 0, 0, 0}, sum_gain[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * kRows; first < count; first += stride) {
        const bool there = kRows == 1 || first + sub < count;
        const int64_t row = there ? first + sub : count - 1;
        load_row(row);
        float t[8], d[8], r[8], x[8], g[8], whole_front[8];
        widen(t_raw, t);
        widen(d_raw, d);
        widen(r_raw, r);
        widen(x_raw, x);
        if (gates) widen(g_raw, g);
        // (the elements that are kept have nothing to do with the loads)
        const Kept8 kept = kept_8(p.drop, seed, row, col);
        float v3[3] = {0, 0, 0};                    // squares of total, of x; a total
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v3[0] += t[e] * t[e];
            v3[1] += x[e] * x[e];
            v3[2] += d[e] * t[e] * gain[e];
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) v3[k] = in ? v3[k] : 0.0f;
        first_sums.run(v3);
        RowFactors f{0, 0, 1};
        if (kBoth || p.dy) {
            f.q = p.inv_rms ? p.inv_rms[row] : rsqrtf(v3[0] * per + p.eps);
            f.f = v3[2] * per * f.q * f.q;
        }
        if (p.norm_x) f.qx = p.inv_rms_x ? p.inv_rms_x[row] : rsqrtf(v3[1] * per + p.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) whole_front[e] = gates ? front[e] * g[e] : front[e];
        const GradOf8 o = grad_of_8(f, kept, t, d, r, x, gain, whole_front);
        float v1[1] = {0};
#pragma unroll
        for (int e = 0; e < 8; ++e) v1[0] += o.w[e] * x[e];
        const auto add_gain = [&] {
#pragma unroll
            for (int e = 0; e < 8; ++e) sum_gain[e] += d[e] * t[e] * f.q;
        };
        if (p.dresidual && there) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = p.residual_scale * o.dt[e];
            store_row_8<TYPE, ROWS>(p.dresidual, row * p.dresidual_ld, col, p.width, v);
        }
        if (p.dgate && gates && there) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = kept.on[e] ? o.dt[e] * x[e] * (f.qx * front[e]) : 0.0f;
            store_row_8<TYPE, ROWS>(p.dgate, row * p.dgate_ld, col, p.width, v);
        }
        if (!kGainLast && there) add_gain();
        float out[8];
        if (p.norm_x) {
            v1[0] = in ? v1[0] : 0.0f;
            last_sum.run(v1);
            const float fx = v1[0] * per * f.qx * f.qx;
#pragma unroll
            for (int e = 0; e < 8; ++e) out[e] = f.qx * (o.w[e] - x[e] * fx);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) out[e] = o.w[e];
        }
        if (kGainLast && there) add_gain();
        if (there)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum_s[e] += kept.on[e] ? o.dt[e] * x[e] * (gates ? g[e] * f.qx : f.qx) : 0.0f;
        if (there) store_row_8<TYPE, ROWS>(p.dx, row * p.dx_ld, col, p.width, out);
    }
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        if (!places.asked[k]) continue;
        const float(&sum)[8] = k == kSumS ? sum_s : sum_gain;
        float* to = part + (static_cast<int64_t>(places.at[k]) * gridDim.x + blockIdx.x) * p.width;
        if (kRows == 1) {
            store_row_8<kF32, ROWS>(to, 0, col, p.width, sum);
            continue;
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) s_sum[sub][col + e] = sum[e];
        __syncthreads();
        for (int c = threadIdx.x; c < p.width; c += kThreads) {
            float v = 0;
#pragma unroll
            for (int j = 0; j < kRows; ++j) v += s_sum[j][c];
            to[c] = v;
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
    const float per = 1.0f / static_cast<float>(p.width);
    const auto part_of = [&](int k) { return part + (static_cast<int64_t>(places.at[k]) * gridDim.x + blockIdx.x) * p.width; };
    const float zeros[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int k = 0; k < kSums; ++k)
        if (places.asked[k])
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
                dot += d[e] * t[e] * gain[e];
                square_x += x[e] * x[e];
            }
        }
        RowFactors f{0, 0, 1};
        if (p.dy) {
            f.q = p.inv_rms ? p.inv_rms[row] : rsqrtf(row_sum<kWideThreads>(square, s) * per + p.eps);
            f.f = row_sum<kWideThreads>(dot, s) * per * f.q * f.q;
        }
        if (p.norm_x) f.qx = p.inv_rms_x ? p.inv_rms_x[row] : rsqrtf(row_sum<kWideThreads>(square_x, s) * per + p.eps);
        float dot_x = 0, fx = 0;
        for (int pass = p.norm_x ? 0 : 1; pass < 2; ++pass) {
            for (int col = threadIdx.x * 8; col < p.width; col += kWideThreads * 8) {
                const int valid = p.width - col;
                float t[8], d[8], r[8], x[8], gain[8], front[8], gate[8];
                vector_of(p.dy ? p.total : nullptr, row * p.total_ld + col, valid, 0, t);
                vector_of(p.dy, row * p.dy_ld + col, valid, 0, d);
                vector_of(p.dtotal, row * p.dtotal_ld + col, valid, 0, r);
                vector_of(p.x, row * p.x_ld + col, valid, 0, x);
                vector_of(p.gain, col, valid, 1, gain);
                vector_of(p.gain_x, col, valid, 1, front);
                vector_of(p.gate, row * p.gate_ld + col, valid, 1, gate);
                float whole_front[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    front[e] *= p.drop.scale;
                    whole_front[e] = front[e] * gate[e];
                }
                const Kept8 kept = kept_8(p.drop, seed, row, col);
                const GradOf8 o = grad_of_8(f, kept, t, d, r, x, gain, whole_front);
                if (pass == 0) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) dot_x += o.w[e] * x[e];
                    continue;
                }
                float sum[kSums][8], v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    sum[kSumS][e] = kept.on[e] ? o.dt[e] * x[e] * (p.gate_ld ? gate[e] * f.qx : f.qx) : 0.0f;
                    sum[kSumGain][e] = d[e] * t[e] * f.q;
                }
#pragma unroll
                for (int k = 0; k < kSums; ++k) {
                    if (!places.asked[k]) continue;
                    load_8_of<kF32>(part_of(k), col, valid, v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] += sum[k][e];
                    store_8_of<kF32>(part_of(k), col, valid, v);
                }
                if (p.dgate && p.gate_ld) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = kept.on[e] ? o.dt[e] * x[e] * (f.qx * front[e]) : 0.0f;
                    store_8_of<TYPE>(p.dgate, row * p.dgate_ld + col, valid, v);
                }
                if (p.dresidual) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = p.residual_scale * o.dt[e];
                    store_8_of<TYPE>(p.dresidual, row * p.dresidual_ld + col, valid, v);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = p.norm_x ? f.qx * (o.w[e] - x[e] * fx) : o.w[e];
                store_8_of<TYPE>(p.dx, row * p.dx_ld + col, valid, v);
            }
            if (pass == 0) fx = row_sum<kWideThreads>(dot_x, s) * per * f.qx * f.qx;
        }
    }
}

// The workgroups' sums, and what they are multiplied by: see above.
template <int TYPE>
__global__ __launch_bounds__(kBlock) void join_sum_kernel(JoinGradJob p, SumPlaces places, const float* part, int n_parts) {
    const bool of_s = places.asked[kSumS] && blockIdx.y == 0;
    const float* from = part + static_cast<int64_t>(blockIdx.y) * n_parts * p.width;
    sum_columns(from, n_parts, p.width, blockIdx.x * kSumColumns, [&](int32_t col, float v) {
        if (!of_s) {
            store_1(TYPE, p.dgain, col, v);
            return;
        }
        v *= p.drop.scale;
        if (p.dgate && !p.gate_ld) store_1(TYPE, p.dgate, col, p.gain_x ? v * load_1<TYPE>(p.gain_x, col) : v);
        if (p.dgain_x) store_1(TYPE, p.dgain_x, col, p.gate && !p.gate_ld ? v * load_1<TYPE>(p.gate, col) : v);
    });
}

constexpr int32_t kMostInRegisters = 8192;
template <int TYPE, int ROWS, int WITH, class RUN>
auto by_width(int32_t width, RUN run) {
    if (width <= 128) return run.template go<TYPE, 16, ROWS, WITH>();
    if (width <= 512) return run.template go<TYPE, 64, ROWS, WITH>();
    if (width <= 1024) return run.template go<TYPE, 128, ROWS, WITH>();
    if (width <= 2048) return run.template go<TYPE, 256, ROWS, WITH>();
    if (width <= 4096) return run.template go<TYPE, 512, ROWS, WITH>();
    if (width <= kMostInRegisters) return run.template go<TYPE, 1024, ROWS, WITH>();
    return run.template wide<TYPE>();
}
struct GradBlocks {                               // workgroups of the gradient
    int64_t rows;
    template <int TYPE, int LANES, int ROWS, int WITH>
    unsigned go() const {
        typedef GradShape<LANES> Shape;
        return static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>((rows + Shape::kRows - 1) / Shape::kRows, Shape::kMostBlocks)));
    }
    template <int TYPE>
    unsigned wide() const {
        return static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>(rows, kWideBlocks)));
    }
};
unsigned blocks_of(const JoinGradJob& job) { return by_width<kF32, kWholeRows, kWithAny>(job.width, GradBlocks{job.rows.host}); }
struct RunGrad {
    hipStream_t stream;
    JoinGradJob job;
    SumPlaces places;
    float* part;
    template <int TYPE, int LANES, int ROWS, int WITH>
    hipError_t go() const {
        hipLaunchKernelGGL((join_grad_kernel<TYPE, LANES, ROWS, WITH>), dim3(blocks_of(job)), dim3(GradShape<LANES>::kThreads), 0, stream, job, places, part);
        return hipGetLastError();
    }
    template <int TYPE>
    hipError_t wide() const {
        hipLaunchKernelGGL((join_grad_wide_kernel<TYPE>), dim3(blocks_of(job)), dim3(kWideThreads), 0, stream, job, places, part);
        return hipGetLastError();
    }
    template <int TYPE, int ROWS>
    hipError_t with() const {
        if (!job.dy || !job.dtotal) return by_width<TYPE, ROWS, kWithAny>(job.width, *this);
        return job.gate_ld ? by_width<TYPE, ROWS, kWithGates>(job.width, *this) : by_width<TYPE, ROWS, kWithOneGate>(job.width, *this);
    }
    template <int TYPE>
    hipError_t all() const {
        const int arrays = 2 + 2 * (job.dy != nullptr) + (job.dtotal != nullptr) + (job.gate_ld != 0) + (job.dgate && job.gate_ld) + (job.dresidual != nullptr);
        const Rows rows = rows_of(job.width, job.rows.host * job.width * arrays * type_bytes(TYPE));
        const hipError_t e = rows == kShortRows ? go<TYPE, 16, kShortRows, kWithAny>()
                           : rows == kRowsWithRest ? with<TYPE, kRowsWithRest>()
                           : rows == kStreamedRows ? with<TYPE, kStreamedRows>()
                           : with<TYPE, kWholeRows>();
        if (e != hipSuccess || places.n == 0) return e;
        const dim3 grid(static_cast<unsigned>((job.width + kSumColumns - 1) / kSumColumns), static_cast<unsigned>(places.n));
        hipLaunchKernelGGL(join_sum_kernel<TYPE>, grid, dim3(kBlock), 0, stream, job, places, part, static_cast<int>(blocks_of(job)));
        return hipGetLastError();
    }
};

}  // namespace

size_t join_grad_scratch_bytes(const JoinGradJob& job) { return sizeof(float) * sums_of(job).n * blocks_of(job) * static_cast<size_t>(job.width); }

hipError_t launch_join_grad(hipStream_t stream, const JoinGradJob& job, void* scratch) {
    const RunGrad run{stream, job, sums_of(job), static_cast<float*>(scratch)};
    return job.type == kF32 ? run.all<kF32>() : job.type == kF16 ? run.all<kF16>() : run.all<kBF16>();
}

}  // namespace helios
