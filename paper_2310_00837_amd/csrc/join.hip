// Dropout, and the join of a layer's output with the rows that went around the layer.
//
//   u = x * gain_x / sqrt(mean(x^2) + eps);  total = r * residual + gate * drop(u);  y = total * gain / sqrt(mean(total^2) + eps)
//
// A row is held in the registers of the lanes that share it, in 32 bits, as in the norm: both norms, the dropped elements and
// the 8-bit output are one pass over what has to be read and written, with two sums over the row, the second of which needs the first.
// Lanes go through rows and ask for the next one while they work on this one; what is the same for all rows stays in registers.
// What bounds it is memory, and the vector unit close behind: 100 003 rows of 1024 in half precision with both norms, a gate, dropout and both outputs
// are 144 us, 5.7 TB/s, for which each of a row's two waves issues 282 vector instructions, of which the generator is a third.
// Rows of more than 8192 columns are more than the registers hold: 50 to 182 of them go to memory and back, and 2046 rows of 8200, which pay for the lanes of 32 768,
// take 323 us in single precision and 196 in bfloat16, where 2048 of 8192 take 82 and 40.
#include "drop_dev.hpp"

#include <algorithm>

namespace helios {

namespace {

constexpr int64_t kMostBlocks = 1 << 21;            // of a launch
constexpr int kItems = 2;                           // of a thread of the dropout kernel, in flight together

// An item is eight neighbouring columns of a row; items are numbered along the rows.  Bound by memory and the generator: 26 624 rows of 512 in bfloat16
// 10.6 us, 5.1 TB/s, 100 003 of 1024 in
// half precision 64 us, 6.4 TB/s, what a large copy reaches.
template <int TYPE, int ROWS>
__global__ __launch_bounds__(kBlock) void dropout_kernel(DropoutJob p) {
    const uint32_t blocks = static_cast<uint32_t>(p.width + 7) / 8;
    const int64_t items = p.rows.get() * blocks, step = static_cast<int64_t>(gridDim.x) * kBlock * kItems;
    const uint64_t seed = drop_seed(p.drop);
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * kBlock * kItems; base < items; base += step) {
        const ItemPlaces places(base, blocks);
        const uint32_t left = items - base < kBlock * kItems ? static_cast<uint32_t>(items - base) : kBlock * kItems;
        Raw8<TYPE> raw[kItems];
        uint32_t down[kItems];
        int32_t col[kItems];
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            const uint32_t i = k * kBlock + threadIdx.x;
            places.get(i < left ? i : left - 1, &down[k], &col[k]);
            raw[k].template load_row<ROWS>(p.x, places.row(p.x_ld, down[k]), col[k], p.width);
        }
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            float v[8];
            const Kept8 kept = kept_8(p.drop, seed, places.row0 + down[k], col[k]);
            raw[k].template align<ROWS>(col[k], p.width);
            widen_8<TYPE>(raw[k].v, v);
            // (what is dropped becomes 0 whatever it was: no product)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = kept.on[e] ? v[e] * p.drop.scale : 0.0f;
            if (k * kBlock + threadIdx.x < left) store_row_8<TYPE, ROWS>(p.y, places.row(p.y_ld, down[k]), col[k], p.width, v);
        }
    }
}

// A lane beyond the last chunk loads what is there, too, and adds nothing to the sums.
// GATES: there is a gate for every row (in rows that are no whole chunks of eight: there may be).
template <int LANES>
struct JoinShape {                                  // up to a wave several rows to a workgroup, else the workgroup has one
    static constexpr int kThreads = LANES <= kWave ? kBlock : LANES, kRows = kThreads / LANES;
};
template <int TYPE, int LANES, int CHUNKS, int ROWS, bool GATES>
__global__ __launch_bounds__(JoinShape<LANES>::kThreads) void join_kernel(JoinJob p) {
    constexpr int kThreads = JoinShape<LANES>::kThreads, kRows = JoinShape<LANES>::kRows;
    const bool gates = GATES || ((ROWS == kRowsWithRest || ROWS == kShortRows) && p.gate_ld != 0);
    constexpr bool kKeep = LANES * CHUNKS <= 1024;      // registers for the next row and what is the same for all (1024 threads with more have none)
    __shared__ float s[kThreads / kWave];
    __shared__ float s_sums[2][1][RowSums<LANES, 1>::kWaves];
    RowSums<LANES, 1> sums{s_sums};
    const auto whole_sum = [&](float v) {
        float one[1] = {v};
        sums.run(one);
        return one[0];
    };
    const int64_t count = p.rows.get(), stride = static_cast<int64_t>(gridDim.x) * kRows;
    const uint64_t seed = drop_seed(p.drop);
    const float per = 1.0f / static_cast<float>(p.width);
    const int lane = threadIdx.x % LANES, sub = row_of_lanes<LANES>();
    Raw8<TYPE> x_raw[CHUNKS], r_raw[CHUNKS], g_raw[CHUNKS];
    const auto load = [&](Raw8<TYPE>& to, const void* base, int64_t at, int c) { to.template load_row<ROWS>(base, at, (c * LANES + lane) * 8, p.width); };
    const auto widen = [&](Raw8<TYPE>& raw, int c, float (&v)[8]) {
        raw.template align<ROWS>((c * LANES + lane) * 8, p.width);
        widen_8<TYPE>(raw.v, v);
    };
    const auto load_row = [&](int64_t row) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) load(x_raw[c], p.x, row * p.x_ld, c);
        if (p.residual)
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) load(r_raw[c], p.residual, row * p.residual_ld, c);
        if (gates)
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) load(g_raw[c], p.gate, row * p.gate_ld, c);
    };
    // gain_x times a gate of one row times the scale of what is kept; and gain
    constexpr int kKept = kKeep ? CHUNKS : 1;
    float front[kKept][8], gain[kKept][8];
    // 0 times that gate, NaN where it is not finite: what becomes of a dropped element.  (Eight registers; a branch for such gates took the scalar unit's:
    // 100 003 rows of 3 in single precision 22.7 us in place of 20.3.)
    float nothing[kKept][8];
    const bool one_gate = p.gate && !gates;
    // All three are on their way before the first is waited for: 20 000 rows of 1001 in half precision 43.4 us, 48.2 with each waited for in its turn.  (Not where no
    // register is left: 2048 rows of 8200 in single precision 423 us, 320 in turn.)
    Raw8<TYPE> gain_x_raw, gate_raw, gain_raw;
    const auto make_front = [&](int c, int kept) {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) front[kept][e] = p.drop.scale, nothing[kept][e] = 0;
        if (p.gain_x) {
            if (!kKeep) load(gain_x_raw, p.gain_x, 0, c);
            widen(gain_x_raw, c, f);
#pragma unroll
            for (int e = 0; e < 8; ++e) front[kept][e] *= f[e];
        }
        if (one_gate) {
            if (!kKeep) load(gate_raw, p.gate, 0, c);
            widen(gate_raw, c, f);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                front[kept][e] *= f[e];
                nothing[kept][e] = 0.0f * f[e];
            }
        }
    };
    const auto make_gain = [&](int c, float (&v)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 1;
        if (p.gain) {
            if (!kKeep) load(gain_raw, p.gain, 0, c);
            widen(gain_raw, c, v);
        }
        // (zeros behind the row, whatever was loaded there: they take part in the maximum of a row in 8 bits.  Short rows have them.)
        const bool in = ROWS == kShortRows || (c * LANES + lane) * 8 < p.width;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = in ? v[e] : 0.0f;
    };
    const int64_t last = count - 1;
    int64_t first = static_cast<int64_t>(blockIdx.x) * kRows;
    if (first < count) load_row(std::min(first + sub, last));
    if (kKeep)
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            if (p.gain_x) load(gain_x_raw, p.gain_x, 0, c);
            if (one_gate) load(gate_raw, p.gate, 0, c);
            if (p.gain) load(gain_raw, p.gain, 0, c);
            make_front(c, c % kKept), make_gain(c, gain[c % kKept]);
        }
    for (; first < count; first += stride) {
        const bool there = first + sub < count;
        const int64_t row = there ? first + sub : last;
        float t[CHUNKS][8], r[CHUNKS][8], g[CHUNKS][8];
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            widen(x_raw[c], c, t[c]);
            if (kKeep && p.residual) widen(r_raw[c], c, r[c]);
            if (kKeep && gates) widen(g_raw[c], c, g[c]);
        }
        if (kKeep && first + stride < count) load_row(std::min(first + stride + sub, last));
        float q = 1;
        if (p.norm_x) {
            float sum = 0;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                float part = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) part += t[c][e] * t[c][e];
                sum += (c * LANES + lane) * 8 < p.width ? part : 0.0f;
            }
            q = rsqrtf(whole_sum(sum) * per + p.eps);
            if (p.inv_rms_x && lane == 0 && there) p.inv_rms_x[row] = q;
        }
        float sum = 0;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int col = (c * LANES + lane) * 8;
            const Kept8 kept = kept_8(p.drop, seed, row, col);
            if (!kKeep) {
                make_front(c, 0);
                if (p.residual) widen(r_raw[c], c, r[c]);
                if (gates) widen(g_raw[c], c, g[c]);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float v = t[c][e] * q * front[c % kKept][e];
                v = kept.on[e] ? v : GATES ? 0.0f : nothing[c % kKept][e];          // (what is dropped becomes 0 whatever it was)
                if (gates) v *= g[c][e];
                if (p.residual) v += p.residual_scale * r[c][e];
                t[c][e] = col < p.width ? v : 0.0f;
            }
            if (p.total && there) store_row_8<TYPE, ROWS>(p.total, row * p.total_ld, col, p.width, t[c]);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += t[c][e] * t[c][e];
        }
        if (p.y) {
            q = rsqrtf(whole_sum(sum) * per + p.eps);
            if (p.inv_rms && lane == 0 && there) p.inv_rms[row] = q;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                if (!kKeep) make_gain(c, gain[0]);
#pragma unroll
                for (int e = 0; e < 8; ++e) t[c][e] *= q * gain[c % kKept][e];
            }
            if (p.y_scale) {
                if (there) finish_row<TYPE, LANES, CHUNKS>(t, p.width, lane, s, p.y, row * p.y_ld, p.y_scale + row);
            } else if (there) {
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) store_row_8<TYPE, ROWS>(p.y, row * p.y_ld, (c * LANES + lane) * 8, p.width, t[c]);
            }
        }
        if (!kKeep && first + stride < count) load_row(std::min(first + stride + sub, last));
    }
}

// The lanes and chunks for a row of `width` elements, as in the norm.
template <int TYPE, int ROWS, bool GATES, class RUN>
auto by_width(int32_t width, RUN run) {
    if (width <= 128) return run.template go<TYPE, 16, 1, ROWS, GATES>();
    if (width <= 512) return run.template go<TYPE, 64, 1, ROWS, GATES>();
    if (width <= 1024) return run.template go<TYPE, 128, 1, ROWS, GATES>();
    if (width <= 2048) return run.template go<TYPE, 256, 1, ROWS, GATES>();
    if (width <= 4096) return run.template go<TYPE, 512, 1, ROWS, GATES>();
    if (width <= 8192) return run.template go<TYPE, 1024, 1, ROWS, GATES>();
    return run.template go<TYPE, 1024, 4, ROWS, GATES>();
}
// Threads of a launch, about: rows in turn after that, so that a row is asked for while another is worked on, but not so many that the last ones
// keep few CUs busy.  100 003 x 1024 in half precision: 153 us for one million, 144 for two, 139 for four, 156 with a row each; 20 000 x 2000 in single precision
// 140, 140, 150, 162; 60 000 x 1000 in bfloat16 to 8 bits 91, 91, 97, 111.  Where four rows share a wave, for half a million, one and two: 100 003 x 100 in single
// precision 36.4, 35.0, 34.8, x 64 in bfloat16 16.0, 16.1, 17.4.
template <int LANES>
constexpr int kJoinThreads = LANES < kWave ? 256 * 4096 : 256 * 8192;
struct RunJoin {
    hipStream_t stream;
    JoinJob job;
    template <int TYPE, int LANES, int CHUNKS, int ROWS, bool GATES>
    hipError_t go() const {
        typedef JoinShape<LANES> Shape;
        const unsigned blocks = static_cast<unsigned>(std::min<int64_t>((job.rows.host + Shape::kRows - 1) / Shape::kRows, kJoinThreads<LANES> / Shape::kThreads));
        hipLaunchKernelGGL((join_kernel<TYPE, LANES, CHUNKS, ROWS, GATES>), dim3(blocks), dim3(Shape::kThreads), 0, stream, job);
        return hipGetLastError();
    }
};
template <int TYPE>
hipError_t run_join(const RunJoin& run) {
    const JoinJob& job = run.job;
    const int arrays = 1 + (job.residual != nullptr) + (job.gate_ld != 0) + (job.total != nullptr) + (job.y && !job.y_scale);
    const Rows rows = rows_of(job.width, job.rows.host * job.width * (arrays * type_bytes(TYPE) + (job.y_scale != nullptr)));
    if (rows == kShortRows) return run.go<TYPE, 16, 1, kShortRows, false>();
    if (rows == kRowsWithRest) return by_width<TYPE, kRowsWithRest, false>(job.width, run);
    if (rows == kStreamedRows) return job.gate_ld ? by_width<TYPE, kStreamedRows, true>(job.width, run) : by_width<TYPE, kStreamedRows, false>(job.width, run);
    return job.gate_ld ? by_width<TYPE, kWholeRows, true>(job.width, run) : by_width<TYPE, kWholeRows, false>(job.width, run);
}

template <int TYPE, int ROWS>
void run_dropout(hipStream_t stream, const DropoutJob& job) {
    const int64_t items = job.rows.host * ((job.width + 7) / 8);
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>((items + kBlock * kItems - 1) / (kBlock * kItems), kMostBlocks)));
    hipLaunchKernelGGL((dropout_kernel<TYPE, ROWS>), grid, dim3(kBlock), 0, stream, job);
}
template <int TYPE>
void run_dropout(hipStream_t stream, const DropoutJob& job) {
    const Rows rows = rows_of(job.width, job.rows.host * job.width * 2 * type_bytes(TYPE));
    if (rows == kWholeRows) run_dropout<TYPE, kWholeRows>(stream, job);
    else if (rows == kStreamedRows) run_dropout<TYPE, kStreamedRows>(stream, job);
    else if (rows == kRowsWithRest) run_dropout<TYPE, kRowsWithRest>(stream, job);
    else run_dropout<TYPE, kShortRows>(stream, job);
}

}  // namespace

hipError_t launch_dropout(hipStream_t stream, const DropoutJob& job) {
    if (job.rows.host < 1) return hipSuccess;
    if (job.type == kF32) run_dropout<kF32>(stream, job);
    else if (job.type == kF16) run_dropout<kF16>(stream, job);
    else run_dropout<kBF16>(stream, job);
    return hipGetLastError();
}

hipError_t launch_join(hipStream_t stream, const JoinJob& job) {
    if (job.rows.host < 1) return hipSuccess;
    const RunJoin run{stream, job};
    return job.x_type == kF32 ? run_join<kF32>(run) : job.x_type == kF16 ? run_join<kF16>(run) : run_join<kBF16>(run);
}

}  // namespace helios
