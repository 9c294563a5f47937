// Mean over the sampled neighbours of a block's rows, and its gradient.
//
//   mean[i] = 1/deg(i) sum over e of row i of x[col[e]]   (zeros where the row has no samples),   own[i] = x[row[i]]
//   dx[u] = sum over the entries of u, in the order of e, of dmean[r(e)] / deg(r(e)), then of down[i] where row[i] = u
//
// A group of lanes has one row (or one source) and eight neighbouring columns to a lane, so a source's row is read as
// one run; sums are held in 32 bits and added in the order of the list, so results do not depend on the launch.  The gradient
// needs the block by source: block_transpose sorts the entries by source with the stable radix sort of the hotness order.
// What bounds it is the latency of the chain entry -> row, hidden by several entries in flight per group, and then HBM/L2
// traffic of the rows.
#include "kernels.hpp"
#include "layer.hpp"
#include "layer_dev.hpp"

#include <algorithm>

namespace helios {

// hotness.hip
size_t hotness_order_scratch_bytes(int64_t n_nodes);
hipError_t launch_hotness_order(hipStream_t stream, const int32_t* counts, int64_t n_nodes, int32_t* order, void* scratch, int32_t* err);

namespace {

constexpr int kAhead = 4;                         // entries of a list whose rows are asked for together
constexpr int kLongList = 64;                     // entries from which a source is shared by a workgroup

template <int TYPE>
__device__ __forceinline__ void copy_8_of(const void* from, int64_t at, void* to, int64_t to_at, int valid) {
    constexpr int kBytes = type_bytes(TYPE);
    const char* p = static_cast<const char*>(from) + at * kBytes;
    char* q = static_cast<char*>(to) + to_at * kBytes;
    if (valid >= 8) {
        store_16(q, load_16(p));
        if (kBytes == 4) store_16(q + 16, load_16(p + 16));
        return;
    }
    for (int e = 0; e < valid; ++e) {
        if (kBytes == 4) reinterpret_cast<uint32_t*>(q)[e] = reinterpret_cast<const uint32_t*>(p)[e];
        else reinterpret_cast<uint16_t*>(q)[e] = reinterpret_cast<const uint16_t*>(p)[e];
    }
}

// Eight columns of a row that may be asked for in vain: zeros then.  (One branch, so that a group whose list is shorter than what is
// asked for together does not go through the elements one by one.)
template <int TYPE>
__device__ __forceinline__ void load_row_8(const void* base, int64_t at, bool wanted, int valid, float (&v)[8]) {
#pragma unroll
    for (int c = 0; c < 8; ++c) v[c] = 0;
    if (wanted) {
        if (valid >= 8) load_8<TYPE>(base, at, v);
        else load_8_of<TYPE>(base, at, valid, v);
    }
}

template <int TYPE, int LANES>
__global__ __launch_bounds__(kBlock) void block_mean_kernel(MeanJob p) {
    const int64_t count = p.rows.get();
    const int col = (blockIdx.y * LANES + threadIdx.x % LANES) * 8, valid = p.width - col;
    for (int64_t row = static_cast<int64_t>(blockIdx.x) * (kBlock / LANES) + threadIdx.x / LANES; row < count; row += static_cast<int64_t>(gridDim.x) * (kBlock / LANES)) {
        const RowBounds list = row_bounds(p.indptr, static_cast<uint32_t>(row));
        if (p.own) {
            const int64_t self = p.row ? p.row[row] : row;
            if (self >= 0 && self < p.n_src) copy_8_of<TYPE>(p.x, self * p.x_ld + col, p.own, row * p.own_ld + col, valid);
            else raise(p.err, kErrData);
        }
        const bool fits = list.lo >= 0 && list.lo <= list.hi && list.hi <= p.n_col;
        if (!fits) raise(p.err, kErrData);
        float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        const int64_t end = fits ? list.hi : list.lo;
        for (int64_t e = list.lo; e < end; e += kAhead) {
            int32_t src[kAhead];
            float v[kAhead][8];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) src[k] = p.col[e + k < end ? e + k : e];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const bool good = static_cast<uint32_t>(src[k]) < static_cast<uint64_t>(p.n_src);
                if (!good) raise(p.err, kErrData);
                load_row_8<TYPE>(p.x, static_cast<int64_t>(src[k]) * p.x_ld + col, e + k < end && good, valid, v[k]);
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
#pragma unroll
                for (int c = 0; c < 8; ++c) sum[c] += v[k][c];
        }
        const float n = end > list.lo ? static_cast<float>(end - list.lo) : 1.0f;
    #pragma unroll
        for (int c = 0; c < 8; ++c) sum[c] /= n;
        store_8_of<TYPE>(p.mean, row * p.mean_ld + col, valid, sum);
    }
}

// ---- the block by source

struct TransposeArgs {
    TransposeJob job;
    int64_t n;                                    // entries: n_col, and one for every row if there are own sources
    int32_t *keys, *entry, *order;                // scratch [n]
};

// Sort keys: n_src - source, so that the descending order of the sort is the ascending order of the sources, and 0, behind all of
// them, for places that hold no entry.
constexpr int kKeyLanes = 8;
__global__ __launch_bounds__(kBlock) void transpose_keys_kernel(TransposeArgs a) {
    const TransposeJob& p = a.job;
    const int64_t count = p.rows.get(), stride = static_cast<int64_t>(gridDim.x) * kBlock, t = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x;
    const auto put = [&](int64_t at, int32_t src, int32_t entry) {
        const bool good = src >= 0 && src < p.n_src;
        if (!good) raise(p.err, kErrData);
        a.keys[at] = good ? static_cast<int32_t>(p.n_src - src) : 0;
        a.entry[at] = entry;
    };
    for (int64_t k = t; k < count * kKeyLanes; k += stride) {
        const int64_t row = k / kKeyLanes;
        const RowBounds list = row_bounds(p.indptr, static_cast<uint32_t>(row));
        if (list.lo < 0 || list.lo > list.hi || list.hi > p.n_col) {
            raise(p.err, kErrData);
            continue;
        }
        for (int64_t e = list.lo + k % kKeyLanes; e < list.hi; e += kKeyLanes) put(e, p.col[e], static_cast<int32_t>(row));
    }
    const int64_t used = count > 0 ? p.indptr[count] : 0;
    for (int64_t e = (used < 0 ? 0 : used) + t; e < p.n_col; e += stride) a.keys[e] = 0;
    if (p.row)
        for (int64_t i = t; i < a.n - p.n_col; i += stride) {
            if (i < count) put(p.n_col + i, p.row[i], ~static_cast<int32_t>(i));
            else a.keys[p.n_col + i] = 0;
        }
}

// The sorted entries and where every source's begin.
__global__ __launch_bounds__(kBlock) void transpose_finish_kernel(TransposeArgs a) {
    const TransposeJob& p = a.job;
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kBlock;
    const auto source = [&](int64_t j) {
        const int32_t e = a.order[j];
        const int32_t key = e >= 0 && e < a.n ? a.keys[e] : 0;
        return key > 0 && key <= p.n_src ? p.n_src - key : p.n_src;
    };
    // (whole waves go round, so that a wave can fill its lanes' gaps together)
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x - lane_id(); base <= a.n; base += stride) {
        const int64_t j = base + lane_id();
        int64_t from = 0, to = 0;                 // sources whose entries begin at j: [from, to)
        if (j <= a.n) {
            from = j > 0 ? source(j - 1) + 1 : 0;
            const int64_t src = j < a.n ? source(j) : p.n_src;
            to = src + 1;
            if (j < a.n && src < p.n_src) p.src_entry[j] = a.entry[a.order[j]];
        }
        for (uint64_t look = __ballot(from < to); look != 0; look &= look - 1) {
            const int lane = __ffsll(static_cast<long long>(look)) - 1;
            const int64_t lo = __shfl(from, lane), hi = __shfl(to, lane);
            for (int64_t u = lo + lane_id(); u < hi; u += kWave) p.src_indptr[u] = static_cast<int32_t>(base + lane);
        }
    }
}

template <int TYPE, int LANES>
__global__ __launch_bounds__(kBlock) void block_mean_grad_kernel(MeanGradJob p) {
    constexpr int kGroups = kBlock / LANES, kCols = LANES * 8;
    __shared__ float s_part[kGroups][kCols];
    __shared__ int s_long[kGroups], s_n_long;
    const int group = threadIdx.x / LANES, lane = threadIdx.x % LANES, col = (blockIdx.y * LANES + lane) * 8, valid = p.width - col;
    const auto bounds = [&](int64_t src, int64_t* lo, int64_t* hi) {
        *lo = p.src_indptr[src];
        *hi = p.src_indptr[src + 1];
        if (*lo < 0 || *lo > *hi || *hi > p.n_entries) {
            raise(p.err, kErrData);
            *lo = *hi = 0;
        }
    };
    const auto add_up = [&](int64_t lo, int64_t hi, float (&sum)[8]) {
#pragma unroll
        for (int c = 0; c < 8; ++c) sum[c] = 0;
        for (int64_t k0 = lo; k0 < hi; k0 += kAhead) {
            int32_t entry[kAhead];
            float v[kAhead][8], weight[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) entry[k] = p.src_entry[k0 + k < hi ? k0 + k : k0];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const bool own = entry[k] < 0;
                const int64_t row = own ? ~entry[k] : entry[k];
                const bool good = row < p.n_rows && (!own || p.down), wanted = k0 + k < hi && good;
                if (!good) raise(p.err, kErrData);
                weight[k] = 1.0f;
                if (wanted && !own) {
                    const RowBounds list = row_bounds(p.indptr, static_cast<uint32_t>(row));
                    weight[k] = static_cast<float>(list.hi - list.lo);
                }
                load_row_8<TYPE>(own ? p.down : p.dmean, row * (own ? p.down_ld : p.dmean_ld) + col, wanted, valid, v[k]);
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
#pragma unroll
                for (int c = 0; c < 8; ++c) sum[c] += v[k][c] / weight[k];
        }
    };
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * kGroups; first < p.n_src; first += static_cast<int64_t>(gridDim.x) * kGroups) {
        if (threadIdx.x == 0) s_n_long = 0;
        __syncthreads();
        const int64_t src = first + group;
        if (src < p.n_src) {
            int64_t lo, hi;
            bounds(src, &lo, &hi);
            if (hi - lo <= kLongList) {
                float sum[8];
                add_up(lo, hi, sum);
                store_8_of<TYPE>(p.dx, src * p.dx_ld + col, valid, sum);
            } else if (lane == 0) s_long[atomicAdd(&s_n_long, 1)] = group;
        }
        __syncthreads();
        // Sources with long lists: every group takes a part of the list, and the parts are added in order.
        const int n_long = s_n_long;
        for (int k = 0; k < n_long; ++k) {
            const int64_t it = first + s_long[k];
            int64_t lo, hi;
            bounds(it, &lo, &hi);
            const int64_t per = (hi - lo + kGroups - 1) / kGroups, lo_mine = lo + group * per, hi_mine = lo_mine + per < hi ? lo_mine + per : hi;
            float sum[8];
            add_up(lo_mine, hi_mine, sum);
    #pragma unroll
            for (int c = 0; c < 8; ++c) s_part[group][lane * 8 + c] = sum[c];
            __syncthreads();
            if (group == 0) {
                for (int q = 1; q < kGroups; ++q)
    #pragma unroll
                    for (int c = 0; c < 8; ++c) sum[c] += s_part[q][lane * 8 + c];
                store_8_of<TYPE>(p.dx, it * p.dx_ld + col, valid, sum);
            }
            __syncthreads();
        }
        __syncthreads();
    }
}

// lanes for a row: eight columns to each, up to a wave; wider rows take several workgroups
template <int TYPE, class RUN>
hipError_t by_width(int32_t width, RUN run) {
    if (width <= 64) return run.template go<TYPE, 8>();
    if (width <= 128) return run.template go<TYPE, 16>();
    if (width <= 256) return run.template go<TYPE, 32>();
    return run.template go<TYPE, 64>();
}
template <class RUN>
hipError_t by_type(int type, int32_t width, RUN run) {
    if (type == kF32) return by_width<kF32>(width, run);
    if (type == kF16) return by_width<kF16>(width, run);
    return by_width<kBF16>(width, run);
}
dim3 grid_of(int64_t rows, int32_t width, int lanes) {
    const int per = kBlock / lanes, cols = lanes * 8;
    return dim3(static_cast<unsigned>(std::min<int64_t>((rows + per - 1) / per, 1 << 21)), static_cast<unsigned>((width + cols - 1) / cols));
}
struct RunMean {
    hipStream_t stream;
    MeanJob job;
    template <int TYPE, int LANES>
    hipError_t go() const {
        hipLaunchKernelGGL((block_mean_kernel<TYPE, LANES>), grid_of(job.rows.host, job.width, LANES), dim3(kBlock), 0, stream, job);
        return hipGetLastError();
    }
};
struct RunMeanGrad {
    hipStream_t stream;
    MeanGradJob job;
    template <int TYPE, int LANES>
    hipError_t go() const {
        hipLaunchKernelGGL((block_mean_grad_kernel<TYPE, LANES>), grid_of(job.n_src, job.width, LANES), dim3(kBlock), 0, stream, job);
        return hipGetLastError();
    }
};

struct TransposePlan {
    int64_t n;
    size_t keys, entry, order, sort, bytes;
    explicit TransposePlan(const TransposeJob& j) {
        const auto up = [](size_t b) { return (b + 255) / 256 * 256; };
        n = j.n_col + (j.row ? j.rows.host : 0);
        const size_t ints = up(sizeof(int32_t) * static_cast<size_t>(std::max<int64_t>(n, 1)));
        keys = 0;
        entry = ints;
        order = 2 * ints;
        sort = 3 * ints;
        bytes = sort + hotness_order_scratch_bytes(std::max<int64_t>(n, 1));
    }
};

}  // namespace

hipError_t launch_block_mean(hipStream_t stream, const MeanJob& job) {
    if (job.rows.host < 1) return hipSuccess;
    return by_type(job.type, job.width, RunMean{stream, job});
}

size_t block_transpose_scratch_bytes(const TransposeJob& job) { return TransposePlan(job).bytes; }

hipError_t launch_block_transpose(hipStream_t stream, const TransposeJob& job, void* scratch) {
    const TransposePlan plan(job);
    char* at = static_cast<char*>(scratch);
    TransposeArgs a{job, plan.n, reinterpret_cast<int32_t*>(at + plan.keys), reinterpret_cast<int32_t*>(at + plan.entry), reinterpret_cast<int32_t*>(at + plan.order)};
    hipError_t e = hipSuccess;
    const auto blocks = [](int64_t n) { return dim3(static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>((n + kBlock - 1) / kBlock, 4096)))); };
    if (a.n > 0) {
        hipLaunchKernelGGL(transpose_keys_kernel, blocks(std::max(a.n, job.rows.host * kKeyLanes)), dim3(kBlock), 0, stream, a);
        e = hipGetLastError();
        if (e == hipSuccess) e = launch_hotness_order(stream, a.keys, a.n, a.order, at + plan.sort, job.err);
    }
    if (e == hipSuccess) {
        hipLaunchKernelGGL(transpose_finish_kernel, blocks(a.n + 1), dim3(kBlock), 0, stream, a);
        e = hipGetLastError();
    }
    return e;
}

hipError_t launch_block_mean_grad(hipStream_t stream, const MeanGradJob& job) {
    if (job.n_src < 1) return hipSuccess;
    return by_type(job.type, job.width, RunMeanGrad{stream, job});
}

}  // namespace helios
