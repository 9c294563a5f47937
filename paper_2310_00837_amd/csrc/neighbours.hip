// Mean over the sampled neighbours of a block's rows, and its gradient.
//
//   mean[i] = 1/deg(i) sum over e of row i of x[col[e]]   (zeros where the row has no samples),   own[i] = x[row[i]]
//   dx[u] = sum over the entries of u, in the order of e, of dmean[r(e)] / deg(r(e)), then of down[i] where row[i] = u
//
// A group of lanes has one row (or one source) and eight neighbouring columns to a lane, so a source's row is read as
// one run; sums are held in 32 bits and added in the order of the list, so results do not depend on the launch.  The gradient
// needs the block by source, entries in their order: block_transpose finds it in one launch up to 131 072 places, and beyond them with
// the stable radix sort of the hotness order.
// What bounds it is the latency of the chain list -> entry -> row, hidden by several entries in flight per group, and then HBM/L2
// traffic of the rows: means of 25 600 rows of ten, 128 columns in single precision, 26 us, of 640 rows of five, 64 columns, 4.4 us of
// kernel; the gradient of 24 000 sources of 26 600 entries, 256 columns in bfloat16, 30 us: 11 by source, 15 of sums, 4 for
// a launch that finds no long list.
#include "kernels.hpp"
#include "layer.hpp"
#include "layer_dev.hpp"

#include <algorithm>

namespace helios {

// hotness.hip
size_t hotness_order_scratch_bytes(int64_t n_nodes);
hipError_t launch_hotness_order(hipStream_t stream, const int32_t* counts, int64_t n_nodes, int32_t* order, void* scratch, int32_t* err);

namespace {

constexpr int kMeanAhead = 8;                     // entries of a list whose rows are asked for together (lists are 5 to 25 long)
constexpr int kAhead = 4;                         // ... in the gradient, where a list begins (most have one or two)
constexpr int kPiece = 256;                       // entries of a long list that a workgroup adds up
constexpr int kLongBlock = 256;                   // ... and its threads
constexpr uint32_t kLines = 8, kLineWords = 32;   // of the counters
static_assert((1 + kLines) * kLineWords <= kLayerCounters, "a context has room for as many counters");
constexpr int kLongList = 32;                     // entries of a source that a group adds up by itself; longer ones would hold up their wave

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

// sum += eight columns of a row, times weight
template <int TYPE>
__device__ __forceinline__ void add_8(const Raw8<TYPE>& row, float weight, float (&sum)[8]) {
    float v[8];
    widen_8<TYPE>(row.v, v);
#pragma unroll
    for (int c = 0; c < 8; ++c) sum[c] += v[c] * weight;
}

// Whether a row's list lies in col.
__device__ __forceinline__ bool good_list(const RowBounds& list, int64_t n_col) { return list.lo >= 0 && list.lo <= list.hi && list.hi <= n_col; }

template <int TYPE, int LANES>
__global__ __launch_bounds__(kBlock) void block_mean_kernel(MeanJob p) {
    const int64_t count = p.rows.get();
    const int col = (blockIdx.y * LANES + threadIdx.x % LANES) * 8, valid = p.width - col;
    for (int64_t row = static_cast<int64_t>(blockIdx.x) * (kBlock / LANES) + threadIdx.x / LANES; row < count; row += static_cast<int64_t>(gridDim.x) * (kBlock / LANES)) {
        const RowBounds list = row_bounds(p.indptr, static_cast<uint32_t>(row));
        if (p.own) {
            const int64_t self = p.row ? p.row[row] : row;
            if (self >= 0 && self < p.n_src) copy_8_of<TYPE>(p.x, self * p.x_ld + col, p.own, row * p.own_ld + col, valid);
            else {
                const float none[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                store_8_of<TYPE>(p.own, row * p.own_ld + col, valid, none);
                raise(p.err, kErrData);
            }
        }
        const bool fits = good_list(list, p.n_col);
        if (!fits) raise(p.err, kErrData);
        float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        const int64_t end = fits ? list.hi : list.lo;
        for (int64_t e = list.lo; e < end; e += kMeanAhead) {
            int32_t src[kMeanAhead];
            Raw8<TYPE> v[kMeanAhead];
#pragma unroll
            for (int k = 0; k < kMeanAhead; ++k) src[k] = p.col[e + k < end ? e + k : e];
#pragma unroll
            for (int k = 0; k < kMeanAhead; ++k) {
                const bool good = static_cast<uint32_t>(src[k]) < static_cast<uint64_t>(p.n_src);
                if (!good) raise(p.err, kErrData);
                v[k].clear();                     // (rows asked for in vain: zeros)
                if (e + k < end && good) v[k].load(p.x, static_cast<int64_t>(src[k]) * p.x_ld + col, valid);
            }
#pragma unroll
            for (int k = 0; k < kMeanAhead; ++k) add_8<TYPE>(v[k], 1.0f, sum);
        }
        const float weight = 1.0f / (end > list.lo ? static_cast<float>(end - list.lo) : 1.0f);
#pragma unroll
        for (int c = 0; c < 8; ++c) sum[c] *= weight;
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
// them, for places that hold no entry: those in front of the first list and behind the last, and those of lists that are not good.  All
// keys are 0 before the lists' own are written.
constexpr int kKeyLanes = 8;
__global__ __launch_bounds__(kBlock) void transpose_clear_kernel(TransposeArgs a) {
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kBlock;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x; i < a.n; i += stride) a.keys[i] = 0;
}
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
        if (!good_list(list, p.n_col)) {
            raise(p.err, kErrData);
            continue;
        }
        for (int64_t e = list.lo + k % kKeyLanes; e < list.hi; e += kKeyLanes) put(e, p.col[e], static_cast<int32_t>(row));
    }
    if (p.row)
        for (int64_t i = t; i < count; i += stride) put(p.n_col + i, p.row[i], ~static_cast<int32_t>(i));
}

// The sorted entries and where every source's begin.
__global__ __launch_bounds__(kBlock) void transpose_finish_kernel(TransposeArgs a) {
    const TransposeJob& p = a.job;
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kBlock;
    const auto source = [&](int64_t j, int32_t* place) {
        const int32_t e = a.order[j];
        const int32_t key = e >= 0 && e < a.n ? a.keys[e] : 0;
        if (place) *place = e;
        return key > 0 && key <= p.n_src ? p.n_src - key : p.n_src;
    };
    // (whole waves go round, so that a wave can fill its lanes' gaps together)
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x - lane_id(); base <= a.n; base += stride) {
        const int64_t j = base + lane_id();
        int64_t from = 0, to = 0;                 // sources whose entries begin at j: [from, to)
        int32_t e = -1;
        const int64_t src = j < a.n ? source(j, &e) : p.n_src;
        int64_t before = __shfl_up(src, 1);
        if (lane_id() == 0) before = j > 0 ? source(j - 1, nullptr) : -1;
        if (j <= a.n) {
            from = before + 1;
            to = src + 1;
            if (src < p.n_src) p.src_entry[j] = a.entry[e];
        }
        for (uint64_t look = __ballot(from < to); look != 0; look &= look - 1) {
            const int lane = __ffsll(static_cast<long long>(look)) - 1;
            const int64_t lo = __shfl(from, lane), hi = __shfl(to, lane);
            for (int64_t u = lo + lane_id(); u < hi; u += kWave) p.src_indptr[u] = static_cast<int32_t>(base + lane);
        }
    }
}

// The same in one launch, for lists that are short enough for every workgroup to look through all of them: a workgroup has a range of
// sources, counts what belongs to sources before it, and gathers what belongs to its own in LDS, where it is sorted by source
// and place.  Lists that hold more for a range than LDS does are gone through again, in windows of as many places.
constexpr int kRangeBlock = 1024, kRangeMost = 1024, kRangeHeld = 8192, kRangeSteps = 1024;
struct RangeLds {
    unsigned long long held[kRangeHeld];          // (source in the range, place)
    uint32_t count[kRangeMost];                   // of a source; then where its next entry goes
    uint32_t taken[kRangeMost];
    int32_t step[kRangeSteps + 1];                // indptr at every stride-th row
    uint32_t wave[kRangeBlock / kWave];
    uint32_t n_held, below, longest;
};

// held[0, n) in ascending order, n <= 2^bits; the words from n on are the largest there is.
__device__ void sort_held(unsigned long long* held, uint32_t size) {
    for (uint32_t k = 2; k <= size; k <<= 1)
        for (uint32_t j = k >> 1; j > 0; j >>= 1) {
            __syncthreads();
            for (uint32_t i = threadIdx.x; i < size / 2; i += kRangeBlock) {
                const uint32_t lo = 2 * i - (i & (j - 1)), hi = lo + j;
                const unsigned long long a = held[lo], b = held[hi];
                if ((a > b) == ((lo & k) == 0)) held[lo] = b, held[hi] = a;
            }
        }
    __syncthreads();
}

__global__ __launch_bounds__(kRangeBlock) void transpose_range_kernel(TransposeArgs a, uint32_t range) {
    __shared__ RangeLds s;
    const TransposeJob& p = a.job;
    const int64_t count = p.rows.get();
    const uint32_t first = blockIdx.x * range, t = threadIdx.x;
    const uint32_t sources = first >= p.n_src ? 0u : static_cast<uint32_t>(p.n_src - first < range ? p.n_src - first : range);
    // (the lists are looked at by all workgroups together)
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kRangeBlock + t; i < count; i += static_cast<int64_t>(gridDim.x) * kRangeBlock)
        if (!good_list(row_bounds(p.indptr, static_cast<uint32_t>(i)), p.n_col)) raise(p.err, kErrData);
    if (sources == 0) return;
    // The lists are neighbours, so they take the places [n_first, n_col), and the rows' own sources those from there to n.
    RowBounds all{0, 0};
    if (count > 0) all = RowBounds{p.indptr[0], p.indptr[count]};
    if (!good_list(all, p.n_col)) {
        raise(p.err, kErrData);
        all = RowBounds{0, 0};
    }
    const uint32_t n_first = static_cast<uint32_t>(all.lo), n_col = static_cast<uint32_t>(all.hi), n = n_col + (p.row ? static_cast<uint32_t>(count) : 0u);
    // where rows begin, roughly: the row of a place is looked up there first
    const uint32_t stride = static_cast<uint32_t>((count + kRangeSteps - 1) / kRangeSteps) > 0 ? static_cast<uint32_t>((count + kRangeSteps - 1) / kRangeSteps) : 1u;
    const uint32_t steps = static_cast<uint32_t>((count + stride - 1) / stride);
    for (uint32_t i = t; i < steps; i += kRangeBlock) s.step[i] = static_cast<int32_t>(p.indptr[static_cast<int64_t>(i) * stride]);
    for (uint32_t i = t; i < sources; i += kRangeBlock) s.count[i] = s.taken[i] = 0;
    if (t == 0) s.n_held = s.below = s.longest = 0;
    __syncthreads();

    const auto source = [&](uint32_t place) { return place < n_col ? p.col[place] : p.row[place - n_col]; };
    const auto hold = [&](uint32_t local, uint32_t place) {
        const uint32_t at = atomicAdd(&s.n_held, 1u);
        if (at < kRangeHeld) s.held[at] = static_cast<unsigned long long>(local) << 32 | place;
    };
    uint32_t below = 0;
    const auto look = [&](int32_t src, uint32_t place) {
        const uint32_t u = static_cast<uint32_t>(src);
        if (u >= p.n_src) raise(p.err, kErrData);
        else if (u < first) ++below;
        else if (u - first < sources) {
            atomicAdd(&s.count[u - first], 1u);
            hold(u - first, place);
        }
    };
    // (sixteen places to a thread are asked for together: a round is a trip to memory)
    const auto look_through = [&](const int32_t* list, uint32_t len, uint32_t base_place) {
        constexpr uint32_t kWords = 4, kRound = kRangeBlock * 4 * kWords;
        for (uint32_t base = 0; base < len; base += kRound) {
            i32x4 v[kWords];
#pragma unroll
            for (uint32_t k = 0; k < kWords; ++k) {
                const uint32_t at = base + (k * kRangeBlock + t) * 4;
                v[k] = at < len ? load_16_of<4>(list + at, len - at) : i32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (uint32_t k = 0; k < kWords; ++k) {
                const uint32_t at = base + (k * kRangeBlock + t) * 4;
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e)
                    if (at + e < len) look(v[k][e], base_place + at + e);
            }
        }
    };
    look_through(p.col + n_first, n_col - n_first, n_first);
    if (p.row) look_through(p.row, n - n_col, n_col);
    below = dpp_sum(below);
    if (lane_id() == 0) atomicAdd(&s.below, below);
    __syncthreads();
    // counts -> where a source's entries begin (a thread to a source)
    const uint32_t mine = t < sources ? s.count[t] : 0, upto = dpp_inclusive_scan(mine);
    if (mine > kRangeBlock) atomicMax(&s.longest, mine);
    if (lane_id() == kWave - 1) s.wave[wave_id()] = upto;
    __syncthreads();
    uint32_t begin = s.below + upto - mine;
    for (int w = 0; w < wave_id(); ++w) begin += s.wave[w];
    if (t < sources) {
        s.count[t] = begin;
        p.src_indptr[first + t] = static_cast<int32_t>(begin);
        if (first + t + 1 == p.n_src) p.src_indptr[p.n_src] = static_cast<int32_t>(begin + mine);
    }
    const uint32_t found = s.n_held;
    __syncthreads();

    const auto row_of = [&](uint32_t place) {                // the last row that begins at or before the place
        uint32_t lo = 0, hi = steps;
        while (hi - lo > 1) {
            const uint32_t mid = (lo + hi) / 2;
            if (s.step[mid] <= static_cast<int32_t>(place)) lo = mid;
            else hi = mid;
        }
        int64_t r0 = static_cast<int64_t>(lo) * stride, r1 = r0 + stride < count ? r0 + stride : count;
        while (r1 - r0 > 1) {
            const int64_t mid = (r0 + r1) / 2;
            if (p.indptr[mid] <= place) r0 = mid;
            else r1 = mid;
        }
        return static_cast<int32_t>(r0);
    };
    // sorts what is held and writes it behind what its sources have got so far
    const auto place_held = [&](uint32_t held) {
        uint32_t size = 2;
        while (size < held) size <<= 1;
        for (uint32_t i = held + t; i < size; i += kRangeBlock) s.held[i] = ~0ull;
        sort_held(s.held, size);
        for (uint32_t i = t; i < held; i += kRangeBlock) {
            const uint32_t local = static_cast<uint32_t>(s.held[i] >> 32), place = static_cast<uint32_t>(s.held[i]);
            uint32_t lo = 0, hi = i;                         // the source's first entry among those held
            while (lo < hi) {
                const uint32_t mid = (lo + hi) / 2;
                if (s.held[mid] >> 32 < local) lo = mid + 1;
                else hi = mid;
            }
            const uint32_t to = s.count[local] + (i - lo);
            if (to < a.n) p.src_entry[to] = place < n_col ? row_of(place) : ~static_cast<int32_t>(place - n_col);
        }
        __syncthreads();
    };
    if (found <= kRangeHeld && s.longest <= kRangeBlock) {
        // They are put together by source (in the memory that held them), and an entry counts those of its source that come before it.
        constexpr int kEach = kRangeHeld / kRangeBlock;
        unsigned long long mine[kEach];
#pragma unroll
        for (int q = 0; q < kEach; ++q) mine[q] = t + q * kRangeBlock < found ? s.held[t + q * kRangeBlock] : 0;
        __syncthreads();
        uint32_t* placed = reinterpret_cast<uint32_t*>(s.held);
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            if (t + q * kRangeBlock >= found) continue;
            const uint32_t local = static_cast<uint32_t>(mine[q] >> 32);
            placed[s.count[local] - s.below + atomicAdd(&s.taken[local], 1u)] = static_cast<uint32_t>(mine[q]);
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            if (t + q * kRangeBlock >= found) continue;
            const uint32_t local = static_cast<uint32_t>(mine[q] >> 32), place = static_cast<uint32_t>(mine[q]);
            const uint32_t begin = s.count[local] - s.below, end = begin + s.taken[local];
            uint32_t before = 0;
#pragma unroll 4
            for (uint32_t i = begin; i < end; ++i) before += placed[i] < place;
            const uint32_t to = s.count[local] + before;
            if (to < a.n) p.src_entry[to] = place < n_col ? row_of(place) : ~static_cast<int32_t>(place - n_col);
        }
        return;
    }
    if (found <= kRangeHeld) {
        place_held(found);
        return;
    }
    for (uint32_t base = n_first; base < n; base += kRangeHeld) {
        if (t == 0) s.n_held = 0;
        __syncthreads();
        for (uint32_t k = t; k < kRangeHeld; k += kRangeBlock)
            if (base + k < n && static_cast<uint32_t>(source(base + k)) - first < sources) hold(static_cast<uint32_t>(source(base + k)) - first, base + k);
        __syncthreads();
        const uint32_t held = s.n_held;
        place_held(held);
        for (uint32_t i = t; i < held; i += kRangeBlock) {   // (the last of a source among those held moves it on)
            const uint32_t local = static_cast<uint32_t>(s.held[i] >> 32);
            if (i + 1 < held && s.held[i + 1] >> 32 == local) continue;
            uint32_t lo = 0, hi = i;
            while (lo < hi) {
                const uint32_t mid = (lo + hi) / 2;
                if (s.held[mid] >> 32 < local) lo = mid + 1;
                else hi = mid;
            }
            s.count[local] += i - lo + 1;
        }
        __syncthreads();
    }
}

// Sources with long lists wait for the second kernel, cut into pieces; the pieces of one source are neighbours.
struct LongPiece {
    int32_t src, piece, pieces;
    int32_t left;                                 // (of the first piece) workgroups that have not added up theirs
    uint32_t slot;                                // where the piece's sums go, if there are several
};
struct GradScratch {
    uint32_t* counters;                           // pieces waiting, slots taken, eighths that are done; from kLineWords on the eighths' counts.  Zero between calls
    LongPiece* piece;                             // [most]
    float* part;                                  // [slots][width]: sums of pieces
    uint32_t most, slots;
};

// An entry's share of the gradient: a row of dmean and 1 / its samples, or of down and 1; nothing and an error if there is no such row.
template <int TYPE>
__device__ __forceinline__ void share_of(const MeanGradJob& p, int32_t entry, bool wanted, int col, int valid, Raw8<TYPE>& v, float* weight) {
    const bool own = entry < 0;
    const int64_t row = own ? ~entry : entry;
    bool good = row < p.n_rows && (!own || p.down);
    *weight = 1.0f;
    if (wanted && good && !own) {
        const RowBounds list = row_bounds(p.indptr, static_cast<uint32_t>(row));
        good = list.lo < list.hi;                 // (a row without samples has no share)
        *weight = good ? 1.0f / static_cast<float>(list.hi - list.lo) : 0.0f;
    }
    if (wanted && !good) raise(p.err, kErrData);
    v.clear();
    if (wanted && good) v.load(own ? p.down : p.dmean, row * (own ? p.down_ld : p.dmean_ld) + col, valid);
}
// sum += the shares of the entries [lo, hi), AHEAD at a time, in order
template <int TYPE, int AHEAD>
__device__ __forceinline__ void add_shares(const MeanGradJob& p, int32_t lo, int32_t hi, int col, int valid, float (&sum)[8]) {
    for (int32_t k0 = lo; k0 < hi; k0 += AHEAD) {
        int32_t entry[AHEAD];
        Raw8<TYPE> v[AHEAD];
        float weight[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) entry[k] = p.src_entry[k0 + k < hi ? k0 + k : k0];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) share_of<TYPE>(p, entry[k], k0 + k < hi, col, valid, v[k], &weight[k]);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) add_8<TYPE>(v[k], weight[k], sum);
    }
}

// A group of lanes has a source.  (Two to a group, with the loads of both together, took half as long again: 20.6 and 12.0 us for
// 24 000 sources of 26 600 entries and 256 columns in bfloat16, as fewer waves fit.)
template <int TYPE, int LANES>
__global__ __launch_bounds__(kBlock) void block_mean_grad_kernel(MeanGradJob p, GradScratch s) {
    constexpr int kGroups = kBlock / LANES;
    const int lane = threadIdx.x % LANES, col = (blockIdx.y * LANES + lane) * 8, valid = p.width - col;
    for (int64_t src = static_cast<int64_t>(blockIdx.x) * kGroups + threadIdx.x / LANES; src < p.n_src; src += static_cast<int64_t>(gridDim.x) * kGroups) {
        int32_t lo = p.src_indptr[src], hi = p.src_indptr[src + 1];
        if (lo < 0 || lo > hi || hi > p.n_entries) {
            raise(p.err, kErrData);
            lo = hi = 0;
        }
        if (hi - lo > kLongList) {
            if (lane == 0 && blockIdx.y == 0) {
                const uint32_t pieces = (hi - lo + kPiece - 1) / kPiece, at = atomicAdd(s.counters, pieces);
                const uint32_t slot = pieces > 1 ? atomicAdd(s.counters + 1, pieces) : 0u;
                const bool room = at + pieces <= s.most && (pieces == 1 || slot + pieces <= s.slots);
                if (!room) raise(p.err, kErrData);          // (only if lists overlap)
                for (uint32_t k = 0; k < pieces && at + k < s.most; ++k)
                    s.piece[at + k] = LongPiece{static_cast<int32_t>(src), static_cast<int32_t>(k), room ? static_cast<int32_t>(pieces) : 0,
                                                static_cast<int32_t>(pieces * gridDim.y), slot + k};
            }
            continue;
        }
        float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        add_shares<TYPE, kAhead>(p, lo, hi < lo + kAhead ? hi : lo + kAhead, col, valid, sum);
        add_shares<TYPE, 8>(p, lo + kAhead, hi, col, valid, sum);
        store_8_of<TYPE>(p.dx, src * p.dx_ld + col, valid, sum);
    }
}

// The pieces of long lists, a workgroup to each at a time: its groups share the entries, and their sums are added in order.  Who
// finishes the last piece of a source adds the pieces up, in order.
template <int TYPE, int LANES>
__global__ __launch_bounds__(kLongBlock) void block_mean_grad_long_kernel(MeanGradJob p, GradScratch s) {
    constexpr int kGroups = kLongBlock / LANES, kCols = LANES * 8;
    __shared__ float s_part[kGroups][kCols];
    __shared__ int s_last;
    const int group = threadIdx.x / LANES, lane = threadIdx.x % LANES, col = (blockIdx.y * LANES + lane) * 8, valid = p.width - col;
    const uint32_t waiting = s.counters[0], n = waiting < s.most ? waiting : s.most;
    for (uint32_t at = blockIdx.x; at < n; at += gridDim.x) {
        const LongPiece it = s.piece[at];
        if (it.pieces == 0) continue;
        const int32_t lo = p.src_indptr[it.src] + it.piece * kPiece, end = p.src_indptr[it.src + 1], hi = lo + kPiece < end ? lo + kPiece : end;
        const int32_t per = (hi - lo + kGroups - 1) / kGroups, lo_mine = lo + group * per, hi_mine = lo_mine + per < hi ? lo_mine + per : hi;
        float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        add_shares<TYPE, 8>(p, lo_mine, hi_mine, col, valid, sum);
#pragma unroll
        for (int c = 0; c < 8; ++c) s_part[group][lane * 8 + c] = sum[c];
        __syncthreads();
        if (group == 0) {
            for (int q = 1; q < kGroups; ++q)
#pragma unroll
                for (int c = 0; c < 8; ++c) sum[c] += s_part[q][lane * 8 + c];
            if (it.pieces == 1) store_8_of<TYPE>(p.dx, it.src * p.dx_ld + col, valid, sum);
            else store_8_of<kF32>(s.part, static_cast<int64_t>(it.slot) * p.width + col, valid, sum);
        }
        if (it.pieces > 1) {
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0) s_last = atomicSub(&s.piece[at - it.piece].left, 1) == 1;
            __syncthreads();
            if (s_last) {                          // (of all columns: the workgroups of the other columns have left their sums, too)
                __threadfence();
                for (int c0 = threadIdx.x * 8; c0 < p.width; c0 += kLongBlock * 8) {
                    float total[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll 8
                    for (int k = 0; k < it.pieces; ++k) {
                        float v[8];
                        load_8_of<kF32>(s.part, static_cast<int64_t>(it.slot - it.piece + k) * p.width + c0, p.width - c0, v);
#pragma unroll
                        for (int c = 0; c < 8; ++c) total[c] += v[c];
                    }
                    store_8_of<TYPE>(p.dx, it.src * p.dx_ld + c0, p.width - c0, total);
                }
            }
        }
        __syncthreads();
    }
    // The last workgroup leaves the counters as it found them.  (A word that hundreds add to costs 60 ns for each of them, so they
    // count by eighths first.)
    if (threadIdx.x == 0) {
        const uint32_t all = gridDim.x * gridDim.y, me = blockIdx.y * gridDim.x + blockIdx.x, line = me % kLines, lines = all < kLines ? all : kLines;
        uint32_t* count = s.counters + (1 + line) * kLineWords;
        if (atomicAdd(count, 1u) + 1 == (all - line + kLines - 1) / kLines) {
            *count = 0;
            if (atomicAdd(s.counters + 2, 1u) + 1 == lines) s.counters[0] = s.counters[1] = s.counters[2] = 0;
        }
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
// Most pieces that lists of n entries in all can be cut into (one of kLongList + 1 entries is one piece), and most of them that belong to
// lists of several (kPiece + 1 entries are two).
int64_t most_pieces(int64_t n) { return n / kLongList + 1; }
int64_t most_slots(int64_t n) { return 2 * n / kPiece + 2; }
struct RunMeanGrad {
    hipStream_t stream;
    MeanGradJob job;
    GradScratch s;
    template <int TYPE, int LANES>
    hipError_t go() const {
        const dim3 grid = grid_of(job.n_src, job.width, LANES);
        hipLaunchKernelGGL((block_mean_grad_kernel<TYPE, LANES>), grid, dim3(kBlock), 0, stream, job, s);
        hipError_t e = hipGetLastError();
        if (e == hipSuccess && job.n_entries > kLongList) {
            const unsigned most = static_cast<unsigned>(std::min<int64_t>(most_pieces(job.n_entries), 256));
            hipLaunchKernelGGL((block_mean_grad_long_kernel<TYPE, LANES>), dim3(most, grid.y), dim3(kLongBlock), 0, stream, job, s);
            e = hipGetLastError();
        }
        return e;
    }
};

// By ranges where looking through all places takes less than the sort's eight launches.  us by sort / by ranges: 27 000 places
// 59 / 11, 65 000 59 / 18, 105 000 60 / 26 (of 4000 sources 57 / 29), 131 000 64 / 31 (of 2000 sources, where a range holds more than its
// LDS, 36 / 46); every workgroup reads every place, so the time grows with them (282 000 72 / 62).
constexpr int64_t kRangePlaces = 1 << 17;
struct TransposePlan {
    int64_t n, ranges;                            // (ranges: 0 by a sort)
    size_t keys, entry, order, sort, bytes;
    explicit TransposePlan(const TransposeJob& j) {
        const auto up = [](size_t b) { return (b + 255) / 256 * 256; };
        n = j.n_col + (j.row ? j.rows.host : 0);
        ranges = n > kRangePlaces || j.n_src < 1 ? 0 : std::max<int64_t>(std::min<int64_t>(256, (j.n_src + 31) / 32), (j.n_src + kRangeMost - 1) / kRangeMost);
        if (ranges > 4096) ranges = 0;
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
    if (plan.ranges > 0) {
        const uint32_t range = static_cast<uint32_t>((std::max<int64_t>(job.n_src, 1) + plan.ranges - 1) / plan.ranges);
        hipLaunchKernelGGL(transpose_range_kernel, dim3(static_cast<unsigned>(plan.ranges)), dim3(kRangeBlock), 0, stream, a, range);
        return hipGetLastError();
    }
    hipError_t e = hipSuccess;
    const auto blocks = [](int64_t n) { return dim3(static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>((n + kBlock - 1) / kBlock, 4096)))); };
    if (a.n > 0) {
        hipLaunchKernelGGL(transpose_clear_kernel, blocks(a.n), dim3(kBlock), 0, stream, a);
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

namespace {
struct GradPlan {
    size_t part, bytes;
    explicit GradPlan(const MeanGradJob& j) {
        part = (sizeof(LongPiece) * static_cast<size_t>(most_pieces(j.n_entries)) + 255) / 256 * 256;
        bytes = part + sizeof(float) * static_cast<size_t>(most_slots(j.n_entries)) * static_cast<size_t>(j.width);
    }
};
}  // namespace

size_t block_mean_grad_scratch_bytes(const MeanGradJob& job) { return GradPlan(job).bytes; }

hipError_t launch_block_mean_grad(hipStream_t stream, const MeanGradJob& job, uint32_t* counters, void* scratch) {
    if (job.n_src < 1) return hipSuccess;
    char* at = static_cast<char*>(scratch);
    const GradScratch s{counters, reinterpret_cast<LongPiece*>(at), reinterpret_cast<float*>(at + GradPlan(job).part),
                        static_cast<uint32_t>(most_pieces(job.n_entries)), static_cast<uint32_t>(most_slots(job.n_entries))};
    return by_type(job.type, job.width, RunMeanGrad{stream, job, s});
}

}  // namespace helios
