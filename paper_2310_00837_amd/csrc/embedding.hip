// Learnt rows by ID, and the gradient of their table by the sorted list of IDs.
//
//   y[i] = add[i] + scale * table[id_i];   dtable[k] = scale * sum of dy[i] over the positions i with id_i = k
//
// The lookup is bound by memory: every row that is met once, add and y.  The gradient sorts {ID, position} (stable, so that an ID's positions
// keep their order), cuts the sorted list into chunks of equal length whatever the IDs, and lets a group of lanes sum a chunk, run of
// equal IDs by run: a run that lies in one chunk is finished there, one that goes on leaves a part for every chunk it meets, and a last
// kernel adds these.  So a list of one ID costs what a list of distinct ones does, no sum is made by atomics, and the same list gives the
// same bits.  What bounds it is the rows of dy, read once, and in front of that the chain of short launches that sorts the list:
// lists of up to 2048 are ranked by comparing all with all, longer ones go through a radix sort of two launches for every digit.
#include "layer.hpp"
#include "layer_dev.hpp"

#include <algorithm>

namespace helios {

namespace {

constexpr int64_t kMostBlocks = 1 << 21;            // of a launch

// ---- lookup

constexpr int kItems = 2;                           // of a thread, in flight together
template <int TABLE, int Y>
__global__ __launch_bounds__(kBlock) void embedding_kernel(EmbeddingJob p) {
    const uint32_t blocks = static_cast<uint32_t>(p.width + 7) / 8;
    const int64_t items = p.rows.get() * blocks, step = static_cast<int64_t>(gridDim.x) * kBlock * kItems;
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * kBlock * kItems; base < items; base += step) {
        const ItemPlaces places(base, blocks);
        Raw8<TABLE> row_raw[kItems];
        Raw8<Y> add_raw[kItems];
        int64_t row[kItems];
        int32_t col[kItems], valid[kItems], id[kItems];
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            const uint32_t i = k * kBlock + threadIdx.x;
            places.get(i, &row[k], &col[k]);
            valid[k] = base + i < items ? p.width - col[k] : 0;
            id[k] = valid[k] > 0 ? p.ids[row[k]] : -1;
        }
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            const bool there = id[k] >= 0 && id[k] < p.n_table;
            if (!there && id[k] != -1) raise(p.err, kErrData);
            row_raw[k].load(p.table, there ? id[k] * p.table_ld + col[k] : 0, there ? valid[k] : 0);
            if (p.add) add_raw[k].load(p.add, row[k] * p.add_ld + col[k], valid[k]);
        }
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            const bool there = id[k] >= 0 && id[k] < p.n_table;
            float v[8], a[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            widen_8<TABLE>(row_raw[k].v, v);
            if (p.add) widen_8<Y>(add_raw[k].v, a);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = there ? __builtin_fmaf(v[e], p.scale, a[e]) : a[e];
            store_8_of<Y>(p.y, row[k] * p.y_ld + col[k], valid[k], v);
        }
    }
}

// ---- the sorted list

// An entry of the list: {ID : 32 | position : 32}; what has no row has n_table for an ID, and so comes last.
typedef unsigned long long Entry;
__device__ __forceinline__ uint32_t id_of(Entry e) { return static_cast<uint32_t>(e >> 32); }
__device__ __forceinline__ uint32_t position_of(Entry e) { return static_cast<uint32_t>(e); }

constexpr int kSmall = 2048;                        // lists that are ranked by comparing all with all
constexpr int kSortBlock = 512, kSortItems = 8, kSortTile = kSortBlock * kSortItems, kSortWaves = kSortBlock / kWave;
constexpr int kMostDigitBits = 8, kMostBins = 1 << kMostDigitBits, kLeastDigitBits = 4;
constexpr int kMostGroups = 256;                    // of consecutive tiles, a workgroup each
constexpr int kHeadGroups = 512;
constexpr int kFillBlocks = 2048;
constexpr int kMostChunks = 8192;                   // of a list of more than kSmall

struct GradArgs {
    Count rows;
    int32_t width;
    float scale;
    uint32_t n_table;
    const int32_t* ids;
    const void* dy;
    int64_t dy_ld;
    void* out;
    int64_t out_ld;
    int32_t* row_id;
    int64_t* n_distinct;                            // null: out is the whole table
    int32_t* err;
    // how the list is cut
    bool small;
    uint32_t n_groups, group_tiles;                 // of the sort
    uint32_t chunk;                                 // entries of a chunk: a power of two, 16 or more
    uint32_t head_span;                             // entries that a workgroup of heads_kernel counts
    uint32_t column_blocks;                         // of sum_kernel
    uint32_t fill_blocks;                           // workgroups of the first launch that clear dtable
    // scratch
    Entry* list[2];
    uint32_t* counts;                               // [n_groups][bins]
    uint32_t* chunk_rank;                           // heads of runs in front of a chunk, of those that its workgroup of heads_kernel counts
    uint32_t* group_heads;                          // heads that a workgroup of heads_kernel has counted
    int32_t* info;                                  // of a chunk: the row of the run that begins there and goes on; kThrough; or kNothing
    float* part;                                    // [chunks][2][width]: the part of a run from before, that of one that goes on
};
constexpr int32_t kNothing = -1, kThrough = -2;     // (kThrough: all of the chunk is one run that comes from before it and goes on)

__device__ __forceinline__ uint32_t key_of(const GradArgs& a, uint32_t position) {
    const int32_t id = a.ids[position];
    if (id >= 0 && static_cast<uint32_t>(id) < a.n_table) return static_cast<uint32_t>(id);
    if (id != -1) raise(a.err, kErrData);
    return a.n_table;
}

// dtable is cleared by workgroups of the first launch that have nothing else to do (rows that are met are written again later).
template <int TYPE>
__device__ __forceinline__ void clear_table(const GradArgs& a, uint32_t block) {
    const uint32_t blocks = static_cast<uint32_t>(a.width + 7) / 8;
    const int64_t items = static_cast<int64_t>(a.n_table) * blocks;
    const float zeros[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int64_t base = static_cast<int64_t>(block) * kSortBlock; base < items; base += static_cast<int64_t>(a.fill_blocks) * kSortBlock) {
        int64_t row;
        int32_t col;
        ItemPlaces(base, blocks).get(threadIdx.x, &row, &col);
        if (base + threadIdx.x < items) store_8_of<TYPE>(a.out, row * a.out_ld + col, a.width - col, zeros);
    }
}

// Short lists: a workgroup ranks 64 of the IDs, each of its waves against a share of all of them.
constexpr uint32_t kRanked = kWave;
template <int TYPE>
__global__ __launch_bounds__(kSortBlock) void rank_kernel(GradArgs a, uint32_t rank_blocks) {
    __shared__ uint32_t s_key[kSmall];
    __shared__ uint32_t s_rank[kSortWaves][kRanked];
    if (blockIdx.x >= rank_blocks) {
        clear_table<TYPE>(a, blockIdx.x - rank_blocks);
        return;
    }
    const uint32_t n = static_cast<uint32_t>(a.rows.get());
    for (uint32_t i = threadIdx.x; i < n; i += kSortBlock) s_key[i] = key_of(a, i);
    __syncthreads();
    const uint32_t lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, first = blockIdx.x * kRanked, mine = first + lane;
    const uint32_t share = (n + kSortWaves - 1) / kSortWaves, from = wave * share, to = min(from + share, n);
    const uint32_t key = mine < n ? s_key[mine] : 0;
    uint32_t rank = 0;
    for (uint32_t j = from; j < to; ++j) rank += s_key[j] < key + (j < mine ? 1u : 0u) ? 1u : 0u;      // (equal IDs: those in front)
    s_rank[wave][lane] = rank;
    __syncthreads();
    if (wave != 0 || mine >= n) return;
    rank = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) rank += s_rank[w][lane];
    a.list[0][rank] = static_cast<Entry>(key) << 32 | mine;
}

// A digit of the radix sort: `bits` bits of the ID from `shift` on.
struct Digit {
    int from;                                       // the list it sorts: -1 the IDs as given, else list[from]
    int to;
    uint32_t shift, bits;
    __device__ __forceinline__ uint32_t bins() const { return 1u << bits; }
    __device__ __forceinline__ uint32_t of(uint32_t key) const { return key >> shift & (bins() - 1); }
};
__device__ __forceinline__ Entry entry_at(const GradArgs& a, const Digit& d, uint32_t i) {
    if (d.from < 0) return static_cast<Entry>(key_of(a, i)) << 32 | i;
    return d.from == 0 ? a.list[0][i] : a.list[1][i];
}

// How many entries of every digit a group of tiles has.
template <int TYPE>
__global__ __launch_bounds__(kSortBlock) void count_kernel(GradArgs a, Digit d) {
    __shared__ uint32_t s_count[kMostBins];
    if (blockIdx.x >= a.n_groups) {
        clear_table<TYPE>(a, blockIdx.x - a.n_groups);
        return;
    }
    const uint32_t n = static_cast<uint32_t>(a.rows.get());
    for (uint32_t b = threadIdx.x; b < d.bins(); b += kSortBlock) s_count[b] = 0;
    __syncthreads();
    for (uint32_t tile = 0; tile < a.group_tiles; ++tile) {
        const uint32_t first = (blockIdx.x * a.group_tiles + tile) * kSortTile + threadIdx.x;
#pragma unroll
        for (int k = 0; k < kSortItems; ++k)
            if (first + k * kSortBlock < n) atomicAdd(s_count + d.of(id_of(entry_at(a, d, first + k * kSortBlock))), 1u);
    }
    __syncthreads();
    for (uint32_t b = threadIdx.x; b < d.bins(); b += kSortBlock) a.counts[blockIdx.x * d.bins() + b] = s_count[b];
}

// An exclusive sum over the threads of a workgroup of kSortBlock; *all: the sum of all.
__device__ __forceinline__ uint32_t sum_before(uint32_t v, uint32_t* s_wave, uint32_t* all) {
    const uint32_t inc = dpp_inclusive_scan(v);
    __syncthreads();
    if (lane_id() == kWave - 1) s_wave[wave_id()] = inc;
    __syncthreads();
    uint32_t before = inc - v;
    *all = 0;
    for (int w = 0; w < static_cast<int>(blockDim.x) / kWave; ++w) {
        if (w < wave_id()) before += s_wave[w];
        *all += s_wave[w];
    }
    return before;
}

// Puts a group's entries where they belong.  Every workgroup adds up the groups' counts itself: all of them for where a digit begins, those of
// the groups before for where its own entries of it go.
__global__ __launch_bounds__(kSortBlock) void place_kernel(GradArgs a, Digit d) {
    __shared__ uint32_t s_next[kMostBins];          // where the next entry of a digit goes
    __shared__ uint32_t s_count[kSortWaves][kMostBins];
    __shared__ uint32_t s_wave[kSortWaves];
    __shared__ uint32_t s_total[kSortBlock][4], s_before[kSortBlock][4];
    typedef uint32_t words4 __attribute__((ext_vector_type(4)));
    const uint32_t n = static_cast<uint32_t>(a.rows.get()), bins = d.bins(), t = threadIdx.x, lane = t % kWave, wave = t / kWave;
    {
        const uint32_t quads = bins / 4, shares = kSortBlock / quads, quad = t % quads, share = t / quads;
        words4 total = {0, 0, 0, 0}, before = {0, 0, 0, 0};
#pragma unroll 8
        for (uint32_t g = share; g < a.n_groups; g += shares) {
            const words4 c = reinterpret_cast<const words4*>(a.counts + g * bins)[quad];
            total += c;
            if (g < blockIdx.x) before += c;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) s_total[t][e] = total[e], s_before[t][e] = before[e];
        __syncthreads();
        uint32_t sum = 0, at = 0;
        if (t < bins)
            for (uint32_t s = 0; s < shares; ++s) sum += s_total[s * quads + t / 4][t % 4], at += s_before[s * quads + t / 4][t % 4];
        uint32_t all;
        const uint32_t digit_begin = sum_before(sum, s_wave, &all);
        if (t < bins) s_next[t] = digit_begin + at;
    }
    for (uint32_t tile = 0; tile < a.group_tiles; ++tile) {
        const uint32_t begin = (blockIdx.x * a.group_tiles + tile) * kSortTile;
        if (begin >= n) break;
        for (uint32_t b = t; b < kSortWaves * bins; b += kSortBlock) s_count[b / bins][b % bins] = 0;
        __syncthreads();
        // a wave has kSortItems times 64 neighbouring entries; a lane's rank among those of its digit: lanes below and rounds before
        Entry entry[kSortItems];
        uint32_t rank[kSortItems];
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) {
            const uint32_t i = begin + wave * (kSortItems * kWave) + k * kWave + lane;
            entry[k] = i < n ? entry_at(a, d, i) : ~Entry{0};
        }
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) {
            const bool there = begin + wave * (kSortItems * kWave) + k * kWave + lane < n;
            const uint32_t digit = d.of(id_of(entry[k]));
            uint64_t peers = __ballot(there);
            for (uint32_t b = 0; b < d.bits; ++b) {
                const bool one = digit >> b & 1;
                const uint64_t ones = __ballot(one);
                peers &= one ? ones : ~ones;
            }
            const uint32_t below = rank_in_mask(peers);
            volatile uint32_t* word = &s_count[wave][digit];
            rank[k] = *word + below;
            __builtin_amdgcn_wave_barrier();
            if (there && below == 0) *word = *word + static_cast<uint32_t>(__popcll(peers));
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        if (t < bins) {
            uint32_t at = s_next[t];
            for (int w = 0; w < kSortWaves; ++w) {
                const uint32_t c = s_count[w][t];
                s_count[w][t] = at;
                at += c;
            }
            s_next[t] = at;
        }
        __syncthreads();
        Entry* to = d.to == 0 ? a.list[0] : a.list[1];
#pragma unroll
        for (int k = 0; k < kSortItems; ++k)
            if (begin + wave * (kSortItems * kWave) + k * kWave + lane < n) to[s_count[wave][d.of(id_of(entry[k]))] + rank[k]] = entry[k];
        __syncthreads();
    }
}

// ---- runs of equal IDs

// The heads of runs among the eight entries from `at` on (those of IDs that have a row).
__device__ __forceinline__ uint32_t heads_of_8(const Entry* list, uint32_t at, uint32_t n, uint32_t n_table) {
    uint32_t heads = 0, before = at > 0 && at < n ? id_of(list[at - 1]) : ~0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t id = at + e < n ? id_of(list[at + e]) : n_table;
        heads += id < n_table && id != before ? 1u : 0u;
        before = id;
    }
    return heads;
}
__global__ __launch_bounds__(kSortBlock) void heads_kernel(GradArgs a, const Entry* list) {
    __shared__ uint32_t s_wave[kSortWaves];
    const uint32_t n = static_cast<uint32_t>(a.rows.get());
    uint32_t run = 0;
    for (uint32_t from = 0; from < a.head_span; from += kSortTile) {
        const uint32_t at = blockIdx.x * a.head_span + from + threadIdx.x * 8;
        uint32_t all;
        const uint32_t before = sum_before(heads_of_8(list, at, n, a.n_table), s_wave, &all);
        if (at < n && at % a.chunk == 0) a.chunk_rank[at / a.chunk] = run + before;
        run += all;
    }
    if (threadIdx.x == 0) a.group_heads[blockIdx.x] = run;
}

// The bits of a wave's mask that belong to this group of G lanes.
template <int G>
__device__ __forceinline__ uint64_t group_bits(uint64_t mask) {
    if (G == kWave) return mask;
    return mask >> (threadIdx.x % kWave / G * G) & ((uint64_t{1} << (G % 64)) - 1);
}

// A chunk to a group of G lanes, eight columns to a lane.
constexpr int kRowsAhead = 8;
template <int TYPE, int Y, int G>
__global__ __launch_bounds__(kBlock) void sum_kernel(GradArgs a, const Entry* list, uint32_t n_tasks) {
    __shared__ uint32_t s_wave[kBlock / kWave];
    __shared__ uint32_t s_rank[kSmall / 16];
    constexpr uint32_t kGroups = kBlock / G;
    const uint32_t n = static_cast<uint32_t>(a.rows.get()), n_chunks = (n + a.chunk - 1) / a.chunk, lane = threadIdx.x % G;
    if (a.n_distinct && a.small) {
        uint32_t all;
        const uint32_t before = sum_before(heads_of_8(list, threadIdx.x * 8, n, a.n_table), s_wave, &all);
        if (threadIdx.x * 8 < n && threadIdx.x * 8 % a.chunk == 0) s_rank[threadIdx.x * 8 / a.chunk] = before;
        __syncthreads();
    }
    for (uint32_t task = blockIdx.x; task < n_tasks; task += gridDim.x) {
        const uint32_t column_block = task % a.column_blocks, chunk = task / a.column_blocks * kGroups + threadIdx.x / G;
        const int32_t col = static_cast<int32_t>(column_block * G + lane) * 8, valid = a.width - col;
        const uint32_t begin = chunk < n_chunks ? chunk * a.chunk : n, end = min(begin + a.chunk, n);

        // the row of drow of the first run that begins here
        uint32_t rank = 0;
        if (a.n_distinct && a.small) {
            if (begin < n) rank = s_rank[chunk];
        } else if (a.n_distinct) {
            if (begin < n)
                for (uint32_t g = lane; g < begin / a.head_span; g += G) rank += a.group_heads[g];
#pragma unroll
            for (int d = G / 2; d >= 1; d >>= 1) rank += __shfl_xor(rank, d, kWave);
            if (begin < n) rank += a.chunk_rank[chunk];
        }

        float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        bool any = false, headless = true;              // something in acc; no run has begun here so far
        int32_t row = 0;                                // of the run in acc
        const auto to_part = [&](int which) { store_8_of<kF32>(a.part, (static_cast<int64_t>(chunk) * 2 + which) * a.width + col, valid, acc); };
        const auto to_row = [&] {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = acc[e] * a.scale;
            store_8_of<TYPE>(a.out, row * a.out_ld + col, valid, v);
        };
        const uint32_t batch = a.chunk < G ? a.chunk : G;
        for (uint32_t from = 0; from < a.chunk; from += batch) {
            const uint32_t at = begin + from + lane;
            const bool in = lane < batch && at < end;
            const Entry mine = in ? list[at] : 0;
            const bool there = in && id_of(mine) < a.n_table, head = there && (at == 0 || id_of(list[at - 1]) != id_of(mine));
            const uint64_t theres = group_bits<G>(__ballot(there)), heads = group_bits<G>(__ballot(head));
            if (head && a.n_distinct && column_block == 0) a.row_id[rank + __popcll(heads & ((uint64_t{1} << lane) - 1))] = static_cast<int32_t>(id_of(mine));
            for (uint32_t q = 0; q < batch; q += kRowsAhead) {
                Raw8<Y> raw[kRowsAhead];
                int32_t id[kRowsAhead];
#pragma unroll
                for (int k = 0; k < kRowsAhead; ++k) {
                    const uint32_t position = __shfl(position_of(mine), q + k, G);
                    id[k] = __shfl(static_cast<int32_t>(id_of(mine)), q + k, G);
                    raw[k].load(a.dy, position * a.dy_ld + col, theres >> (q + k) & 1 ? valid : 0);
                }
#pragma unroll
                for (int k = 0; k < kRowsAhead; ++k) {
                    if (!(theres >> (q + k) & 1)) continue;
                    if (heads >> (q + k) & 1) {
                        if (any && headless) to_part(0);
                        else if (any) to_row();
                        headless = false;
                        row = a.n_distinct ? static_cast<int32_t>(rank) : id[k];
                        ++rank;
#pragma unroll
                        for (int e = 0; e < 8; ++e) acc[e] = 0;
                    }
                    any = true;
                    float v[8];
                    widen_8<Y>(raw[k].v, v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[e] += v[e];
                }
            }
        }
        if (begin < n) {
            const uint32_t last = id_of(list[end - 1]);
            const bool goes_on = last < a.n_table && end < n && id_of(list[end]) == last;
            if (any && headless) to_part(0);
            else if (any && goes_on) to_part(1);
            else if (any) to_row();
            if (column_block == 0 && lane == 0) a.info[chunk] = !any || !goes_on ? kNothing : headless ? kThrough : row;
        }
        if (a.n_distinct && column_block == 0 && lane == 0 && chunk + 1 == (n_chunks > 0 ? n_chunks : 1)) *a.n_distinct = rank;
    }
}

// Adds the parts of a run that begins in a chunk and goes on: eight lanes to 64 columns, and as many parts at a time as there are such lanes.
constexpr int kMergeColumns = 64, kMergeSubs = kBlock / (kMergeColumns / 8);
template <int TYPE>
__global__ __launch_bounds__(kBlock) void merge_kernel(GradArgs a, uint32_t column_blocks, uint32_t n_tasks) {
    __shared__ float s[kMergeSubs][kMergeColumns + 1];
    __shared__ uint32_t s_last;
    const uint32_t n = static_cast<uint32_t>(a.rows.get()), n_chunks = (n + a.chunk - 1) / a.chunk;
    for (uint32_t task = blockIdx.x; task < n_tasks; task += gridDim.x) {
        const uint32_t chunk = task / column_blocks;
        const int32_t row = chunk < n_chunks ? a.info[chunk] : kNothing;
        if (row < 0) continue;
        if (threadIdx.x == 0) s_last = n_chunks;
        __syncthreads();
        for (uint32_t from = chunk + 1; from < n_chunks; from += kBlock) {       // the first chunk that the run does not go through
            const uint32_t c = from + threadIdx.x;
            if (c < n_chunks && a.info[c] != kThrough) atomicMin(&s_last, c);
            __syncthreads();
            const bool found = s_last < n_chunks;
            __syncthreads();
            if (found) break;
        }
        const uint32_t last = min(s_last, n_chunks - 1), sub = threadIdx.x / 8;
        const int32_t first_col = static_cast<int32_t>(task % column_blocks) * kMergeColumns, at = threadIdx.x % 8 * 8, col = first_col + at, valid = a.width - col;
        float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (valid > 0) {
            if (sub == 0) load_8_of<kF32>(a.part, (static_cast<int64_t>(chunk) * 2 + 1) * a.width + col, valid, acc);
#pragma unroll 4
            for (uint32_t c = chunk + 1 + sub; c <= last; c += kMergeSubs) {
                float v[8];
                load_8_of<kF32>(a.part, static_cast<int64_t>(c) * 2 * a.width + col, valid, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] += v[e];
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) s[sub][at + e] = acc[e];
        __syncthreads();
        if (threadIdx.x < kMergeColumns && first_col + static_cast<int32_t>(threadIdx.x) < a.width) {
            float v = 0;
#pragma unroll
            for (int k = 0; k < kMergeSubs; ++k) v += s[k][threadIdx.x];
            store_1(TYPE, a.out, row * a.out_ld + first_col + static_cast<int32_t>(threadIdx.x), v * a.scale);
        }
        __syncthreads();
    }
}

// ---- launches

int lanes_for(int32_t width) { return width <= 128 ? 16 : width <= 256 ? 32 : 64; }
uint32_t ceil_div(int64_t a, int64_t b) { return static_cast<uint32_t>((a + b - 1) / b); }

// How a list is cut, and how much scratch it takes.
struct GradPlan {
    GradArgs a;
    uint32_t n_chunks, head_groups;
    size_t bytes;
    GradPlan(const EmbeddingGradJob& job, char* scratch) {
        const int64_t n = job.rows.host;
        a = GradArgs{};
        a.rows = job.rows;
        a.width = job.width, a.scale = job.scale, a.n_table = static_cast<uint32_t>(job.n_table);
        a.ids = job.ids, a.dy = job.dy, a.dy_ld = job.dy_ld, a.out = job.out, a.out_ld = job.out_ld;
        a.row_id = job.row_id, a.n_distinct = job.n_distinct, a.err = job.err;
        a.small = n <= kSmall;
        const int64_t tiles = (n + kSortTile - 1) / kSortTile;
        a.group_tiles = std::max<uint32_t>(1, ceil_div(tiles, kMostGroups));
        a.n_groups = ceil_div(tiles, a.group_tiles);
        a.chunk = a.small ? 16 : 32;
        while (n > static_cast<int64_t>(a.chunk) * kMostChunks) a.chunk *= 2;
        a.head_span = std::max<uint32_t>(1, ceil_div(tiles, kHeadGroups)) * kSortTile;
        a.column_blocks = ceil_div(a.width, 8 * lanes_for(a.width));
        a.fill_blocks = job.n_distinct ? 0 : static_cast<uint32_t>(std::min<int64_t>(kFillBlocks, ceil_div(job.n_table * ((job.width + 7) / 8), kSortBlock)));
        n_chunks = ceil_div(n, a.chunk);
        head_groups = ceil_div(n, a.head_span);
        bytes = 0;
        const auto take = [&](auto** to, size_t count) {
            *to = reinterpret_cast<std::remove_reference_t<decltype(**to)>*>(scratch + bytes);
            bytes = (bytes + count * sizeof(**to) + 255) / 256 * 256;
        };
        take(&a.list[0], n);
        take(&a.list[1], a.small ? 0 : n);
        take(&a.counts, a.small ? 0 : static_cast<size_t>(a.n_groups) * kMostBins);
        take(&a.chunk_rank, n_chunks);
        take(&a.group_heads, head_groups);
        take(&a.info, n_chunks);
        take(&a.part, static_cast<size_t>(n_chunks) * 2 * a.width);
    }
};

template <int TYPE, int Y>
hipError_t run_grad(hipStream_t stream, const GradPlan& plan) {
    const GradArgs& a = plan.a;
    const int64_t n = a.rows.host;
    const Entry* list = a.list[0];
    if (a.small) {
        const uint32_t rank_blocks = ceil_div(n, kRanked);
        if (rank_blocks + a.fill_blocks > 0)
            hipLaunchKernelGGL(rank_kernel<TYPE>, dim3(rank_blocks + a.fill_blocks), dim3(kSortBlock), 0, stream, a, rank_blocks);
    } else {
        const uint32_t id_bits = 32 - static_cast<uint32_t>(__builtin_clz(a.n_table | 1)), passes = ceil_div(id_bits, kMostDigitBits);
        const uint32_t bits = std::max<uint32_t>(kLeastDigitBits, ceil_div(id_bits, passes));
        for (uint32_t p = 0; p < passes; ++p) {
            const Digit d{static_cast<int>(p == 0 ? -1 : (p - 1) % 2), static_cast<int>(p % 2), p * bits, bits};
            hipLaunchKernelGGL(count_kernel<TYPE>, dim3(a.n_groups + (p == 0 ? a.fill_blocks : 0)), dim3(kSortBlock), 0, stream, a, d);
            hipLaunchKernelGGL(place_kernel, dim3(a.n_groups), dim3(kSortBlock), 0, stream, a, d);
        }
        list = a.list[(passes - 1) % 2];
        if (a.n_distinct) hipLaunchKernelGGL(heads_kernel, dim3(plan.head_groups), dim3(kSortBlock), 0, stream, a, list);
    }
    if (n < 1 && !a.n_distinct) return hipGetLastError();
    const int lanes = lanes_for(a.width);
    const uint32_t tasks = std::max<uint32_t>(1, ceil_div(plan.n_chunks, kBlock / lanes)) * a.column_blocks;      // (fewer than 2^31: kMostChunks)
    const dim3 grid(std::min<uint32_t>(tasks, kMostBlocks));
    if (lanes == 16) hipLaunchKernelGGL((sum_kernel<TYPE, Y, 16>), grid, dim3(kBlock), 0, stream, a, list, tasks);
    else if (lanes == 32) hipLaunchKernelGGL((sum_kernel<TYPE, Y, 32>), grid, dim3(kBlock), 0, stream, a, list, tasks);
    else hipLaunchKernelGGL((sum_kernel<TYPE, Y, 64>), grid, dim3(kBlock), 0, stream, a, list, tasks);
    if (plan.n_chunks > 1) {
        const uint32_t columns = ceil_div(a.width, kMergeColumns), merges = plan.n_chunks * columns;
        hipLaunchKernelGGL(merge_kernel<TYPE>, dim3(std::min<uint32_t>(merges, kMostBlocks)), dim3(kBlock), 0, stream, a, columns, merges);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embedding(hipStream_t stream, const EmbeddingJob& job) {
    if (job.rows.host < 1) return hipSuccess;
    const int64_t items = job.rows.host * ((job.width + 7) / 8);
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>((items + kBlock * kItems - 1) / (kBlock * kItems), kMostBlocks))), block(kBlock);
    if (job.table_type == kF16) hipLaunchKernelGGL((embedding_kernel<kF16, kF16>), grid, block, 0, stream, job);
    else if (job.table_type == kBF16) hipLaunchKernelGGL((embedding_kernel<kBF16, kBF16>), grid, block, 0, stream, job);
    else if (job.y_type == kF16) hipLaunchKernelGGL((embedding_kernel<kF32, kF16>), grid, block, 0, stream, job);
    else if (job.y_type == kBF16) hipLaunchKernelGGL((embedding_kernel<kF32, kBF16>), grid, block, 0, stream, job);
    else hipLaunchKernelGGL((embedding_kernel<kF32, kF32>), grid, block, 0, stream, job);
    return hipGetLastError();
}

size_t embedding_grad_scratch_bytes(const EmbeddingGradJob& job) { return GradPlan(job, nullptr).bytes; }

hipError_t launch_embedding_grad(hipStream_t stream, const EmbeddingGradJob& job, void* scratch) {
    const GradPlan plan(job, static_cast<char*>(scratch));
    if (job.table_type == kF16) return run_grad<kF16, kF16>(stream, plan);
    if (job.table_type == kBF16) return run_grad<kBF16, kBF16>(stream, plan);
    if (job.y_type == kF16) return run_grad<kF32, kF16>(stream, plan);
    if (job.y_type == kBF16) return run_grad<kF32, kBF16>(stream, plan);
    return run_grad<kF32, kF32>(stream, plan);
}

}  // namespace helios
