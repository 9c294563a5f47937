// Learnt rows by ID, and the gradient of their table by the sorted list of IDs.
//
//   y[i] = add[i] + scale * table[id_i];   dtable[k] = scale * sum of dy[i] over the positions i with id_i = k
//
// The lookup is bound by memory: every row that is met once, add and y (204 800 rows of 256, the table in single precision, add and y in half: 71 us,
// 5.9 TB/s, where a large copy reaches 6.4).
// The gradient of a longer list sorts {ID, position} (stable), cuts the sorted list into chunks of equal length whatever the IDs, and lets a wave sum a
// chunk, run of equal IDs by run: a run that lies in one chunk is finished there, one that goes on leaves a part for every chunk it meets, and a
// last kernel adds these.  So a list of one ID costs what a list of distinct ones does, no sum is made by atomics, and the same list gives
// the same bits.  What bounds it is the rows of dy, read once, and in front of that the chain of short launches that sorts the list, two for every
// digit: 281 600 rows of 128 in single precision, IDs below two million, are 100 us, 50 for the rows, 5 for the parts, and 41 for the list.
// Lists of up to 4096 are not sorted (few_kernel) unless their rows are wide.
#include "layer.hpp"
#include "layer_dev.hpp"

#include <algorithm>

namespace helios {

namespace {

constexpr int64_t kMostBlocks = 1 << 21;            // of a launch

// ---- lookup

constexpr int kItems = 2;                           // of a thread, in flight together
// (An ID without a row loads the table's first, so that the load depends on no branch)
template <int TABLE, int Y, int ROWS>
__global__ __launch_bounds__(kBlock) void embedding_kernel(EmbeddingJob p) {
    const uint32_t blocks = static_cast<uint32_t>(p.width + 7) / 8;
    const int64_t items = p.rows.get() * blocks, step = static_cast<int64_t>(gridDim.x) * kBlock * kItems;
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * kBlock * kItems; base < items; base += step) {
        const ItemPlaces places(base, blocks);
        const uint32_t left = items - base < kBlock * kItems ? static_cast<uint32_t>(items - base) : kBlock * kItems;
        Raw8<TABLE> row_raw[kItems];
        Raw8<Y> add_raw[kItems];
        uint32_t down[kItems];
        int32_t col[kItems], id[kItems];
        bool there[kItems];
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            const uint32_t i = k * kBlock + threadIdx.x;
            places.get(i < left ? i : left - 1, &down[k], &col[k]);
            id[k] = (p.ids + places.row0)[down[k]];
        }
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            there[k] = id[k] >= 0 && id[k] < p.n_table;
            if (!there[k] && id[k] != -1) raise(p.err, kErrData);
            row_raw[k].clear();
            if (p.n_table > 0) row_raw[k].template load_row<ROWS>(p.table, (there[k] ? id[k] : 0) * p.table_ld, col[k], p.width);
            if (p.add) add_raw[k].template load_row<ROWS>(p.add, places.row(p.add_ld, down[k]), col[k], p.width);
        }
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            float v[8], a[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            row_raw[k].template align<ROWS>(col[k], p.width);
            widen_8<TABLE>(row_raw[k].v, v);
            if (p.add) {
                add_raw[k].template align<ROWS>(col[k], p.width);
                widen_8<Y>(add_raw[k].v, a);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = there[k] ? __builtin_fmaf(v[e], p.scale, a[e]) : a[e];
            if (k * kBlock + threadIdx.x < left) store_row_8<Y, ROWS>(p.y, places.row(p.y_ld, down[k]), col[k], p.width, v);
        }
    }
}

// ---- the sorted list

// An entry of the list: {ID : 32 | position : 32}; what has no row has n_table for an ID, and so comes last.
typedef unsigned long long Entry;
__device__ __forceinline__ uint32_t id_of(Entry e) { return static_cast<uint32_t>(e >> 32); }
__device__ __forceinline__ uint32_t position_of(Entry e) { return static_cast<uint32_t>(e); }

// A list that is not sorted (few_kernel) has kFew entries at most, and its rows few columns: every workgroup of few_kernel goes through the whole list, so
// that what it takes grows with (entries + 1000) for every 512 workgroups, where the sorted list is paid for once.  Distinct IDs, single
// precision, us for both: 4096 of 256 (512 workgroups) 26 and 33, of 512 49 and 34, of 1024 96 and 36; 2048 of 1024 (1024 workgroups) 29 and 32, of 2048 60 and 33;
// 1000 of 2048 (1000) 19 and 30, of 4096 38 and 32; 300 of 8192 (1216) 14 and 28.
constexpr int kFew = 4096;
constexpr int64_t kFewWork = 3'900'000;             // workgroups times (entries + 1000)
constexpr int kSortBlock = 512, kSortItems = 4, kSortTile = kSortBlock * kSortItems, kSortWaves = kSortBlock / kWave;
constexpr int kMostDigitBits = 9, kMostBins = 1 << kMostDigitBits, kLeastDigitBits = 4;
constexpr int kMostGroups = 256;                    // of consecutive tiles, a workgroup each
constexpr int kHeadGroups = 512;
constexpr int kFillBlocks = 2048;
// Workgroups that clear dtable times (entries + 1000) beside few_kernel's others, where they go through the list too, to see which rows are met; more are a launch
// in front, for 2.5 us.  The larger the table, the more of this hides behind memory.  Of 256 columns in single precision, us beside and in front: 4096 entries
// and 2000 rows 18.5 and 18.2, 16 000 rows 42 and 26, 200 000 rows 116 and 62; 1000 entries 7.5 and 9.9, 22 and 16, 53 and 45; 300 entries and 200 000 rows 39 and 43.
constexpr int64_t kFillWork = 1 << 20, kFillHidden = 100;             // (and a workgroup times an entry for every 100 bytes of the table)
constexpr int kMostChunks = 4096;                   // of a list

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
    bool few;                                       // it is not sorted at all (few_kernel)
    uint32_t n_groups, group_tiles;                 // of the sort
    uint32_t chunk;                                 // entries of a chunk: a power of two, 32 or more
    uint32_t head_span;                             // entries that a workgroup of heads_kernel counts
    uint32_t column_blocks;                         // of sum_kernel
    uint32_t fill_blocks;                           // workgroups of the first launch that clear dtable
    bool fill_first;                                // ... which is a launch of its own, in front of few_kernel
    // scratch
    Entry* list[2];
    uint32_t* counts;                               // [n_groups][bins]
    uint32_t* chunk_rank;                           // heads of runs in front of a chunk, of those that its workgroup of heads_kernel counts
    uint32_t* group_heads;                          // heads that a workgroup of heads_kernel has counted
    int32_t* info;                                  // of a chunk: the row of the run that begins there and goes on; kThrough; or kNothing
    float* part;                                    // [chunks][2][width]: the part of a run from before, that of one that goes on
};
constexpr int32_t kNothing = -1, kThrough = -2;     // (kThrough: all of the chunk is one run that comes from before it and goes on)

// The ID an entry has, if it is there.
__device__ __forceinline__ uint32_t key_of(const GradArgs& a, int32_t id, bool there) {
    if (there && id >= 0 && static_cast<uint32_t>(id) < a.n_table) return static_cast<uint32_t>(id);
    if (there && id != -1) raise(a.err, kErrData);
    return a.n_table;
}

// dtable is cleared by workgroups of the first launch that have nothing else to do (rows that are met are written again later).
template <int TYPE>
__device__ __forceinline__ void clear_table(const GradArgs& a, uint32_t block) {
    const uint32_t blocks = static_cast<uint32_t>(a.width + 7) / 8;
    const int64_t items = static_cast<int64_t>(a.n_table) * blocks;
    const float zeros[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int64_t base = static_cast<int64_t>(block) * kSortBlock; base < items; base += static_cast<int64_t>(a.fill_blocks) * kSortBlock) {
        const ItemPlaces places(base, blocks);
        uint32_t down;
        int32_t col;
        places.get(threadIdx.x, &down, &col);
        if (base + threadIdx.x < items) store_8_of<TYPE>(a.out, places.row(a.out_ld, down) + col, a.width - col, zeros);
    }
}

template <int TYPE>
__global__ __launch_bounds__(kSortBlock) void clear_kernel(GradArgs a) { clear_table<TYPE>(a, blockIdx.x); }

// A digit of the radix sort: `bits` bits of the ID from `shift` on.
struct Digit {
    int from;                                       // the list it sorts: -1 the IDs as given, else list[from]
    int to;
    uint32_t shift, bits;
    __device__ __forceinline__ uint32_t bins() const { return 1u << bits; }
    __device__ __forceinline__ uint32_t of(uint32_t key) const { return key >> shift & (bins() - 1); }
};
// kSortItems entries, `step` apart from `first` on; all ones where there are none.  (No load depends on a branch: what is not there reads the last entry,
// or the first place of an empty list.)
__device__ __forceinline__ void load_entries(const GradArgs& a, const Digit& d, uint32_t first, uint32_t step, uint32_t n, Entry (&entry)[kSortItems]) {
    const uint32_t last = n > 0 ? n - 1 : 0;
    if (d.from < 0) {
        int32_t id[kSortItems];
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) id[k] = a.ids[min(first + k * step, last)];
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) entry[k] = static_cast<Entry>(key_of(a, id[k], first + k * step < n)) << 32 | (first + k * step);
    } else {
        const Entry* list = d.from == 0 ? a.list[0] : a.list[1];
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) entry[k] = list[min(first + k * step, last)];
    }
#pragma unroll
    for (int k = 0; k < kSortItems; ++k)
        if (first + k * step >= n) entry[k] = ~Entry{0};
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
        Entry entry[kSortItems];
        load_entries(a, d, first, kSortBlock, n, entry);
#pragma unroll
        for (int k = 0; k < kSortItems; ++k)
            if (first + k * kSortBlock < n) atomicAdd(s_count + d.of(id_of(entry[k])), 1u);
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
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t c = s_wave[w];
        if (w < wave_id()) before += c;
        *all += c;
    }
    return before;
}

// Puts a group's entries where they belong.  Every workgroup adds up the groups' counts itself: all of them for where a digit begins, those of
// the groups before for where its own entries of it go.  The entries of a tile are ranked among each other while the counts are on their way.
// A chain of loads, 7.5 us for 281 600 entries and digits of 7 bits (9 with loads of entries and counts behind branches): with digits of 10 or 11 bits, for a pass less, the whole gradient took twice as long;
// with at most 8, for which the 349 IDs of the other case take two passes, 44 us in place of 40.
constexpr int kCountsAhead = 8;
__global__ __launch_bounds__(kSortBlock) void place_kernel(GradArgs a, Digit d) {
    __shared__ uint32_t s_next[kMostBins];          // entries of the digit in the groups before; then where the next one of it goes
    __shared__ uint32_t s_total[kMostBins];
    __shared__ uint32_t s_count[kSortWaves * kMostBins];      // [waves][bins]
    __shared__ uint32_t s_wave[kSortWaves];
    typedef uint32_t words4 __attribute__((ext_vector_type(4)));
    const uint32_t n = static_cast<uint32_t>(a.rows.get()), bins = d.bins(), t = threadIdx.x, lane = t % kWave, wave = t / kWave;
    // a wave has kSortItems times 64 neighbouring entries of a tile
    const uint32_t first = blockIdx.x * a.group_tiles * kSortTile + wave * (kSortItems * kWave) + lane;
    Entry entry[kSortItems];
    const auto load = [&](uint32_t tile) { load_entries(a, d, first + tile * kSortTile, kWave, n, entry); };
    load(0);
    const uint32_t quads = bins / 4, shares = kSortBlock / quads, quad = t % quads, share = t / quads;
    words4 total = {0, 0, 0, 0}, before = {0, 0, 0, 0};
    for (uint32_t from = share; from < a.n_groups; from += kCountsAhead * shares) {
        words4 c[kCountsAhead];
#pragma unroll
        for (int k = 0; k < kCountsAhead; ++k) c[k] = reinterpret_cast<const words4*>(a.counts + min(from + k * shares, a.n_groups - 1) * bins)[quad];
#pragma unroll
        for (int k = 0; k < kCountsAhead; ++k) {
            const uint32_t g = from + k * shares;
            if (g < a.n_groups) total += c[k];
            if (g < blockIdx.x) before += c[k];
        }
    }
    for (uint32_t b = t; b < bins; b += kSortBlock) s_next[b] = s_total[b] = 0;
    for (uint32_t tile = 0; tile < a.group_tiles; ++tile) {
        const uint32_t at = first + tile * kSortTile;
        if (tile > 0) load(tile);
        for (uint32_t b = t; b < kSortWaves * bins; b += kSortBlock) s_count[b] = 0;
        __syncthreads();
        // a lane's rank among those of its digit: lanes below and rounds before
        uint32_t rank[kSortItems];
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) {
            const bool there = at + k * kWave < n;
            const uint32_t digit = d.of(id_of(entry[k]));
            uint64_t peers = __ballot(there);
            for (uint32_t b = 0; b < d.bits; ++b) {
                const bool one = digit >> b & 1;
                const uint64_t ones = __ballot(one);
                peers &= one ? ones : ~ones;
            }
            const uint32_t below = rank_in_mask(peers);
            volatile uint32_t* word = s_count + wave * bins + digit;
            rank[k] = *word + below;
            __builtin_amdgcn_wave_barrier();
            if (there && below == 0) *word = *word + static_cast<uint32_t>(__popcll(peers));
            __builtin_amdgcn_wave_barrier();
        }
        if (tile == 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                atomicAdd(s_total + 4 * quad + e, static_cast<uint32_t>(total[e]));
                atomicAdd(s_next + 4 * quad + e, static_cast<uint32_t>(before[e]));
            }
        }
        __syncthreads();
        if (tile == 0) {
            uint32_t run = 0;                       // entries of the digits before
            for (uint32_t from = 0; from < bins; from += kSortBlock) {
                const uint32_t b = from + t;
                uint32_t all;
                const uint32_t digit_begin = sum_before(b < bins ? s_total[b] : 0, s_wave, &all);
                if (b < bins) s_next[b] += run + digit_begin;
                run += all;
            }
        }
        for (uint32_t b = t; b < bins; b += kSortBlock) {
            uint32_t to = s_next[b], c[kSortWaves];
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) c[w] = s_count[w * bins + b];
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) {
                s_count[w * bins + b] = to;
                to += c[w];
            }
            s_next[b] = to;
        }
        __syncthreads();
        Entry* to = d.to == 0 ? a.list[0] : a.list[1];
#pragma unroll
        for (int k = 0; k < kSortItems; ++k)
            if (at + k * kWave < n) to[s_count[wave * bins + d.of(id_of(entry[k]))] + rank[k]] = entry[k];
        __syncthreads();
    }
}

// ---- runs of equal IDs

// The heads of runs among the eight entries from `at` on (those of IDs that have a row).
__device__ __forceinline__ uint32_t heads_of_8(const Entry* list, uint32_t at, uint32_t n, uint32_t n_table) {
    const uint32_t last = n > 0 ? n - 1 : 0;
    uint32_t heads = 0, id[9];
#pragma unroll
    for (int e = 0; e < 9; ++e) id[e] = id_of(list[min(at + e > 0 ? at + e - 1 : 0, last)]);
#pragma unroll
    for (int e = 0; e < 8; ++e) heads += at + e < n && id[e + 1] < n_table && (at + e == 0 || id[e] != id[e + 1]) ? 1u : 0u;
    return heads;
}
__global__ __launch_bounds__(kSortBlock) void heads_kernel(GradArgs a, const Entry* list) {
    __shared__ uint32_t s_wave[kSortWaves];
    const uint32_t n = static_cast<uint32_t>(a.rows.get());
    uint32_t run = 0;
    for (uint32_t from = 0; from < a.head_span; from += kSortBlock * 8) {
        const uint32_t at = blockIdx.x * a.head_span + from + threadIdx.x * 8;
        uint32_t all;
        const uint32_t before = sum_before(heads_of_8(list, at, n, a.n_table), s_wave, &all);
        if (at < n && at % a.chunk == 0) a.chunk_rank[at / a.chunk] = run + before;
        run += all;
    }
    if (threadIdx.x == 0) a.group_heads[blockIdx.x] = run;
}

// Where a row's elements are, V neighbouring ones to a lane of a wave (the fewest that reach over the row, at most 16 bytes), in blocks of 64 V columns.
// A lane whose columns would reach beyond the last takes the last V, and so reads, adds and writes what another does, too: no load depends on a
// branch, and so none waits for the one before it (sum_kernel on 281 600 rows of 128 in single precision: 50 us, with a branch around each 81).
template <int V>
struct LaneColumns {
    uint32_t at;                                    // the first of them
    bool any;                                       // a lane of which no column exists reads like the last that has some, and writes nothing
    __device__ __forceinline__ LaneColumns(uint32_t lane, uint32_t first, int32_t width) {
        const uint32_t w = static_cast<uint32_t>(width);
        any = first + lane * V < w;
        at = min(first + lane * V, w - V);
    }
};
// V neighbouring elements of a row, as they are in memory (rows start anywhere an element may).
template <int TYPE, int V>
struct Few {
    typedef typename ElementOf<TYPE>::type T;
    typedef T vector __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    T v[V];
    __device__ __forceinline__ void load(const T* p) { take(*reinterpret_cast<const vector*>(p)); }
    // hinted to leave the caches to others
    __device__ __forceinline__ void load_once(const T* p) { take(__builtin_nontemporal_load(reinterpret_cast<const vector*>(p))); }
    __device__ __forceinline__ void take(vector x) {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = x[e];
    }
    __device__ __forceinline__ void store(T* p) const {
        vector x;
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = v[e];
        *reinterpret_cast<vector*>(p) = x;
    }
    __device__ __forceinline__ void add(bool there, float (&to)[V]) const {
#pragma unroll
        for (int e = 0; e < V; ++e) to[e] += there ? static_cast<float>(v[e]) : 0.0f;
    }
};
// (one rounding to TYPE, to nearest, ties to even)
template <int TYPE, int V>
__device__ __forceinline__ void store_scaled(void* base, int64_t at, const float (&v)[V], float by) {
    typedef typename ElementOf<TYPE>::type T;
    Few<TYPE, V> o;
#pragma unroll
    for (int e = 0; e < V; ++e) o.v[e] = static_cast<T>(v[e] * by);
    o.store(static_cast<T*>(base) + at);
}

// ---- short lists

// The distinct IDs of a short list, in LDS.  A slot of the table holds a position, which stands for its ID; in the end the ID's first one.
struct FewLds {
    uint32_t key[kFew];
    uint32_t slot[2 * kFew];                        // twice as many as there are entries, so that a search ends soon, and ends
    unsigned long long heads[kFew / kWave];         // a bit for every position: the first one of an ID that has a row
};
constexpr uint32_t kNone = ~0u;
struct Slots {
    uint32_t bits;
    __device__ __forceinline__ explicit Slots(uint32_t n) : bits(n > kWave ? 33 - static_cast<uint32_t>(__builtin_clz(n - 1)) : 7) {}
    __device__ __forceinline__ uint32_t count() const { return 1u << bits; }
    __device__ __forceinline__ uint32_t first(uint32_t key) const { return key * 0x9e3779b1u >> (32 - bits); }
    __device__ __forceinline__ uint32_t next(uint32_t slot) const { return (slot + 1) & (count() - 1); }
};
__device__ __forceinline__ void find_distinct(const GradArgs& a, uint32_t n, const Slots& slots, FewLds& s) {
    constexpr int kMine = kFew / kSortBlock;
    uint32_t slot[kMine];
    int32_t id[kMine];
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
        if (k * kSortBlock >= n) break;
        id[k] = a.ids[min(k * kSortBlock + threadIdx.x, n - 1)];
    }
    for (uint32_t i = threadIdx.x; i < slots.count(); i += kSortBlock) s.slot[i] = kNone;
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
        const uint32_t i = k * kSortBlock + threadIdx.x;
        if (k * kSortBlock >= n) break;
        s.key[i] = key_of(a, id[k], i < n);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
        if (k * kSortBlock >= n) break;
        const uint32_t i = k * kSortBlock + threadIdx.x, key = s.key[i];
        slot[k] = slots.first(key);
        if (key >= a.n_table) continue;
        for (;;) {
            const uint32_t there = atomicCAS(s.slot + slot[k], kNone, i);
            if (there == kNone) break;
            if (s.key[there] == key) {
                atomicMin(s.slot + slot[k], i);
                break;
            }
            slot[k] = slots.next(slot[k]);
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
        if (k * kSortBlock >= n) break;
        const uint32_t i = k * kSortBlock + threadIdx.x;
        const unsigned long long heads = __ballot(s.key[i] < a.n_table && s.slot[slot[k]] == i);
        if (lane_id() == 0) s.heads[i / kWave] = heads;
    }
    __syncthreads();
}
__device__ __forceinline__ bool is_met(const FewLds& s, const Slots& slots, uint32_t key) {
    for (uint32_t at = slots.first(key); s.slot[at] != kNone; at = slots.next(at))
        if (s.key[s.slot[at]] == key) return true;
    return false;
}

// A list of up to kFew IDs in one launch and without a sort: every workgroup finds the distinct IDs for itself; a wave has a position, and if
// that is its ID's first one, looks through the whole list for the ID's other positions and for how many distinct IDs are less, which
// is the row's number.  An ID with more than kLongRun positions is left to all waves of its workgroup.  Rows of dtable that are not met are cleared by
// workgroups of their own, or by a launch in front (kFillWork).  What bounds it is the chain of steps in LDS: 777 rows of 200 take 7 us, 2600 of 128 17 (sorted: 38), 4000 28 (39); at 6000,
// for which LDS has room for one workgroup on a CU, 87 and 40, so that kFew is 4096.
constexpr int kLongRun = 64, kRowsAhead = 8;
template <int TYPE, int Y, int V>
__global__ __launch_bounds__(kSortBlock) void few_kernel(GradArgs a, uint32_t sum_blocks) {
    typedef typename ElementOf<Y>::type T;
    __shared__ FewLds s;
    __shared__ uint32_t s_position[kSortWaves][kLongRun];
    __shared__ uint32_t s_long[kSortWaves];         // the ID of a wave's long run, and its row
    __shared__ uint32_t s_row[kSortWaves];
    __shared__ float s_part[kSortWaves][V][kWave];
    const uint32_t n = static_cast<uint32_t>(a.rows.get());
    const Slots slots(n);
    find_distinct(a, n, slots, s);
    if (blockIdx.x >= sum_blocks) {
        const uint32_t blocks = static_cast<uint32_t>(a.width + 7) / 8;
        const int64_t items = static_cast<int64_t>(a.n_table) * blocks;
        const float zeros[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        for (int64_t base = static_cast<int64_t>(blockIdx.x - sum_blocks) * kSortBlock; base < items; base += static_cast<int64_t>(a.fill_blocks) * kSortBlock) {
            const ItemPlaces places(base, blocks);
            uint32_t down;
            int32_t col;
            places.get(threadIdx.x, &down, &col);
            if (base + threadIdx.x < items && !is_met(s, slots, static_cast<uint32_t>(places.row0 + down)))
                store_8_of<TYPE>(a.out, places.row(a.out_ld, down) + col, a.width - col, zeros);
        }
        return;
    }
    const uint32_t wave = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(wave_id())), lane = lane_id(), words = (n + kWave - 1) / kWave;
    const uint32_t column_block = blockIdx.x % a.column_blocks, mine = blockIdx.x / a.column_blocks * kSortWaves + wave;
    const LaneColumns<V> columns(lane, column_block * (kWave * V), a.width);
    const T* dy = static_cast<const T*>(a.dy) + columns.at;
    if (a.n_distinct && blockIdx.x == 0 && threadIdx.x == 0) {
        int64_t u = 0;
        for (uint32_t w = 0; w < words; ++w) u += __popcll(s.heads[w]);
        *a.n_distinct = u;
    }
    float acc[V];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0;
    const auto to_row = [&](uint32_t row) {
        if (columns.any) store_scaled<TYPE, V>(a.out, row * a.out_ld + columns.at, acc, a.scale);
    };
    if (lane == 0) s_long[wave] = kNone;
    if (mine < n && (s.heads[mine / kWave] >> (mine % kWave) & 1)) {
        const uint32_t id = s.key[mine];
        uint32_t found = 0, row = id;
        if (a.n_distinct) row = 0;
        for (uint32_t w = 0; w < words; ++w) {
            const uint32_t key = s.key[w * kWave + lane];
            const uint64_t same = __ballot(key == id);
            if (a.n_distinct) row += __popcll(__ballot(key < id) & s.heads[w]);
            const uint32_t at = found + rank_in_mask(same);
            if (key == id && at < kLongRun) s_position[wave][at] = w * kWave + lane;
            found += __popcll(same);
        }
        __builtin_amdgcn_wave_barrier();
        if (a.n_distinct && column_block == 0 && lane == 0) a.row_id[row] = static_cast<int32_t>(id);
        if (found > kLongRun) {
            if (lane == 0) s_long[wave] = id, s_row[wave] = row;
        } else {
            for (uint32_t q = 0; q < found; q += kRowsAhead) {
                Few<Y, V> rows[kRowsAhead];
#pragma unroll
                for (int k = 0; k < kRowsAhead; ++k) rows[k].load(dy + s_position[wave][min(q + k, found - 1)] * a.dy_ld);
#pragma unroll
                for (int k = 0; k < kRowsAhead; ++k) rows[k].add(q + k < found, acc);
            }
            to_row(row);
        }
    }
    __syncthreads();
    for (int run = 0; run < kSortWaves; ++run) {
        const uint32_t id = s_long[run];
        if (id == kNone) continue;
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = 0;
        for (uint32_t w = wave; w < words; w += kSortWaves) {
            uint64_t left = __ballot(s.key[w * kWave + lane] == id);
            while (left) {
                Few<Y, V> rows[kRowsAhead];
                int in = 0;
                uint32_t at = 0;
#pragma unroll
                for (int k = 0; k < kRowsAhead; ++k) {
                    if (left) at = w * kWave + static_cast<uint32_t>(__ffsll(static_cast<long long>(left)) - 1), ++in;
                    left &= left - 1;
                    rows[k].load(dy + at * a.dy_ld);
                }
#pragma unroll
                for (int k = 0; k < kRowsAhead; ++k) rows[k].add(k < in, acc);
            }
        }
#pragma unroll
        for (int e = 0; e < V; ++e) s_part[wave][e][lane] = acc[e];
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                acc[e] = 0;
#pragma unroll
                for (int w = 0; w < kSortWaves; ++w) acc[e] += s_part[w][e][lane];
            }
            to_row(s_row[run]);
        }
        __syncthreads();
    }
}

// ---- sums of the sorted list

// A chunk to a wave: what it does next is the same for all lanes, so that the list, the places of rows and the branches are the scalar unit's, and
// an entry costs a lane a load and V additions.  281 600 rows of 128 in single precision: 50 us, in which 144 MB of rows that lie
// anywhere are read and 98 MB written (4.8 TB/s); 16 or 32 lanes to
// a chunk took 65.  100 003 rows of 256 in bfloat16, 349 IDs: 11.6 us.
constexpr int kAhead = 16;
template <int TYPE, int Y, int V>
__global__ __launch_bounds__(kBlock) void sum_kernel(GradArgs a, const Entry* list, uint32_t n_tasks) {
    typedef typename ElementOf<Y>::type T;
    const uint32_t n = static_cast<uint32_t>(a.rows.get()), n_chunks = (n + a.chunk - 1) / a.chunk, lane = lane_id();
    const uint32_t wave = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(wave_id()));
    for (uint32_t task = blockIdx.x * kWavesPerBlock + wave; task < n_tasks; task += gridDim.x * kWavesPerBlock) {
        const uint32_t column_block = task % a.column_blocks, chunk = task / a.column_blocks;
        if (chunk >= n_chunks) {
            if (a.n_distinct && n_chunks == 0 && task == 0 && lane == 0) *a.n_distinct = 0;
            continue;
        }
        const LaneColumns<V> columns(lane, column_block * (kWave * V), a.width);
        const T* dy = static_cast<const T*>(a.dy) + columns.at;
        const uint32_t begin = chunk * a.chunk, end = min(begin + a.chunk, n);

        // the row of drow of the first run that begins here
        uint32_t rank = 0;
        if (a.n_distinct) {
            for (uint32_t g = lane; g < begin / a.head_span; g += kWave) rank += a.group_heads[g];
            rank = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(wave_sum(rank)))) + a.chunk_rank[chunk];
        }
        float acc[V];
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = 0;
        bool any = false, headless = true;          // something in acc; no run has begun here so far
        uint32_t row = 0;                           // of the run in acc
        const auto to_part = [&](int which) {
            if (columns.any) store_scaled<kF32, V>(a.part, (static_cast<int64_t>(chunk) * 2 + which) * a.width + columns.at, acc, 1.0f);
        };
        const auto to_row = [&] {
            if (columns.any) store_scaled<TYPE, V>(a.out, row * a.out_ld + columns.at, acc, a.scale);
        };
        for (uint32_t from = begin; from < end; from += kWave) {
            const uint32_t at = from + lane;
            const Entry mine = list[min(at, end - 1)], before = list[at > 0 ? min(at, end) - 1 : 0];
            const bool there = at < end && id_of(mine) < a.n_table, head = there && (at == 0 || id_of(before) != id_of(mine));
            const uint64_t heads = __ballot(head);
            if (head && a.n_distinct && column_block == 0) a.row_id[rank + rank_in_mask(heads)] = static_cast<int32_t>(id_of(mine));
            const uint32_t in = static_cast<uint32_t>(__popcll(__ballot(there)));        // (those that have a row come first)
            for (uint32_t q = 0; q < in; q += kAhead) {
                Few<Y, V> rows[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) rows[k].load_once(dy + lane_value(position_of(mine), min(q + k, in - 1)) * a.dy_ld);
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    if (heads >> (q + k) & 1) {
                        if (any && headless) to_part(0);
                        else if (any) to_row();
                        headless = false;
                        row = a.n_distinct ? rank : lane_value(id_of(mine), q + k);
                        ++rank;
#pragma unroll
                        for (int e = 0; e < V; ++e) acc[e] = 0;
                    }
                    any = true;
                    rows[k].add(q + k < in, acc);
                }
            }
        }
        const uint32_t last = id_of(list[end - 1]);
        const bool goes_on = last < a.n_table && end < n && id_of(list[end]) == last;
        if (any && headless) to_part(0);
        else if (any && goes_on) to_part(1);
        else if (any) to_row();
        if (column_block == 0 && lane == 0) {
            a.info[chunk] = !any || !goes_on ? kNothing : headless ? kThrough : static_cast<int32_t>(row);
            if (a.n_distinct && chunk + 1 == n_chunks) *a.n_distinct = rank;
        }
    }
}

// Adds the parts of a run that begins in a chunk and goes on.  A wave has 16 V columns of a chunk, 16 lanes to a part and four parts at a time; a run
// that goes through the next 63 chunks is left to all waves of the workgroup, which have neighbouring chunks and so at most one of these among them (four, with
// the same chunk's blocks of columns beside one another, took twice as long).  4.8 us and 8 in the two cases above, a chain of dependent loads; with a
// list of the runs to be added, taken by a counter, it took 18.
constexpr int kMergeLanes = 16, kMergeSubs = kWave / kMergeLanes, kMergeWaves = 8, kMergeBlock = kMergeWaves * kWave;
template <int TYPE, int V>
__global__ __launch_bounds__(kMergeBlock) void merge_kernel(GradArgs a, uint32_t all_chunks, uint32_t n_tasks) {
    __shared__ float s[kMergeWaves][V][kMergeLanes];
    __shared__ uint32_t s_long[kMergeWaves], s_last;
    const uint32_t n = static_cast<uint32_t>(a.rows.get()), n_chunks = (n + a.chunk - 1) / a.chunk;
    const uint32_t wave = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(wave_id())), lane = lane_id() % kMergeLanes, sub = lane_id() / kMergeLanes;
    float acc[V];
    // the part of the chunk where the run begins, if there is one to be had for this lane, and those of first, first + step, ... up to `last`
    const auto add_parts = [&](uint32_t chunk, bool begins, uint32_t first, uint32_t last, uint32_t step, uint32_t col) {
        Few<kF32, V> begin;
        begin.load(a.part + (static_cast<int64_t>(chunk) * 2 + 1) * a.width + col);
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = begins ? begin.v[e] : 0.0f;
        for (uint32_t c = first; c <= last; c += step * kRowsAhead) {
            Few<kF32, V> parts[kRowsAhead];
#pragma unroll
            for (int k = 0; k < kRowsAhead; ++k) parts[k].load(a.part + static_cast<int64_t>(min(c + k * step, last)) * 2 * a.width + col);
#pragma unroll
            for (int k = 0; k < kRowsAhead; ++k) parts[k].add(c + k * step <= last, acc);
        }
        // over the lanes that share a column
#pragma unroll
        for (int e = 0; e < V; ++e) {
            acc[e] += __shfl_xor(acc[e], 16, kWave);
            acc[e] += __shfl_xor(acc[e], 32, kWave);
        }
    };
    const auto columns_of = [&](uint32_t task) { return LaneColumns<V>(lane, task / all_chunks * (kMergeLanes * V), a.width); };
    for (uint32_t base = blockIdx.x * kMergeWaves; base < n_tasks; base += gridDim.x * kMergeWaves) {
        const uint32_t task = base + wave, chunk = task % all_chunks;
        const uint32_t c = chunk + lane_id();
        const int32_t info = task < n_tasks && c < n_chunks ? a.info[c] : kNothing, row = __builtin_amdgcn_readfirstlane(info);
        const uint64_t ends = ~__ballot(info == kThrough) & ~uint64_t{1};        // chunks that a run from the first one does not go through
        if (lane_id() == 0) s_long[wave] = row >= 0 && ends == 0 ? task : kNone;
        if (row >= 0 && ends != 0) {
            const LaneColumns<V> columns = columns_of(task);
            add_parts(chunk, sub == 0, chunk + 1 + sub, chunk + static_cast<uint32_t>(__ffsll(static_cast<long long>(ends)) - 1), kMergeSubs, columns.at);
            if (sub == 0 && columns.any) store_scaled<TYPE, V>(a.out, row * a.out_ld + columns.at, acc, a.scale);
        }
        __syncthreads();
        for (int w = 0; w < kMergeWaves; ++w) {
            const uint32_t task = s_long[w], chunk = task % all_chunks;
            if (task == kNone) continue;
            if (threadIdx.x == 0) s_last = n_chunks;
            __syncthreads();
            for (uint32_t from = chunk + kWave; from < n_chunks; from += kMergeBlock) {       // the first chunk that the run does not go through
                const uint32_t c = from + threadIdx.x;
                if (c < n_chunks && a.info[c] != kThrough) atomicMin(&s_last, c);
                __syncthreads();
                const bool found = s_last < n_chunks;
                __syncthreads();
                if (found) break;
            }
            const LaneColumns<V> columns = columns_of(task);
            add_parts(chunk, wave == 0 && sub == 0, chunk + 1 + wave * kMergeSubs + sub, min(s_last, n_chunks - 1), kMergeSubs * kMergeWaves, columns.at);
            if (sub == 0)
#pragma unroll
                for (int e = 0; e < V; ++e) s[wave][e][lane] = acc[e];
            __syncthreads();
            if (wave == 0 && sub == 0 && columns.any) {
#pragma unroll
                for (int e = 0; e < V; ++e)
#pragma unroll
                    for (int k = 1; k < kMergeWaves; ++k) acc[e] += s[k][e][lane];
                store_scaled<TYPE, V>(a.out, a.info[chunk] * a.out_ld + columns.at, acc, a.scale);
            }
            __syncthreads();
        }
        __syncthreads();
    }
}

// ---- launches

uint32_t ceil_div(int64_t a, int64_t b) { return static_cast<uint32_t>((a + b - 1) / b); }

// How a list is cut, and how much scratch it takes.
struct GradPlan {
    GradArgs a;
    uint32_t n_chunks, head_groups;
    int64_t few_blocks;                             // workgroups of few_kernel that sum
    int per_lane;                                   // neighbouring columns of a row
    size_t bytes;
    GradPlan(const EmbeddingGradJob& job, char* scratch) {
        const int64_t n = job.rows.host;
        a = GradArgs{};
        a.rows = job.rows;
        a.width = job.width, a.scale = job.scale, a.n_table = static_cast<uint32_t>(job.n_table);
        a.ids = job.ids, a.dy = job.dy, a.dy_ld = job.dy_ld, a.out = job.out, a.out_ld = job.out_ld;
        a.row_id = job.row_id, a.n_distinct = job.n_distinct, a.err = job.err;
        per_lane = 1;
        while (per_lane * type_bytes(job.y_type) < 16 && per_lane * kWave < job.width) per_lane *= 2;
        const int64_t tiles = (n + kSortTile - 1) / kSortTile;
        a.group_tiles = std::max<uint32_t>(1, ceil_div(tiles, kMostGroups));
        a.n_groups = ceil_div(tiles, a.group_tiles);
        a.chunk = 32;
        while (n > static_cast<int64_t>(a.chunk) * kMostChunks) a.chunk *= 2;
        a.head_span = std::max<uint32_t>(1, ceil_div(n, int64_t{kHeadGroups} * kSortBlock * 8)) * kSortBlock * 8;
        a.column_blocks = ceil_div(job.width, per_lane * kWave);
        a.fill_blocks = job.n_distinct ? 0 : static_cast<uint32_t>(std::min<int64_t>(kFillBlocks, ceil_div(job.n_table * ((job.width + 7) / 8), kSortBlock)));
        few_blocks = std::max<int64_t>(ceil_div(n, kSortWaves), a.n_distinct ? 1 : 0) * a.column_blocks;
        a.few = n == 0 || (n <= kFew && few_blocks * (n + 1000) <= kFewWork);
        a.fill_first = a.few && a.fill_blocks * (n + 1000) > kFillWork + job.n_table * a.width * type_bytes(job.table_type) / kFillHidden;
        n_chunks = ceil_div(n, a.chunk);
        head_groups = ceil_div(n, a.head_span);
        bytes = 0;
        const auto take = [&](auto** to, size_t count) {
            *to = reinterpret_cast<std::remove_reference_t<decltype(**to)>*>(scratch + bytes);
            bytes = (bytes + count * sizeof(**to) + 255) / 256 * 256;
        };
        if (a.few) return;
        take(&a.list[0], n);
        take(&a.list[1], n);
        take(&a.counts, static_cast<size_t>(a.n_groups) * kMostBins);
        take(&a.chunk_rank, n_chunks);
        take(&a.group_heads, head_groups);
        take(&a.info, n_chunks);
        take(&a.part, static_cast<size_t>(n_chunks) * 2 * a.width);
    }
};

template <int TYPE, int Y, int V>
void launch_sums(hipStream_t stream, const GradPlan& plan, const Entry* list) {
    const GradArgs& a = plan.a;
    if (a.few) {
        const uint32_t sum_blocks = static_cast<uint32_t>(plan.few_blocks);
        if (a.fill_first) hipLaunchKernelGGL(clear_kernel<TYPE>, dim3(a.fill_blocks), dim3(kSortBlock), 0, stream, a);
        const uint32_t blocks = sum_blocks + (a.fill_first ? 0 : a.fill_blocks);
        if (blocks > 0) hipLaunchKernelGGL((few_kernel<TYPE, Y, V>), dim3(blocks), dim3(kSortBlock), 0, stream, a, sum_blocks);
        return;
    }
    const uint32_t tasks = plan.n_chunks * a.column_blocks;      // (fewer than 2^31: kMostChunks)
    hipLaunchKernelGGL((sum_kernel<TYPE, Y, V>), dim3(std::min<uint32_t>(ceil_div(tasks, kWavesPerBlock), kMostBlocks)), dim3(kBlock), 0, stream, a, list, tasks);
}
template <int TYPE, int V>
void launch_merge(hipStream_t stream, const GradPlan& plan) {
    const uint32_t columns = ceil_div(plan.a.width, V * kMergeLanes), tasks = plan.n_chunks * columns;
    hipLaunchKernelGGL((merge_kernel<TYPE, V>), dim3(std::min<uint32_t>(ceil_div(tasks, kMergeWaves), kMostBlocks)), dim3(kMergeBlock), 0, stream, plan.a, plan.n_chunks, tasks);
}
template <int TYPE, int Y>
hipError_t run_grad(hipStream_t stream, const GradPlan& plan) {
    const GradArgs& a = plan.a;
    const Entry* list = nullptr;
    if (!a.few) {
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
    if (plan.per_lane == 1) launch_sums<TYPE, Y, 1>(stream, plan, list);
    else if (plan.per_lane == 2) launch_sums<TYPE, Y, 2>(stream, plan, list);
    else if (plan.per_lane == 4) launch_sums<TYPE, Y, 4>(stream, plan, list);
    else if constexpr (Y != kF32) launch_sums<TYPE, Y, 8>(stream, plan, list);
    if (!a.few) {
        if (a.width >= 4) launch_merge<TYPE, 4>(stream, plan);
        else launch_merge<TYPE, 1>(stream, plan);
    }
    return hipGetLastError();
}

template <int TABLE, int Y, int ROWS>
void run_lookup(hipStream_t stream, const EmbeddingJob& job) {
    const int64_t items = job.rows.host * ((job.width + 7) / 8);
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>((items + kBlock * kItems - 1) / (kBlock * kItems), kMostBlocks)));
    hipLaunchKernelGGL((embedding_kernel<TABLE, Y, ROWS>), grid, dim3(kBlock), 0, stream, job);
}
template <int TABLE, int Y>
void run_lookup(hipStream_t stream, const EmbeddingJob& job) {
    const int64_t met = std::min(job.rows.host, job.n_table);            // rows of the table, at most
    const Rows rows = rows_of(job.width, job.width * (met * type_bytes(TABLE) + job.rows.host * type_bytes(Y) * (job.add ? 2 : 1)));
    if (rows == kWholeRows) run_lookup<TABLE, Y, kWholeRows>(stream, job);
    else if (rows == kStreamedRows) run_lookup<TABLE, Y, kStreamedRows>(stream, job);
    else if (rows == kRowsWithRest) run_lookup<TABLE, Y, kRowsWithRest>(stream, job);
    else run_lookup<TABLE, Y, kShortRows>(stream, job);
}

}  // namespace

hipError_t launch_embedding(hipStream_t stream, const EmbeddingJob& job) {
    if (job.rows.host < 1) return hipSuccess;
    if (job.table_type == kF16) run_lookup<kF16, kF16>(stream, job);
    else if (job.table_type == kBF16) run_lookup<kBF16, kBF16>(stream, job);
    else if (job.y_type == kF16) run_lookup<kF32, kF16>(stream, job);
    else if (job.y_type == kBF16) run_lookup<kF32, kBF16>(stream, job);
    else run_lookup<kF32, kF32>(stream, job);
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
