// Matrix products of a layer: y = act(x w^T + bias) + residual, and their gradients.
//
// All three products are D[M][N] = sum over k of A[m][k] B[n][k], in tiles that a workgroup stages through LDS:
//   forward   A = x  (rows of k),           B = w (rows of k)
//   dx        A = dz (rows of k = n_out),   B = w (k-strided: [k][n])
//   dw        A = dz (k-strided, k = rows), B = x (k-strided)
// A stage of an operand is 128 bytes of k for every row (64 elements of 16 bits, 32 of 32 bits, 128 of 8 bits), or
// as many k-strided rows.  Chunks of 16 bytes lie in LDS where a swizzle puts them, so that the 16 lanes that read a
// column of a tile hit different banks; k-strided tiles of 16-bit elements are transposed by the read (ds_read_b64_tr_b16).
// Elements of 16 bits go to the matrix instructions as they are, e4m3 after widening to half precision, single precision in
// three parts of bfloat16, gradients that 16 bits cannot hold in two.  Sums are held in 32 bits (MFMA accumulators); the epilogue works on 32-bit sums and rounds once.
//
// Measured: 100 000 x 2048 x 512 in half precision with bias, ReLU and z kept 256-267 us (0.8 PFLOP/s; matrix units busy 0.41 of the
// time); 50 003 x 1024 x 1024 in e4m3 with scales, SiLU and residual 131-138 us (0.78 PFLOP/s; 0.33); the gradient of 26 624 x 512 x 256
// with GELU in bfloat16 64-66 us (0.23), of 11 264 x 256 x 256 with ReLU in single precision 45 us (0.17); one row 256 x 256 4 us of kernel.
// What bounds the large ones is the step: a stage's loads, LDS reads and products, with two workgroups to a CU to fill each
// other's waits; the small ones a launch and one trip to memory.
#include "layer.hpp"
#include "layer_dev.hpp"

#include <algorithm>

namespace helios {

namespace {

constexpr uint32_t kMostBlocks = 1u << 22;        // of a launch
constexpr int kStageBytes = 128;                  // of k, per row of a tile

// What one 16-byte chunk of A and one of B contribute to a tile of 16 x 16: their elements as the matrix instructions take
// them, and the instructions (swapped, so that a lane holds one row of A and four neighbouring columns).
// e4m3 goes to 16 bits first, which is exact: the matrix instructions for 8 bits lose the sum's lower bits (measured: off by
// up to 2^-13 of the sum of the products' magnitudes, 2^-22 by way of 16 bits).
template <int TYPE> struct Mma;
template <> struct Mma<kF16> {
    typedef f16x8 Part;
    static __device__ __forceinline__ Part part(i32x4 v) { return __builtin_bit_cast(f16x8, v); }
    static __device__ __forceinline__ f32x4 run(const Part& a, const Part& b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(b, a, c, 0, 0, 0); }
};
template <> struct Mma<kBF16> {
    typedef bf16x8 Part;
    static __device__ __forceinline__ Part part(i32x4 v) { return __builtin_bit_cast(bf16x8, v); }
    static __device__ __forceinline__ f32x4 run(const Part& a, const Part& b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, a, c, 0, 0, 0); }
};
template <> struct Mma<kF32> {
    typedef f32x4 Part;
    static __device__ __forceinline__ Part part(i32x4 v) { return __builtin_bit_cast(f32x4, v); }
    static __device__ __forceinline__ f32x4 run(const Part& a, const Part& b, f32x4 c) {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(b[j], a[j], c, 0, 0, 0);
        return c;
    }
};
template <> struct Mma<kE4M3> {
    struct Part {
        f16x8 half[2];
    };
    static __device__ __forceinline__ Part part(i32x4 v) {
        typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
        Part p;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const f16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v[k], 1.0f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v[k], 1.0f, true);
            const int at = k % 2 * 4;
            p.half[k / 2][at] = lo.x, p.half[k / 2][at + 1] = lo.y, p.half[k / 2][at + 2] = hi.x, p.half[k / 2][at + 3] = hi.y;
        }
        return p;
    }
    static __device__ __forceinline__ f32x4 run(const Part& a, const Part& b, f32x4 c) {
#pragma unroll
        for (int k = 0; k < 2; ++k) c = __builtin_amdgcn_mfma_f32_16x16x32_f16(b.half[k], a.half[k], c, 0, 0, 0);
        return c;
    }
};

__device__ const int32_t kZeroChunk[4] __attribute__((aligned(16))) = {0, 0, 0, 0};

struct Operand {
    const char* data;
    int64_t ld;                                   // bytes from one row to the next
    int64_t rows, cols;                           // of the array in memory, in elements; what lies outside counts as zeros
};

// One operand's share of a stage: WIDTH rows of ROW bytes of k, or (STRIDED) as many k-strided rows of WIDTH columns.
// (SWIZZLED: the order in which threads take the chunks is that of LDS; else that of memory.)
template <int TYPE, int WIDTH, int ROW, bool STRIDED, int THREADS, bool SWIZZLED = true>
struct Stage {
    static constexpr int kBytes = type_bytes(TYPE);
    static constexpr int kPer = 16 / kBytes;      // elements of a chunk
    static constexpr int kK = ROW / kBytes;
    static constexpr int kChunks = WIDTH * (ROW / 16);
    static constexpr int kLoads = kChunks / THREADS;
    static constexpr int kRowChunks = STRIDED ? WIDTH * kBytes / 16 : ROW / 16;
    static_assert(kChunks % THREADS == 0, "every thread stages as many chunks");

    static __device__ __forceinline__ uint32_t swizzle(uint32_t row) {
        if (!STRIDED) return ROW == 128 ? (row >> 1) & 7 : (row >> 2) & 3;
        if (kBytes == 4) return ((row >> 2) & 3) << 2;
        return ((row & 3) | (((row >> 3) & 1) << 2)) % (kRowChunks / 2) << 1;
    }
    // Where the chunks that a thread stages begin, for the tile whose first row (k-strided: column) is `first`.  Chunks of rows or columns
    // that do not exist are taken from the last that does: whatever they hold stays in rows and columns that are not written.
    // Chunks of k that do not exist are zeros.
    struct Source {
        const char* at[kLoads];
        int valid[STRIDED ? kLoads : 1];          // elements of the chunk that exist (rows of any width)
    };
    static __device__ __forceinline__ uint32_t row_of(int l) { return (threadIdx.x + l * THREADS) / kRowChunks; }
    static __device__ __forceinline__ uint32_t chunk_of(int l) { return ((threadIdx.x + l * THREADS) % kRowChunks) ^ (SWIZZLED ? swizzle(row_of(l)) : 0u); }
    static __device__ __forceinline__ Source source(const Operand& o, int64_t first) {
        Source s;
#pragma unroll
        for (int l = 0; l < kLoads; ++l) {
            const uint32_t row = row_of(l), chunk = chunk_of(l);
            if (STRIDED) {
                const int64_t c = first + chunk * kPer, last = (o.cols - 1) / kPer * kPer, at = c < last ? c : last;
                s.at[l] = o.data + row * o.ld + at * kBytes;
                s.valid[l] = o.cols - at < kPer ? static_cast<int>(o.cols - at) : kPer;
            } else {
                const int64_t r = first + row, last = o.rows - 1;
                s.at[l] = o.data + (r < last ? r : last) * o.ld + chunk * 16;
            }
        }
        return s;
    }
    // The stage whose first k is k0, into registers: rows of any width and alignment (WHOLE: of whole chunks at 16-byte addresses).
    template <bool WHOLE>
    static __device__ __forceinline__ void load(const Operand& o, const Source& s, int64_t k0, i32x4 (&regs)[kLoads]) {
        const int64_t step = STRIDED ? k0 * o.ld : k0 * kBytes, left = (STRIDED ? o.rows : o.cols) - k0;
#pragma unroll
        for (int l = 0; l < kLoads; ++l) {
            const char* at = s.at[l] + step;
            const int64_t there = left - (STRIDED ? row_of(l) : chunk_of(l) * kPer);       // of k
            if (WHOLE) {
                if (left < kK && there <= 0) at = reinterpret_cast<const char*>(&kZeroChunk);
                regs[l] = *reinterpret_cast<const i32x4*>(at);
            } else if (STRIDED) {
                regs[l] = i32x4{0, 0, 0, 0};
                if (left >= kK || there > 0) regs[l] = load_16_of<kBytes>(at, s.valid[l]);
            } else {
                if (left >= kK) regs[l] = load_16(at);
                else regs[l] = load_16_of<kBytes>(at, there);
            }
        }
    }
    // The same straight into LDS, without a trip through registers, for rows of whole chunks at 16-byte addresses.
    static __device__ __forceinline__ void load_lds(const Operand& o, const Source& s, int64_t k0, char* lds) {
        const int64_t step = STRIDED ? k0 * o.ld : k0 * kBytes, left = (STRIDED ? o.rows : o.cols) - k0;
        const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
#pragma unroll
        for (int l = 0; l < kLoads; ++l) {
            const char* p = s.at[l] + step;
            if (left < kK && static_cast<int64_t>(STRIDED ? row_of(l) : chunk_of(l) * kPer) >= left) p = reinterpret_cast<const char*>(&kZeroChunk);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p,
                                             (__attribute__((address_space(3))) void*)(lds + (wave * kWave + l * THREADS) * 16), 16, 0, 0);
        }
    }
    static __device__ __forceinline__ void put(char* lds, const i32x4 (&regs)[kLoads]) {
#pragma unroll
        for (int l = 0; l < kLoads; ++l) *reinterpret_cast<i32x4*>(lds + (threadIdx.x + l * THREADS) * 16) = regs[l];
    }
    // A lane's chunk of the 16 rows (or columns) from `at` on: lane r of group g holds row at + r, and of k the 16 bytes at
    // 16 (g + 4 half).  k-strided 32-bit elements come one by one, 16-bit ones as two transposed reads.
    static __device__ __forceinline__ i32x4 fragment(const char* lds, int at, int half) {
        const uint32_t lane = threadIdx.x & (kWave - 1), r = lane & 15, g = lane >> 4;
        if (!STRIDED) {
            const uint32_t row = at + r;
            return *reinterpret_cast<const i32x4*>(lds + row * ROW + (((g + 4 * half) ^ swizzle(row)) << 4));
        }
        if (kBytes == 4) {
            i32x4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t k = 16 * half + 4 * g + j;
                v[j] = *reinterpret_cast<const int32_t*>(lds + k * (WIDTH * 4) + ((((at + r) >> 2) ^ swizzle(k)) << 4) + (r & 3) * 4);
            }
            return v;
        }
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        typedef int32_t i32x2 __attribute__((ext_vector_type(2)));
        i32x2 part[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t k = 32 * half + 8 * g + 4 * j + (r >> 2), column = at + 4 * (r & 3);
            const char* p = lds + k * (WIDTH * 2) + (((column >> 3) ^ swizzle(k)) << 4) + ((column >> 2) & 1) * 8;
            part[j] = __builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p)));
        }
        return i32x4{part[0].x, part[0].y, part[1].x, part[1].y};
    }
};

// Single precision goes through the 16-bit instructions, which are sixteen times as quick: a value is split into three
// of bfloat16, x = h + m + l exactly, each the nearest to what is left (so that they have either sign, and what is left out no bias), and
// of the nine products the six that matter are added, the smallest first: l h', h l', m m',
// m h', h m', h h' (those left out are at most 2^-23 of the product).  Six instructions stand for eight of single precision that take twice as
// long each.  A stage of 32 elements of k lies in LDS as three planes of 64-byte rows.  An infinity would meet zeros in this and
// leave NaN, so the loads watch for first parts that are not finite, and a tile that has met one is done again by the instructions of
// single precision.  Values below 2^-110 lose their last bits.  Error in the norm for normal values, sums of 1, 2, 8 and 16 products: 3.5e-8, 3.3e-8,
// 3.1e-8 and 3.4e-8; added up one by one in 32 bits 2.5e-8, 3.7e-8, 6.1e-8 and 8.1e-8; with parts cut off, not rounded, 6.3e-8 to 6.9e-8.
struct SplitPart {
    bf16x8 h, m, l;
};
template <int WIDTH, bool STRIDED, int THREADS>
struct SplitStage {
    typedef Stage<kF32, WIDTH, 128, STRIDED, THREADS, false> Whole;                  // (loads and their order; its stage is not used)
    typedef Stage<kBF16, WIDTH, 64, STRIDED, THREADS> Plane;
    static constexpr int kLoads = Whole::kLoads, kPlane = WIDTH * 64;
    // spoilt: 0, until a first part is not finite
    static __device__ __forceinline__ void put(char* lds, const i32x4 (&regs)[kLoads], float* spoilt) {
        typedef int32_t i32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int l = 0; l < kLoads; ++l) {
            const uint32_t row = Whole::row_of(l), chunk = Whole::chunk_of(l);
            typedef float f32x2 __attribute__((ext_vector_type(2)));
            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
            uint32_t part[3][2];                  // [h, m, l][two neighbours]
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int32_t bits[2] = {regs[l][2 * e], regs[l][2 * e + 1]};
                f32x2 x = {__builtin_bit_cast(float, bits[0]), __builtin_bit_cast(float, bits[1])};
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    part[k][e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
                    const float a = __builtin_bit_cast(float, part[k][e] << 16), b = __builtin_bit_cast(float, part[k][e] & 0xffff0000u);
                    if (k == 0) *spoilt = __builtin_fmaf(b, 0.0f, __builtin_fmaf(a, 0.0f, *spoilt));
                    x = f32x2{x.x - a, x.y - b};
                }
            }
            const uint32_t to = STRIDED ? row * (WIDTH * 2) + (((chunk >> 1) ^ Plane::swizzle(row)) << 4) + (chunk & 1) * 8
                                        : row * 64 + (((chunk >> 1) ^ Plane::swizzle(row)) << 4) + (chunk & 1) * 8;
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                i32x2 v;
                v.x = static_cast<int32_t>(part[k][0]);
                v.y = static_cast<int32_t>(part[k][1]);
                *reinterpret_cast<i32x2*>(lds + k * kPlane + to) = v;
            }
        }
    }
    typedef SplitPart Part;
    static __device__ __forceinline__ Part fragment(const char* lds, int at) {
        return Part{__builtin_bit_cast(bf16x8, Plane::fragment(lds, at, 0)), __builtin_bit_cast(bf16x8, Plane::fragment(lds + kPlane, at, 0)),
                    __builtin_bit_cast(bf16x8, Plane::fragment(lds + 2 * kPlane, at, 0))};
    }
};
// (the six products one after the other for all tiles of a wave, so that an instruction seldom waits for the one before it)
template <int TM, int TN>
__device__ __forceinline__ void split_mma(const SplitPart (&a)[TM], const SplitPart (&b)[TN], f32x4 (&c)[TM][TN]) {
#pragma unroll
    for (int k = 0; k < 6; ++k)
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const bf16x8 x = k == 0 ? a[i].l : k == 2 || k == 3 ? a[i].m : a[i].h, y = k == 1 ? b[j].l : k == 2 || k == 4 ? b[j].m : b[j].h;
                c[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, x, c[i][j], 0, 0, 0);
            }
}

// The epilogues.  A thread has eight neighbouring columns, `valid` of them in the matrix, and goes through rows: at() takes what
// belongs to the columns, row() finishes and writes the sums of one row.  The type written and whether the activation needs an
// exponential are the kernel's: a round through a row is a chain that few waves have to bear, and with all types and activations
// in it, it is longer (98 304 x 512 sums of 64 products in half precision: 33 us; branches for every row 44, for every
// element 55).
template <int OUT_TYPE, bool SMOOTH>
struct ForwardOut {
    const float *x_scale, *w_scale;
    const void *bias, *residual;
    int64_t residual_ld;
    void* pre;
    int64_t pre_ld;
    void* y;
    int64_t y_ld;
    int act;
    struct Columns {
        int32_t col, valid;
        float scale[8], bias[8], least;
    };
    __device__ __forceinline__ Columns at(int32_t col, int valid, int) const {
        Columns c{col, valid, {1, 1, 1, 1, 1, 1, 1, 1}, {0, 0, 0, 0, 0, 0, 0, 0}, act == kActRelu ? 0.0f : -__builtin_inff()};
        if (w_scale) load_8_of<kF32>(w_scale, col, valid, c.scale);
        if (bias) load_8_of<OUT_TYPE>(bias, col, valid, c.bias);
        return c;
    }
    // what a row needs from memory, asked for before its sums are there
    struct Ahead {
        i32x4 residual[type_bytes(OUT_TYPE) / 2];
        float scale;
    };
    __device__ __forceinline__ Ahead ahead(const Columns& c, int64_t row) const {
        Ahead a{};
        if (residual) {
            constexpr int kBytes = type_bytes(OUT_TYPE), kPer = 16 / kBytes;
            const char* p = static_cast<const char*>(residual) + (row * residual_ld + c.col) * kBytes;
#pragma unroll
            for (int k = 0; k < 8 / kPer; ++k)
                if (c.valid > k * kPer) a.residual[k] = load_16_of<kBytes>(p + 16 * k, c.valid - k * kPer);
        }
        if (x_scale) a.scale = x_scale[row];
        return a;
    }
    __device__ __forceinline__ void row(const Columns& c, const Ahead& a, int64_t row, float (&v)[8]) const {
        if (x_scale)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = v[e] * a.scale * c.scale[e];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += c.bias[e];
        if (pre) store_8_of<OUT_TYPE>(pre, row * pre_ld + c.col, c.valid, v);
        if (SMOOTH) act_8<OUT_TYPE == kF32>(act, v);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = v[e] < c.least ? c.least : v[e];        // NaN stays
        if (residual) {
            float r[8];
            widen_8<OUT_TYPE>(a.residual, r);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += r[e];
        }
        store_8_of<OUT_TYPE>(y, row * y_ld + c.col, c.valid, v);
    }
};
template <int OUT_TYPE>
struct PlainOut {                                 // (slice: which part of k the sums are of)
    void* y;
    int64_t ld, slice_stride;
    bool in_32_bits;                              // the sums are parts of a sum
    struct Columns {
        int64_t at;
        int32_t valid;
    };
    __device__ __forceinline__ Columns at(int32_t col, int valid, int slice) const { return Columns{slice * slice_stride + col, valid}; }
    struct Ahead {};
    __device__ __forceinline__ Ahead ahead(const Columns&, int64_t) const { return Ahead{}; }
    __device__ __forceinline__ void row(const Columns& c, const Ahead&, int64_t row, float (&v)[8]) const {
        if (in_32_bits) store_8_of<kF32>(y, c.at + row * ld, c.valid, v);
        else store_8_of<OUT_TYPE>(y, c.at + row * ld, c.valid, v);
    }
};

template <class OUT>
struct ProductArgs {
    Operand a, b;
    int64_t a_low;                                // bytes from a value of A to its second part, where A comes in two (PARTS)
    int64_t m, k;                                 // the most; `rows` limits m, or k where that runs over rows
    int32_t n;
    Count rows;
    uint32_t tiles_n, members, tiles;             // (members: of a group)
    bool dealt;                                   // fewer groups than XCDs
    int slices;                                   // parts that k is cut into where it runs over rows, each with sums of its own
    OUT out;
};

// Workgroups go round the eight XCDs, each of which has an L2 of its own.  The tiles that share what is long (rows of A; where k runs
// over rows, a slice of it) are a group, and a group's tiles are neighbours on one XCD; in gradients
// fewer than eight groups are dealt out to all XCDs (gradient of 64 x 2048 x 1024 in bfloat16, all of dw one group: 22.6 us on one XCD, 11.5 on all; 200 x 2048 x 1024 31 and 12).
__device__ __forceinline__ void tile_of(uint32_t block, uint32_t members, bool dealt, uint32_t* group, uint32_t* member) {
    if (dealt) {
        *group = block / members;
        *member = block % members;
        return;
    }
    const uint32_t xcd = block % 8, at = block / 8;
    *group = at / members * 8 + xcd;
    *member = at % members;
}

// Waits until this wave's loads into LDS and its LDS reads are done, then for the other waves.
__device__ __forceinline__ void wait_and_meet() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Shape of a workgroup's tile: rows of A and B, and the waves that share it.
template <int M, int N, int WAVES_M, int WAVES_N>
struct Tile {
    static constexpr int kM = M, kN = N, kWavesM = WAVES_M, kWavesN = WAVES_N;
    static constexpr int kThreads = WAVES_M * WAVES_N * kWave;
};

// LDS of a product: the stages, and after them the sums on their way out.
template <int TYPE, class TILE>
struct ProductLds {
    static constexpr int kTm = TILE::kM / TILE::kWavesM / 16, kTn = TILE::kN / TILE::kWavesN / 16;      // 16 x 16 tiles of a wave
    static constexpr int kStage = (TILE::kM + TILE::kN) * (TYPE == kF32 ? 192 : kStageBytes);      // (single precision: three planes of 64 bytes)
    static constexpr int kOutLd = TILE::kN + 4;
    static constexpr int kOutBytes = TILE::kWavesM * 16 * kOutLd * 4;    // of the sums of one row of tiles of every wave
    static constexpr int kOutTiles = kTm * kOutBytes <= 2 * kStage + 4096 ? kTm : kTm % 2 == 0 && kTm / 2 * kOutBytes <= 2 * kStage ? kTm / 2 : 1;
    static constexpr int kBytes = 2 * kStage > kOutTiles * kOutBytes ? 2 * kStage : kOutTiles * kOutBytes;
    static_assert(kTm % kOutTiles == 0, "the epilogue takes as many rows of tiles at a time");
};

// Products with A in two parts (PARTS: a gradient that 16 bits of x's type cannot hold): a = hi + lo, both in bfloat16, so 16 bits of a value in
// the range of 32-bit ones; off by up to 2^-16 of it.  B is what it is in bfloat16, and for half precision two parts again, exact, cut when they
// are read from LDS; of the four products lo lo', below 2^-16, is left out.  Two (three) instructions in place of one.  Rounded to x's type, as
// the instructions would take it at once, a value is off by 2^-8 (2^-11), which shows in the results (26 624 x 512 x 256 with GELU in bfloat16:
// off by 0.0024 of their norm in place of 0.0017, which is their own rounding, in 47 us in place of 65), and in half precision
// gradients below 2^-25 are lost.
template <int TYPE> struct PartsMma;
template <> struct PartsMma<kBF16> {
    typedef bf16x8 Part;
    static __device__ __forceinline__ Part part(i32x4 v) { return __builtin_bit_cast(bf16x8, v); }
    static __device__ __forceinline__ f32x4 run(const bf16x8& hi, const bf16x8& lo, const Part& b, f32x4 c) {
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, lo, c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, hi, c, 0, 0, 0);
    }
};
template <> struct PartsMma<kF16> {
    struct Part {
        bf16x8 hi, lo;
    };
    static __device__ __forceinline__ Part part(i32x4 v) {
        const f16x8 x = __builtin_bit_cast(f16x8, v);
        Part p;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float f = static_cast<float>(x[e]);
            p.hi[e] = static_cast<__bf16>(f);
            p.lo[e] = static_cast<__bf16>(f - static_cast<float>(p.hi[e]));
        }
        return p;
    }
    static __device__ __forceinline__ f32x4 run(const bf16x8& hi, const bf16x8& lo, const Part& b, f32x4 c) {
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.hi, lo, c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.lo, hi, c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.hi, hi, c, 0, 0, 0);
    }
};
// The same by the instructions of single precision, for tiles with values that are not finite (an infinity would meet a lower part of
// zero, and leave NaN where there is none).
template <int TYPE>
__device__ __forceinline__ f32x4 parts_in_single(i32x4 hi, i32x4 lo, i32x4 b, f32x4 c) {
    const i32x4 h[1] = {hi}, l[1] = {lo}, o[1] = {b};
    float x[8], y[8], z[8];
    widen_8<kBF16>(h, x);
    widen_8<kBF16>(l, y);
    widen_8<TYPE>(o, z);
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(z[e], x[e] + y[e], c, 0, 0, 0);
    return c;
}

// The tiles block, block + blocks, ... of a product.
template <int TYPE, class TILE, bool A_STRIDED, bool B_STRIDED, bool DIRECT, bool PARTS, class OUT>
__device__ __forceinline__ void product(ProductArgs<OUT> p, uint32_t block, uint32_t blocks, char* lds) {
    constexpr int BM = TILE::kM, BN = TILE::kN, WAVES_M = TILE::kWavesM, WAVES_N = TILE::kWavesN, kThreads = TILE::kThreads;
    typedef ProductLds<TYPE, TILE> Lds;
    constexpr int kTm = Lds::kTm, kTn = Lds::kTn, kStage = Lds::kStage, kOutLd = Lds::kOutLd, kOutTiles = Lds::kOutTiles;
    constexpr bool kSplit = TYPE == kF32;
    typedef Stage<TYPE, BM, kStageBytes, A_STRIDED, kThreads> StageA;
    typedef Stage<TYPE, BN, kStageBytes, B_STRIDED, kThreads> StageB;

    const int64_t count = p.rows.get();
    const bool rows_are_k = A_STRIDED;
    const int64_t m_end = rows_are_k ? p.m : count, k_end = rows_are_k ? count : p.k;
    if (rows_are_k) p.a.rows = p.b.rows = count;
    else p.a.rows = count;
    constexpr int kK = PARTS ? StageA::kK / 2 : StageA::kK;              // of a step
    const int64_t steps_all = (k_end + kK - 1) / kK, per = (steps_all + p.slices - 1) / p.slices;

    const int wave = threadIdx.x / kWave, wave_m = wave / WAVES_N, wave_n = wave % WAVES_N;
    for (uint32_t tile = block; tile < p.tiles; tile += blocks) {      // (once round, but for the longest lists)
        uint32_t group, member;
        tile_of(tile, p.members, B_STRIDED && p.dealt, &group, &member);
        const int slice = rows_are_k ? static_cast<int>(group) : 0;
        const int64_t m0 = static_cast<int64_t>(rows_are_k ? member / p.tiles_n : group) * BM;
        const int32_t n0 = static_cast<int32_t>(rows_are_k ? member % p.tiles_n : member) * BN;
        if (m0 >= m_end || slice >= p.slices) continue;
        const int64_t step0 = slice * per, step1 = step0 + per < steps_all ? step0 + per : steps_all;
        f32x4 acc[kTm][kTn];
        const auto clear = [&] {
#pragma unroll
            for (int i = 0; i < kTm; ++i)
#pragma unroll
                for (int j = 0; j < kTn; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
        };
        clear();
        const auto multiply = [&](const char* stage) {
#pragma unroll
            for (int half = 0; half < kStageBytes / 64; ++half) {
                typename Mma<TYPE>::Part fa[kTm], fb[kTn];
#pragma unroll
                for (int i = 0; i < kTm; ++i) fa[i] = Mma<TYPE>::part(StageA::fragment(stage, (wave_m * kTm + i) * 16, half));
#pragma unroll
                for (int j = 0; j < kTn; ++j) fb[j] = Mma<TYPE>::part(StageB::fragment(stage + BM * kStageBytes, (wave_n * kTn + j) * 16, half));
#pragma unroll
                for (int i = 0; i < kTm; ++i)
#pragma unroll
                    for (int j = 0; j < kTn; ++j) acc[i][j] = Mma<TYPE>::run(fa[i], fb[j], acc[i][j]);
            }
        };
        // Two stages in turn and one barrier a step: it waits for the step's loads, and for every wave's reads of the stage before, which the
        // next loads go to.  (Three or four stages, or stages of 64 bytes, were no quicker: what the loads take is hidden by the other
        // workgroup of the CU.)
        const typename StageA::Source sa = StageA::source(p.a, m0);
        const typename StageB::Source sb = StageB::source(p.b, n0);
        if constexpr (PARTS) {
            // (a stage: 64 bytes of k of both parts of A and of B)
            typedef Stage<kBF16, BM, kStageBytes / 2, A_STRIDED, kThreads> PartA;
            typedef Stage<TYPE, BN, kStageBytes / 2, B_STRIDED, kThreads> PartB;
            constexpr int kLow = BM * kStageBytes / 2, kB = 2 * kLow;
            const Operand low{p.a.data + p.a_low, p.a.ld, p.a.rows, p.a.cols};
            const typename PartA::Source s_hi = PartA::source(p.a, m0), s_lo = PartA::source(low, m0);
            const typename PartB::Source s_b = PartB::source(p.b, n0);
            const auto through = [&](auto multiply_stage) {
                if constexpr (DIRECT) {
                    const auto load = [&](int64_t step) {
                        char* to = lds + ((step - step0) & 1) * kStage;
                        PartA::load_lds(p.a, s_hi, step * kK, to);
                        PartA::load_lds(low, s_lo, step * kK, to + kLow);
                        PartB::load_lds(p.b, s_b, step * kK, to + kB);
                    };
                    if (step0 < step1) load(step0);
                    for (int64_t step = step0; step < step1; ++step) {
                        wait_and_meet();
                        if (step + 1 < step1) load(step + 1);
                        multiply_stage(lds + ((step - step0) & 1) * kStage);
                    }
                } else {
                    i32x4 r_hi[PartA::kLoads], r_lo[PartA::kLoads], r_b[PartB::kLoads];
                    const auto load = [&](int64_t step) {
                        PartA::template load<false>(p.a, s_hi, step * kK, r_hi);
                        PartA::template load<false>(low, s_lo, step * kK, r_lo);
                        PartB::template load<false>(p.b, s_b, step * kK, r_b);
                    };
                    if (step0 < step1) load(step0);
                    for (int64_t step = step0; step < step1; ++step) {
                        char* stage = lds + ((step - step0) & 1) * kStage;
                        PartA::put(stage, r_hi);
                        PartA::put(stage + kLow, r_lo);
                        PartB::put(stage + kB, r_b);
                        __syncthreads();
                        if (step + 1 < step1) load(step + 1);
                        multiply_stage(stage);
                    }
                }
            };
            through([&](const char* stage) {
                bf16x8 hi[kTm], lo[kTm];
                typename PartsMma<TYPE>::Part b[kTn];
#pragma unroll
                for (int i = 0; i < kTm; ++i) {
                    hi[i] = __builtin_bit_cast(bf16x8, PartA::fragment(stage, (wave_m * kTm + i) * 16, 0));
                    lo[i] = __builtin_bit_cast(bf16x8, PartA::fragment(stage + kLow, (wave_m * kTm + i) * 16, 0));
                }
#pragma unroll
                for (int j = 0; j < kTn; ++j) b[j] = PartsMma<TYPE>::part(PartB::fragment(stage + kB, (wave_n * kTn + j) * 16, 0));
#pragma unroll
                for (int i = 0; i < kTm; ++i)
#pragma unroll
                    for (int j = 0; j < kTn; ++j) acc[i][j] = PartsMma<TYPE>::run(hi[i], lo[i], b[j], acc[i][j]);
            });
            // (a value that is not finite leaves a sum that is not)
            float spoilt = 0.0f;
#pragma unroll
            for (int i = 0; i < kTm; ++i)
#pragma unroll
                for (int j = 0; j < kTn; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) spoilt = __builtin_fmaf(acc[i][j][e], 0.0f, spoilt);
            if (__syncthreads_or(spoilt != 0.0f)) {
                clear();
                through([&](const char* stage) {
#pragma unroll
                    for (int j = 0; j < kTn; ++j) {
                        const i32x4 b = PartB::fragment(stage + kB, (wave_n * kTn + j) * 16, 0);
#pragma unroll
                        for (int i = 0; i < kTm; ++i)
                            acc[i][j] = parts_in_single<TYPE>(PartA::fragment(stage, (wave_m * kTm + i) * 16, 0),
                                                              PartA::fragment(stage + kLow, (wave_m * kTm + i) * 16, 0), b, acc[i][j]);
                    }
                });
            }
        } else if constexpr (DIRECT && !kSplit) {
            const auto load = [&](int64_t step) {
                char* to = lds + ((step - step0) & 1) * kStage;
                StageA::load_lds(p.a, sa, step * StageA::kK, to);
                StageB::load_lds(p.b, sb, step * StageA::kK, to + BM * kStageBytes);
            };
            if (step0 < step1) load(step0);
            for (int64_t step = step0; step < step1; ++step) {
                wait_and_meet();
                if (step + 1 < step1) load(step + 1);
                multiply(lds + ((step - step0) & 1) * kStage);
            }
        } else {
            const auto by_registers = [&] {
                i32x4 ra[StageA::kLoads], rb[StageB::kLoads];
                if (step0 < step1) {
                    StageA::template load<DIRECT>(p.a, sa, step0 * StageA::kK, ra);
                    StageB::template load<DIRECT>(p.b, sb, step0 * StageA::kK, rb);
                }
                for (int64_t step = step0; step < step1; ++step) {
                    char* stage = lds + ((step - step0) & 1) * kStage;
                    StageA::put(stage, ra);
                    StageB::put(stage + BM * kStageBytes, rb);
                    __syncthreads();
                    if (step + 1 < step1) {
                        StageA::template load<DIRECT>(p.a, sa, (step + 1) * StageA::kK, ra);
                        StageB::template load<DIRECT>(p.b, sb, (step + 1) * StageA::kK, rb);
                    }
                    multiply(stage);
                }
            };
            if constexpr (kSplit) {
                typedef SplitStage<BM, A_STRIDED, kThreads> SplitA;
                typedef SplitStage<BN, B_STRIDED, kThreads> SplitB;
                const typename SplitA::Whole::Source split_a = SplitA::Whole::source(p.a, m0);
                const typename SplitB::Whole::Source split_b = SplitB::Whole::source(p.b, n0);
                i32x4 ra[SplitA::kLoads], rb[SplitB::kLoads];
                float spoilt = 0.0f;
                const auto load = [&](int64_t step) {
                    SplitA::Whole::template load<DIRECT>(p.a, split_a, step * StageA::kK, ra);
                    SplitB::Whole::template load<DIRECT>(p.b, split_b, step * StageA::kK, rb);
                };
                const auto put = [&](int64_t step) {
                    char* stage = lds + ((step - step0) & 1) * kStage;
                    SplitA::put(stage, ra, &spoilt);
                    SplitB::put(stage + 3 * SplitA::kPlane, rb, &spoilt);
                };
                if (step0 < step1) load(step0), put(step0);
                if (step0 + 1 < step1) load(step0 + 1);
                for (int64_t step = step0; step < step1; ++step) {
                    const char* stage = lds + ((step - step0) & 1) * kStage;
                    __syncthreads();
                    SplitPart fa[kTm], fb[kTn];
#pragma unroll
                    for (int i = 0; i < kTm; ++i) fa[i] = SplitA::fragment(stage, (wave_m * kTm + i) * 16);
#pragma unroll
                    for (int j = 0; j < kTn; ++j) fb[j] = SplitB::fragment(stage + 3 * SplitA::kPlane, (wave_n * kTn + j) * 16);
                    split_mma(fa, fb, acc);
                    if (step + 1 < step1) put(step + 1);             // (beside the products: into the stage that was read a step ago)
                    if (step + 2 < step1) load(step + 2);
                }
                if (__syncthreads_or(spoilt != 0.0f)) {
                    clear();
                    by_registers();
                }
            } else by_registers();
        }
        __syncthreads();
        // The sums go through LDS, so that the epilogue reads and writes whole rows; kOutTiles of every wave's rows of tiles at a time.
        float* sums = reinterpret_cast<float*>(lds);
        const int r = threadIdx.x & 15, g = (threadIdx.x & (kWave - 1)) >> 4;
        static_assert(kThreads % (BN / 8) == 0, "a thread stays with its columns");
        const int out_col = threadIdx.x % (BN / 8) * 8;
        const typename OUT::Columns columns = p.out.at(n0 + out_col, p.n - n0 - out_col, slice);
        constexpr int kSlab = kOutTiles * 16, kStep = kThreads / (BN / 8), kOutRows = WAVES_M * kSlab / kStep;      // (a slab: the rows of one row of waves)
        static_assert(WAVES_M * kSlab % kStep == 0, "every thread has as many rows");
        const int valid = p.n - n0 - out_col;
#pragma unroll
        for (int i0 = 0; i0 < kTm; i0 += kOutTiles) {
            const auto row_at = [&](int q) {
                const int at = threadIdx.x / (BN / 8) + q * kStep;
                return m0 + at / kSlab * (kTm * 16) + i0 * 16 + at % kSlab;
            };
            typename OUT::Ahead ahead[kOutRows];
#pragma unroll
            for (int q = 0; q < kOutRows; ++q)
                if (valid > 0 && row_at(q) < m_end) ahead[q] = p.out.ahead(columns, row_at(q));
            if (i0 > 0) __syncthreads();
#pragma unroll
            for (int i = 0; i < kOutTiles; ++i)
#pragma unroll
                for (int j = 0; j < kTn; ++j)
                    *reinterpret_cast<f32x4*>(sums + ((wave_m * kOutTiles + i) * 16 + r) * kOutLd + (wave_n * kTn + j) * 16 + 4 * g) = acc[i0 + i][j];
            __syncthreads();
#pragma unroll
            for (int q = 0; q < kOutRows; ++q) {
                if (valid <= 0 || row_at(q) >= m_end) continue;
                const f32x4* from = reinterpret_cast<const f32x4*>(sums + (threadIdx.x / (BN / 8) + q * kStep) * kOutLd + out_col);
                const f32x4 lo = from[0], hi = from[1];
                float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
                p.out.row(columns, ahead[q], row_at(q), v);
            }
        }
        __syncthreads();
    }
}

// Waves of a SIMD that the registers are to leave room for: two workgroups to a CU where LDS has room for two (single precision: one).
template <int TYPE, class TILE>
constexpr int waves_that_fit() { return TYPE == kF32 ? 1 : TILE::kThreads / kWave / 2; }

template <int TYPE, class TILE, bool DIRECT, class OUT>
__global__ __launch_bounds__(TILE::kThreads, (waves_that_fit<TYPE, TILE>())) void forward_kernel(ProductArgs<OUT> p) {
    __shared__ __align__(16) char lds[ProductLds<TYPE, TILE>::kBytes];
    product<TYPE, TILE, false, false, DIRECT, false>(p, blockIdx.x, gridDim.x, lds);
}

// Both products of the gradient in one launch, each with workgroups of its own: dw's tiles come first, since each takes longest.
template <int TYPE, class TILE, bool DIRECT, bool PARTS>
__global__ __launch_bounds__(TILE::kThreads, (waves_that_fit<TYPE, TILE>())) void backward_kernel(ProductArgs<PlainOut<TYPE>> dw, uint32_t dw_blocks, ProductArgs<PlainOut<TYPE>> dx) {
    __shared__ __align__(16) char lds[ProductLds<TYPE, TILE>::kBytes];
    if (blockIdx.x < dw_blocks) product<TYPE, TILE, true, true, DIRECT, PARTS>(dw, blockIdx.x, dw_blocks, lds);
    else product<TYPE, TILE, false, true, DIRECT, PARTS>(dx, blockIdx.x - dw_blocks, gridDim.x - dw_blocks, lds);
}

// Few tiles: a workgroup has 16 rows of x and 16 of w, its waves share k between them and read both straight into the
// operands of the MFMA, and the eight sums of every element meet in LDS, so that one trip to memory is all that lies between launch and
// epilogue (1 x 256 x 256 in half precision 4.2 us, 777 x 200 x 47 in single 4.0).
constexpr int kFewWaves = 8;
template <int TYPE, class OUT>
__global__ __launch_bounds__(kFewWaves* kWave) void product_few_kernel(ProductArgs<OUT> p) {
    constexpr int kBytes = type_bytes(TYPE), kPer = 16 / kBytes, kK = kStageBytes / kBytes;
    __shared__ float sums[kFewWaves][16][20];
    const int64_t count = p.rows.get(), m0 = static_cast<int64_t>(blockIdx.y) * 16;
    const int32_t n0 = blockIdx.x * 16;
    if (m0 >= count) return;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1), r = lane & 15, g = lane >> 4;
    const bool in_a = m0 + r < count, in_b = n0 + r < p.n;
    const char* a = p.a.data + (in_a ? m0 + r : m0) * p.a.ld;
    const char* b = p.b.data + (in_b ? n0 + r : n0) * p.b.ld;
    f32x4 acc = {0, 0, 0, 0};
    for (int64_t k0 = wave * kK; k0 < p.k; k0 += kFewWaves * kK) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t k = k0 + (g + 4 * h) * kPer;
            i32x4 fa = {0, 0, 0, 0}, fb = {0, 0, 0, 0};
            if (k < p.k) {
                fa = load_16_of<kBytes>(a + k * kBytes, p.k - k);
                fb = load_16_of<kBytes>(b + k * kBytes, p.k - k);
            }
            acc = Mma<TYPE>::run(Mma<TYPE>::part(fa), Mma<TYPE>::part(fb), acc);
        }
    }
    *reinterpret_cast<f32x4*>(&sums[wave][r][4 * g]) = acc;
    __syncthreads();
    if (threadIdx.x < 32) {
        const int row = threadIdx.x / 2, col = threadIdx.x % 2 * 8, valid = p.n - n0 - col;
        if (m0 + row < count && valid > 0) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = 0;
#pragma unroll
                for (int w = 0; w < kFewWaves; ++w) v[e] += sums[w][row][col + e];
            }
            const typename OUT::Columns columns = p.out.at(n0 + col, valid, 0);
            p.out.row(columns, p.out.ahead(columns, m0 + row), m0 + row, v);
        }
    }
}

// ---- the gradient's other steps

// dz = dy * act'(pre) for the products: in 32 bits if they are in single precision, in x's type if that holds it exactly (no activation or ReLU,
// and dy of x's type), else in two parts of bfloat16; and the sums of dz's columns (from the values before they are
// cut) over the rows of a workgroup.  Bound by memory: 26 624 x 256 in bfloat16 with GELU 18 us, for 54 MB of which most
// is HBM's.  (GELU by the library's error function and one row in flight: 19 us.)
constexpr int kSlopeRows = 2;                     // rows that a thread has in flight
struct SlopeArgs {
    Count rows;
    int32_t n;
    int act;
    const void* dy;
    int64_t dy_ld;
    const void* pre;
    int64_t pre_ld;
    void* dz;                                     // nullable
    int64_t dz_ld;
    int64_t dz_low;                               // elements from a value's first part to its second
    float* sums;                                  // [gridDim.y][n], nullable
    void* dbias;                                  // with one row of workgroups: where their sums go at once, in `type`
};
// The two parts of eight values: what is nearest in bfloat16 (the largest there is, for what is finite and would not be), and what is left.
__device__ __forceinline__ void store_8_parts(void* base, int64_t at, int64_t low, int valid, const float (&v)[8]) {
    float hi[8], lo[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float most = 0x1.fep127f, near = static_cast<float>(static_cast<__bf16>(v[e]));
        hi[e] = fabsf(v[e]) > most && fabsf(v[e]) < __builtin_inff() ? __builtin_copysignf(most, v[e]) : near;
        const float rest = v[e] - hi[e];
        lo[e] = rest - rest == 0.0f ? rest : 0.0f;
    }
    store_8_of<kBF16>(base, at, valid, hi);
    store_8_of<kBF16>(base, at + low, valid, lo);
}
// (LANES threads share a row of the workgroup's columns, eight each; the others go through the rows)
constexpr int kInParts = -1;
template <int TYPE, int Z_TYPE, bool SLOPE, int LANES>
__global__ __launch_bounds__(kBlock) void slope_kernel(SlopeArgs p) {
    constexpr int kSubs = kBlock / LANES, kCols = LANES * 8;
    __shared__ float s[kSubs][kCols + 4];
    const int64_t count = p.rows.get(), per = (count + gridDim.y - 1) / gridDim.y;
    const int64_t row0 = blockIdx.y * per, row1 = row0 + per < count ? row0 + per : count;
    const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES, col = blockIdx.x * kCols + lane * 8;
    const int valid = p.n - col < 8 ? p.n - col : 8;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (valid > 0)
        for (int64_t row = row0 + sub; row < row1; row += kSubs * kSlopeRows) {
            float d[kSlopeRows][8], z[kSlopeRows][8];
#pragma unroll
            for (int k = 0; k < kSlopeRows; ++k) {
                const int64_t r = row + kSubs * k < row1 ? row + kSubs * k : row;            // (a row that there is; its values are dropped below)
                load_8_of<TYPE>(p.dy, r * p.dy_ld + col, valid, d[k]);
                if (SLOPE) load_8_of<TYPE>(p.pre, r * p.pre_ld + col, valid, z[k]);
            }
#pragma unroll
            for (int k = 0; k < kSlopeRows; ++k) {
                if (row + kSubs * k >= row1) continue;
                if (SLOPE) scale_by_slope_8<TYPE == kF32>(p.act, z[k], d[k]);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += d[k][e];
                if (!p.dz) continue;
                if constexpr (Z_TYPE == kInParts) store_8_parts(p.dz, (row + kSubs * k) * p.dz_ld + col, p.dz_low, valid, d[k]);
                else store_8_of<Z_TYPE>(p.dz, (row + kSubs * k) * p.dz_ld + col, valid, d[k]);
            }
        }
    if (!p.sums && !p.dbias) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) s[sub][lane * 8 + e] = sum[e];
    __syncthreads();
    if (threadIdx.x < kCols && blockIdx.x * kCols + threadIdx.x < static_cast<uint32_t>(p.n)) {
        float t = 0;
#pragma unroll 16
        for (int k = 0; k < kSubs; ++k) t += s[k][threadIdx.x];
        if (p.dbias) store_1(TYPE, p.dbias, blockIdx.x * kCols + threadIdx.x, t);
        else p.sums[static_cast<int64_t>(blockIdx.y) * p.n + blockIdx.x * kCols + threadIdx.x] = t;
    }
}

// out[r][c] = the sum over s of part[s][r][c]; the column sums of the slope kernel ride on the launch.  `subs` threads share a cell and
// add every subs-th slice, then the shares in turn: the same order in every call.  32 slices of 256 x 512: 6.4 us; parts are L2's.
struct JoinArgs {
    const float* part;
    int64_t cells;                                // of a slice, dense
    int slices;
    int32_t cols;
    void* out;
    int64_t out_ld;
    int type;
    int subs;                                     // threads that share four cells, each with every subs-th slice
    uint32_t cell_blocks;                         // workgroups of this sum; the others have 16 columns each
    const float* sums;
    int32_t n;
    int n_sums, sum_type;
    void* sum_out;
};
__global__ __launch_bounds__(kBlock) void join_kernel(JoinArgs p) {
    if (blockIdx.x >= p.cell_blocks) {
        sum_columns(p.sums, p.n_sums, p.n, (blockIdx.x - p.cell_blocks) * kSumColumns, p.sum_out, p.sum_type);
        return;
    }
    __shared__ f32x4 s_sum[kBlock];
    const int lanes = kBlock / p.subs, lane = threadIdx.x % lanes, sub = threadIdx.x / lanes;
    const int64_t c = (static_cast<int64_t>(blockIdx.x) * lanes + lane) * 4;
    f32x4 t = {0, 0, 0, 0};
    if (c < p.cells) {
#pragma unroll 8
        for (int s = sub; s < p.slices; s += p.subs) t += __builtin_bit_cast(f32x4, load_16_of<4>(p.part + s * p.cells + c, p.cells - c));
    }
    s_sum[threadIdx.x] = t;
    __syncthreads();
    if (sub > 0) return;
    for (int k = 1; k < p.subs; ++k) t += s_sum[k * lanes + lane];
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (c + e < p.cells) store_1(p.type, p.out, (c + e) / p.cols * p.out_ld + (c + e) % p.cols, t[e]);
}

Operand operand(const void* data, int64_t ld, int type, int64_t rows, int64_t cols) {
    return Operand{static_cast<const char*>(data), ld * type_bytes(type), rows, cols};
}

uint32_t tiles_of(int64_t n, int tile) { return static_cast<uint32_t>((n + tile - 1) / tile); }

// Whether rows can go straight to LDS: 16-byte multiples at 16-byte addresses.
bool direct(const Operand& o, int bytes) {
    return reinterpret_cast<uintptr_t>(o.data) % 16 == 0 && o.ld % 16 == 0 && o.cols * bytes % 16 == 0;
}

// The tiles of a product (by_slices: k runs over rows and is cut up; deal: fewer groups than XCDs are dealt out to all of them) and the workgroups for them; false if there are too many.
template <class TILE, class OUT>
bool lay_out(ProductArgs<OUT>* p, bool by_slices, bool deal, uint32_t* blocks) {
    p->tiles_n = tiles_of(p->n, TILE::kN);
    const int64_t tiles_m = tiles_of(p->m, TILE::kM), members = by_slices ? tiles_m * p->tiles_n : p->tiles_n, groups = by_slices ? p->slices : tiles_m;
    p->dealt = deal && groups < 8;
    const int64_t tiles = (p->dealt ? groups : (groups + 7) / 8 * 8) * members;
    p->members = static_cast<uint32_t>(members);
    p->tiles = static_cast<uint32_t>(tiles);
    *blocks = static_cast<uint32_t>(std::min<int64_t>(tiles, kMostBlocks));
    return tiles < 1ll << 32;
}

template <int TYPE, class TILE, class OUT>
hipError_t launch_forward(hipStream_t stream, ProductArgs<OUT> p) {
    uint32_t blocks = 0;
    if (!lay_out<TILE>(&p, false, false, &blocks)) return hipErrorInvalidValue;
    if (direct(p.a, type_bytes(TYPE)) && direct(p.b, type_bytes(TYPE)))
        hipLaunchKernelGGL((forward_kernel<TYPE, TILE, true, OUT>), dim3(blocks), dim3(TILE::kThreads), 0, stream, p);
    else hipLaunchKernelGGL((forward_kernel<TYPE, TILE, false, OUT>), dim3(blocks), dim3(TILE::kThreads), 0, stream, p);
    return hipGetLastError();
}

// dw and dx: nullptr if not asked for
template <int TYPE, class TILE, bool PARTS>
hipError_t launch_backward(hipStream_t stream, ProductArgs<PlainOut<TYPE>>* dw, ProductArgs<PlainOut<TYPE>>* dx) {
    ProductArgs<PlainOut<TYPE>> w{};
    ProductArgs<PlainOut<TYPE>> x{};
    uint32_t dw_blocks = 0, dx_blocks = 0;
    bool straight = true;
    if (dw) {
        if (!lay_out<TILE>(dw, true, true, &dw_blocks)) return hipErrorInvalidValue;
        straight = straight && direct(dw->a, type_bytes(TYPE)) && direct(dw->b, type_bytes(TYPE));
        w = *dw;
    }
    if (dx) {
        if (!lay_out<TILE>(dx, false, true, &dx_blocks)) return hipErrorInvalidValue;
        straight = straight && direct(dx->a, type_bytes(TYPE)) && direct(dx->b, type_bytes(TYPE));
        x = *dx;
    }
    const dim3 grid(dw_blocks + dx_blocks);
    if (straight) hipLaunchKernelGGL((backward_kernel<TYPE, TILE, true, PARTS>), grid, dim3(TILE::kThreads), 0, stream, w, dw_blocks, x);
    else hipLaunchKernelGGL((backward_kernel<TYPE, TILE, false, PARTS>), grid, dim3(TILE::kThreads), 0, stream, w, dw_blocks, x);
    return hipGetLastError();
}

typedef Tile<128, 128, 2, 4> Large;
typedef Tile<64, 64, 2, 2> Small;
typedef Tile<160, 128, 2, 2> Tall;

template <int TYPE, int OUT_TYPE, bool SMOOTH>
hipError_t forward(hipStream_t stream, const LinearJob& j) {
    typedef ForwardOut<OUT_TYPE, SMOOTH> Out;
    ProductArgs<Out> p{};
    p.a = operand(j.x, j.x_ld, TYPE, j.rows.host, j.n_in);
    p.b = operand(j.w, j.w_ld, TYPE, j.n_out, j.n_in);
    p.m = j.rows.host;
    p.n = j.n_out;
    p.k = j.n_in;
    p.rows = j.rows;
    p.slices = 1;
    p.out = Out{j.x_scale, j.w_scale, j.bias, j.residual, j.residual_ld, j.pre, j.pre_ld, j.y, j.y_ld, j.act};
    // Few tiles: 16 x 16 with k shared by eight waves, 3 us + (2 + 0.45 steps) ns a tile, against 3 us + a step's latency (0.33 us with
    // elements of 16 bits, 0.27 with 8, 0.9 with 32) a step, a step being 128 bytes of k.  us, few / small tiles, half precision: 16 x 1024 x 256
    // 4.4 / 8.3, 256 x 1024 x 256 4.7 / 8.8, 777 x 1024 x 256 10.5 / 9.0; single: 777 x 200 x 48 3.4 / 9.5, 1536 x 1024 x 256
    // 27 / 29, 3000 x 256 x 256 17.5 / 11.2.  Large tiles from where they fill the CUs: 3000 x 2048 x 1024 in half precision small 23.8, large 25.5
    // (192 large tiles), 6000 45.4 and 34.3 (376).
    const int64_t steps = (p.k * type_bytes(TYPE) + kStageBytes - 1) / kStageBytes, latency = TYPE == kF32 ? 900 : TYPE == kE4M3 ? 270 : 330;
    if (static_cast<int64_t>(tiles_of(p.m, 16)) * tiles_of(p.n, 16) * (200 + 45 * steps) <= 100 * latency * steps && tiles_of(p.m, 16) <= 65535) {
        const dim3 grid(tiles_of(p.n, 16), tiles_of(p.m, 16));
        hipLaunchKernelGGL((product_few_kernel<TYPE, Out>), grid, dim3(kFewWaves * kWave), 0, stream, p);
        return hipGetLastError();
    }
    // Large lists of 16-bit elements: the height of tile that leaves the last round fullest, two tiles to a CU at a time (one of 160 rows takes a
    // quarter longer than one of 128).  us, 128 / 160 rows (bias and ReLU, z not kept): 100 000 x 2048 x 512 271 / 243, 60 000 159 / 147,
    // 30 000 x 2048 x 1024 145 / 137, but with short k, where the epilogue weighs more, 100 000 x 256 x 512 52.8 / 56.6.
    if constexpr (TYPE == kF16 || TYPE == kBF16) {
        const auto rounds = [&](int height) { return (static_cast<int64_t>(tiles_of(p.m, height)) * tiles_of(p.n, 128) + 511) / 512 * height; };
        if (steps > 8 && rounds(128) > 256 && rounds(160) < rounds(128)) return launch_forward<TYPE, Tall>(stream, p);
    }
    if (static_cast<int64_t>(tiles_of(p.m, 128)) * tiles_of(p.n, 128) >= 256) return launch_forward<TYPE, Large>(stream, p);
    return launch_forward<TYPE, Small>(stream, p);
}
template <int TYPE, int OUT_TYPE>
hipError_t forward(hipStream_t stream, const LinearJob& j) {
    return j.act == kActGelu || j.act == kActSilu ? forward<TYPE, OUT_TYPE, true>(stream, j) : forward<TYPE, OUT_TYPE, false>(stream, j);
}

constexpr int64_t kOneSliceRows = 256;
constexpr int64_t kManyTiles = 256;               // of dw
struct GradPlan {                                 // of linear_grad: what lies where in the scratch, and how far k is cut up
    bool needs_dz, in_parts, large;               // in_parts: dz in two parts; large: by large tiles
    int64_t dz_ld, dz_low;                        // elements from a part of dz to the other
    int slices;                                   // of dw's k
    unsigned slope_blocks;                        // workgroups along the rows of the slope kernel
    size_t dz, part, sums, bytes;
    explicit GradPlan(const LinearGradJob& j) {
        const auto up = [](size_t b) { return (b + 255) / 256 * 256; };
        const int64_t n = j.rows.host;
        needs_dz = (j.dx || j.dw) && (j.act != kActNone || j.out_type != j.x_type);
        in_parts = needs_dz && j.x_type != kF32 && (j.act == kActGelu || j.act == kActSilu || j.out_type != j.x_type);
        dz_ld = (j.n_out + 7) / 8 * 8;
        dz_low = in_parts ? (n * dz_ld + 127) / 128 * 128 : 0;
        // dw's k, the rows, is cut so that there are about 1024 small tiles or 256 large ones, in eights (one for each XCD) of at least
        // four steps.  us, dw of 26 624 x 512 x 256 in bfloat16: small tiles 16 slices 21.7, 32 17.4; large ones 32 20.5, 64 19.3;
        // 50 000 x 2048 x 512: large ones 4 slices 223, 8 141, 16 150.  Where dw's tiles alone fill the CUs, parts of its sums are only more to write
        // (and scratch of eight times dw in 32 bits), us in bfloat16 by eight / one: 4096 x 4096 x 2048 228 / 77, 4096 x 4096 x 4096 457 / 149,
        // 2048 x 8192 x 8192 1345 / 300, 4096 x 2048 x 2048 (256 tiles) 84 / 67; in single precision 530 / 378, 1030 / 760, 2447 / 1541, 246 / 192.  Large tiles where there are enough of them for the CUs (in single
        // precision, where a tile takes longest, for half of them), us by small / large: 5000 x 256 x 256 in bfloat16 16.4 / 18.9, in
        // single precision 32.2 / 29.5; 26 624 x 512 x 256 50.1 / 44.9; 50 000 x 2048 x 512 598 / 333.  The same numbers hold for dz in two parts: with
        // GELU in bfloat16 5000 x 256 x 256 23.4 / 27.0, 26 624 x 512 x 256 68 / 60 (16 slices 70, 32 60, 64 67), 50 000 x 2048 x 512 714 / 529.
        const auto tiles = [](int64_t m, int64_t n, int64_t edge) { return (m + edge - 1) / edge * ((n + edge - 1) / edge); };
        const int64_t steps = (n * type_bytes(j.x_type) + kStageBytes - 1) / kStageBytes;
        const auto cut = [&](int64_t edge, int64_t most) {
            const int64_t alone = tiles(j.n_out, j.n_in, edge), want = std::max<int64_t>(1, std::min<int64_t>(std::max<int64_t>(most / alone, alone < kManyTiles ? 8 : 1), steps / 4));
            return static_cast<int>(want >= 8 ? want / 8 * 8 : want);
        };
        // Where dx is asked for, too, its tiles fill the CUs beside dw's, and in single precision, where a CU has one tile at a time, fewer and longer
        // slices are quicker; without it, two tiles of 16 bits fit a CU, if that leaves slices of a dozen steps.  us by 256 / the other: dx and dw of
        // 26 624 x 512 x 256 in single precision 133 / 127, 100 000 x 128 x 128 71 / 63, 8000 x 512 x 256 41.7 / 39.2; dw alone in bfloat16
        // 15 000 x 1024 x 512 41 / 36, 50 000 x 512 x 256 39.1 / 38.4, 200 000 x 512 x 256 132 / 94, but 26 624 x 512 x 256 36.8 / 39.3.
        const bool longer = j.x_type == kF32 && j.dx, more = j.x_type != kF32 && !j.dx && steps * tiles(j.n_out, j.n_in, 128) >= 12 * 512;
        slices = cut(128, longer ? 128 : more ? 512 : 256);
        large = (j.dx ? tiles(n, j.n_in, 128) : 0) + (j.dw ? tiles(j.n_out, j.n_in, 128) * slices : 0) >= (j.x_type == kF32 ? 128 : 256);
        if (!large) slices = cut(64, 1024);
        slope_blocks = static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>((n + 31) / 32, 512)));
        // (few rows: one slice, whose sums need no joining; a launch less)
        if (n <= kOneSliceRows) slices = 1, slope_blocks = 1;
        dz = 0;
        part = dz + (needs_dz ? up(static_cast<size_t>(n * dz_ld + dz_low) * type_bytes(j.x_type)) : 0);
        sums = part + (j.dw ? up(static_cast<size_t>(slices) * j.n_out * j.n_in * sizeof(float)) : 0);
        bytes = sums + (j.dbias ? up(static_cast<size_t>(slope_blocks) * j.n_out * sizeof(float)) : 0);
    }
};

template <int TYPE, int LANES>
hipError_t launch_slope(hipStream_t stream, const SlopeArgs& s, const LinearGradJob& j, unsigned blocks, bool in_parts) {
    const dim3 grid(tiles_of(j.n_out, LANES * 8), blocks), block(kBlock);
    const bool slope = j.act != kActNone;
    if constexpr (TYPE != kF32) {
        if (in_parts || j.out_type != TYPE) {
            if (j.out_type == TYPE) hipLaunchKernelGGL((slope_kernel<TYPE, kInParts, true, LANES>), grid, block, 0, stream, s);
            else if (slope) hipLaunchKernelGGL((slope_kernel<kF32, kInParts, true, LANES>), grid, block, 0, stream, s);
            else hipLaunchKernelGGL((slope_kernel<kF32, kInParts, false, LANES>), grid, block, 0, stream, s);
            return hipGetLastError();
        }
    }
    if (slope) hipLaunchKernelGGL((slope_kernel<TYPE, TYPE, true, LANES>), grid, block, 0, stream, s);
    else hipLaunchKernelGGL((slope_kernel<TYPE, TYPE, false, LANES>), grid, block, 0, stream, s);
    return hipGetLastError();
}

template <int TYPE>
hipError_t backward(hipStream_t stream, const LinearGradJob& j, char* scratch) {
    const GradPlan plan(j);
    const void* dz = plan.needs_dz ? scratch + plan.dz : j.dy;
    const int64_t dz_ld = plan.needs_dz ? plan.dz_ld : j.dy_ld;
    hipError_t e = hipSuccess;
    if (plan.needs_dz || j.dbias) {
        SlopeArgs s{j.rows, j.n_out, j.act, j.dy, j.dy_ld, j.pre, j.pre_ld, plan.needs_dz ? scratch + plan.dz : nullptr, plan.dz_ld, plan.dz_low,
                    j.dbias && plan.slope_blocks > 1 ? reinterpret_cast<float*>(scratch + plan.sums) : nullptr, plan.slope_blocks > 1 ? nullptr : j.dbias};
        e = j.n_out <= 32 ? launch_slope<TYPE, 4>(stream, s, j, plan.slope_blocks, plan.in_parts) : launch_slope<TYPE, 16>(stream, s, j, plan.slope_blocks, plan.in_parts);
    }
    const bool has_dx = j.dx && j.rows.host > 0;
    if (e == hipSuccess && (has_dx || j.dw)) {
        ProductArgs<PlainOut<TYPE>> x{};
        x.a = operand(dz, dz_ld, TYPE, j.rows.host, j.n_out);
        x.b = operand(j.w, j.w_ld, TYPE, j.n_out, j.n_in);
        x.a_low = plan.dz_low * type_bytes(TYPE);
        x.m = j.rows.host;
        x.n = j.n_in;
        x.k = j.n_out;
        x.rows = j.rows;
        x.slices = 1;
        x.out = PlainOut<TYPE>{j.dx, j.dx_ld, 0, false};
        ProductArgs<PlainOut<TYPE>> w{};
        w.a = x.a;
        w.a_low = x.a_low;
        w.b = operand(j.x, j.x_ld, TYPE, j.rows.host, j.n_in);
        w.m = j.n_out;
        w.n = j.n_in;
        w.k = j.rows.host;
        w.rows = j.rows;
        w.slices = plan.slices;
        w.out = plan.slices > 1 ? PlainOut<TYPE>{scratch + plan.part, j.n_in, static_cast<int64_t>(j.n_out) * j.n_in, true} : PlainOut<TYPE>{j.dw, j.dw_ld, 0, false};
        ProductArgs<PlainOut<TYPE>>*dw = j.dw ? &w : nullptr, *dx = has_dx ? &x : nullptr;
        if constexpr (TYPE != kF32) {
            if (plan.in_parts) e = plan.large ? launch_backward<TYPE, Large, true>(stream, dw, dx) : launch_backward<TYPE, Small, true>(stream, dw, dx);
        }
        if (!plan.in_parts) e = plan.large ? launch_backward<TYPE, Large, false>(stream, dw, dx) : launch_backward<TYPE, Small, false>(stream, dw, dx);
    }
    const bool join_dw = j.dw && plan.slices > 1, join_dbias = j.dbias && plan.slope_blocks > 1;
    if (e == hipSuccess && (join_dw || join_dbias)) {
        JoinArgs a{};
        if (join_dw) {
            a.part = reinterpret_cast<const float*>(scratch + plan.part);
            a.cells = static_cast<int64_t>(j.n_out) * j.n_in;
        }
        a.slices = plan.slices;
        a.cols = j.n_in;
        a.out = j.dw;
        a.out_ld = j.dw_ld;
        a.type = TYPE;
        for (a.subs = 1; a.subs < 16 && a.slices / (2 * a.subs) >= 8;) a.subs *= 2;
        a.cell_blocks = tiles_of(a.cells, 4 * kBlock / a.subs);
        a.sums = reinterpret_cast<const float*>(scratch + plan.sums);
        a.n = j.n_out;
        a.n_sums = static_cast<int>(plan.slope_blocks);
        a.sum_type = j.out_type;
        a.sum_out = j.dbias;
        const uint32_t blocks = a.cell_blocks + (join_dbias ? tiles_of(j.n_out, kSumColumns) : 0);
        hipLaunchKernelGGL(join_kernel, dim3(blocks), dim3(kBlock), 0, stream, a);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

hipError_t launch_linear(hipStream_t stream, const LinearJob& j) {
    if (j.rows.host < 1) return hipSuccess;
    switch (j.x_type) {
        case kF32: return forward<kF32, kF32>(stream, j);
        case kF16: return j.out_type == kF32 ? forward<kF16, kF32>(stream, j) : forward<kF16, kF16>(stream, j);
        case kBF16: return j.out_type == kF32 ? forward<kBF16, kF32>(stream, j) : forward<kBF16, kBF16>(stream, j);
        case kE4M3:
            return j.out_type == kF32 ? forward<kE4M3, kF32>(stream, j) : j.out_type == kF16 ? forward<kE4M3, kF16>(stream, j) : forward<kE4M3, kBF16>(stream, j);
    }
    return hipErrorInvalidValue;
}

size_t linear_grad_scratch_bytes(const LinearGradJob& j) { return GradPlan(j).bytes; }

hipError_t launch_linear_grad(hipStream_t stream, const LinearGradJob& j, void* scratch) {
    char* at = static_cast<char*>(scratch);
    switch (j.x_type) {
        case kF32: return backward<kF32>(stream, j, at);
        case kF16: return backward<kF16>(stream, j, at);
        case kBF16: return backward<kBF16>(stream, j, at);
    }
    return hipErrorInvalidValue;
}

}  // namespace helios
