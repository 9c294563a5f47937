// Device-side helpers of the operators of a model's layer: element types, rows of any alignment, activations.
#pragma once
#include "common.hpp"

#include <type_traits>

namespace helios {

// element types, same values as helios_dtype
constexpr int kF32 = 0, kF16 = 1, kBF16 = 2, kE4M3 = 3;
// activations, same values as helios_act
constexpr int kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3;

__host__ __device__ constexpr int type_bytes(int type) { return type == kF32 ? 4 : type == kE4M3 ? 1 : 2; }

struct E4M3 {                                             // storage of an 8-bit float (4 exponent bits, 3 of mantissa, no infinities)
    uint8_t bits;
};
template <int TYPE> struct ElementOf;
template <> struct ElementOf<kF32> { typedef float type; };
template <> struct ElementOf<kF16> { typedef _Float16 type; };
template <> struct ElementOf<kBF16> { typedef __bf16 type; };
template <> struct ElementOf<kE4M3> { typedef E4M3 type; };

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// 16 bytes at any address: rows may start anywhere an element may (the loads are the same, an unaligned one takes
// the memory pipe a little longer).
typedef int32_t i32x4_any __attribute__((ext_vector_type(4), aligned(1)));
__device__ __forceinline__ i32x4 load_16(const void* p) { return *static_cast<const i32x4_any*>(p); }
__device__ __forceinline__ void store_16(void* p, i32x4 v) { *static_cast<i32x4_any*>(p) = v; }
// The same with STREAM: hinted to leave the caches to others.
template <bool STREAM>
__device__ __forceinline__ i32x4 load_16_once(const void* p) {
    if constexpr (STREAM) return __builtin_nontemporal_load(static_cast<const i32x4_any*>(p));
    else return load_16(p);
}
template <bool STREAM>
__device__ __forceinline__ void store_16_once(void* p, i32x4 v) {
    if constexpr (STREAM) __builtin_nontemporal_store(v, static_cast<i32x4_any*>(p));
    else store_16(p, v);
}

// 16 bytes of a row of which `valid` elements of BYTES bytes exist; zeros in the place of the others
template <int BYTES>
__device__ __forceinline__ i32x4 load_16_of(const void* p, int64_t valid) {
    constexpr int N = 16 / BYTES;
    if (valid >= N) return load_16(p);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < N - 1; ++e) {
        if (e >= valid) break;
        if (BYTES == 4) w[e] = static_cast<const uint32_t*>(p)[e];
        else if (BYTES == 2) w[e / 2] |= static_cast<uint32_t>(static_cast<const uint16_t*>(p)[e]) << (16 * (e & 1));
        else w[e / 4] |= static_cast<uint32_t>(static_cast<const uint8_t*>(p)[e]) << (8 * (e & 3));
    }
    return i32x4{static_cast<int32_t>(w[0]), static_cast<int32_t>(w[1]), static_cast<int32_t>(w[2]), static_cast<int32_t>(w[3])};
}

// Eight neighbouring elements, widened to 32 bits (TYPE: one of the floating types of 16 or 32 bits): from their 16 or 32 bytes ...
template <int TYPE>
__device__ __forceinline__ void widen_8(const i32x4 (&raw)[type_bytes(TYPE) / 2], float (&v)[8]) {
    if constexpr (TYPE == kF32) {
        const f32x4 a = __builtin_bit_cast(f32x4, raw[0]), b = __builtin_bit_cast(f32x4, raw[1]);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = a[e], v[4 + e] = b[e];
    } else if constexpr (TYPE == kF16) {
        const f16x8 a = __builtin_bit_cast(f16x8, raw[0]);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(a[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int32_t two = raw[0][e];
            v[2 * e] = __builtin_bit_cast(float, two << 16);
            v[2 * e + 1] = __builtin_bit_cast(float, two & static_cast<int32_t>(0xffff0000));
        }
    }
}
// Rows that are taken eight elements at a time: their width is a multiple of eight, is not, or is less than eight; or it is a multiple of eight, and what the
// call reads and writes is hinted to leave the caches to others.  That is for calls that pass over more than half of what the last cache (256 MB)
// holds, so that little of it is met again.  100 000 rows of 256 looked up in single precision and added to 16-bit ones (205 MB): 36.9 us with the
// hint, 41.7 without; 50 000 of them 20.2 and 19.1.  Dropout of 52 000 rows of 1024 in 16 bits (213 MB): 35.3 and 39.9.  The join of 100 003 rows of
// 1024 in 16 bits (820 MB): 144.7 and 150.3, of 10 000 (82 MB) 21.9 and 19.6; its gradient for 26 624 of 512 (164 MB): 35.9 and 38.7.
enum Rows { kWholeRows = 0, kRowsWithRest = 1, kShortRows = 2, kStreamedRows = 3 };
constexpr int64_t kStreamBytes = 128ll << 20;
inline Rows rows_of(int32_t width, int64_t bytes) {
    if (width % 8 != 0) return width > 8 ? kRowsWithRest : kShortRows;
    return bytes > kStreamBytes ? kStreamedRows : kWholeRows;
}
// Eight elements as they are in memory, in half the registers where they have 16 bits; zeros where there are none.
template <int TYPE>
struct Raw8 {
    i32x4 v[type_bytes(TYPE) / 2];
    __device__ __forceinline__ void load(const void* base, int64_t at, int valid) {
        constexpr int kBytes = type_bytes(TYPE), kPer = 16 / kBytes;
        const char* p = static_cast<const char*>(base) + at * kBytes;
#pragma unroll
        for (int k = 0; k < 8 / kPer; ++k) {
            v[k] = i32x4{0, 0, 0, 0};
            if (valid > k * kPer) v[k] = load_16_of<kBytes>(p + 16 * k, valid - k * kPer);
        }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int k = 0; k < type_bytes(TYPE) / 2; ++k) v[k] = i32x4{0, 0, 0, 0};
    }
    // The elements from column `col` (a multiple of eight) on of the row of `width` elements that begins at `at`, without a branch that differs from lane
    // to lane, so that no load waits for those before it: where fewer than eight are left, the row's last eight are loaded, and align()
    // puts them in their places.  A lane beyond the row holds values of its end.  (Short rows are loaded with branches.)
    template <int ROWS>
    __device__ __forceinline__ void load_row(const void* base, int64_t at, int32_t col, int32_t width) {
        if (ROWS == kShortRows) {
            load(base, at + col, width - col);
            return;
        }
        const char* p = static_cast<const char*>(base) + (at + (col < width - 8 ? col : width - 8)) * type_bytes(TYPE);
#pragma unroll
        for (int k = 0; k < type_bytes(TYPE) / 2; ++k) v[k] = load_16_once<ROWS == kStreamedRows>(p + 16 * k);
    }
    template <int ROWS>
    __device__ __forceinline__ void align(int32_t col, int32_t width) {
        if (ROWS != kRowsWithRest) return;
        const int rest = width & 7;                       // the same for all lanes: the branches are the scalar unit's
        constexpr int kWords = type_bytes(TYPE) * 2, kPerWord = 4 / type_bytes(TYPE);
        const bool moves = col + 8 > width;
        const int words = (8 - rest) / kPerWord;          // to go down by
        uint32_t w[kWords];
#pragma unroll
        for (int k = 0; k < kWords; ++k) w[k] = static_cast<uint32_t>(v[k / 4][k % 4]);
        const auto down = [&](auto by) {
            constexpr int kBy = decltype(by)::value;
            if (words & kBy)
#pragma unroll
                for (int k = 0; k < kWords; ++k) {
                    const uint32_t from = k + kBy < kWords ? w[(k + kBy) % kWords] : 0u;
                    w[k] = moves ? from : w[k];
                }
        };
        if (kWords == 8) down(std::integral_constant<int, 4>());
        down(std::integral_constant<int, 2>());
        down(std::integral_constant<int, 1>());
        if (kPerWord == 2 && (rest & 1))
#pragma unroll
            for (int k = 0; k < kWords; ++k) w[k] = !moves ? w[k] : w[k] >> 16 | (k + 1 < kWords ? w[k + 1] : 0u) << 16;
#pragma unroll
        for (int k = 0; k < kWords; ++k) v[k / 4][k % 4] = static_cast<int32_t>(w[k]);
    }
};
// ... or from memory
template <int TYPE>
__device__ __forceinline__ void load_8(const void* base, int64_t at, float (&v)[8]) {
    const char* p = static_cast<const char*>(base) + at * type_bytes(TYPE);
    i32x4 raw[type_bytes(TYPE) / 2];
    raw[0] = load_16(p);
    if constexpr (TYPE == kF32) raw[1] = load_16(p + 16);
    widen_8<TYPE>(raw, v);
}
template <int TYPE>
__device__ __forceinline__ float load_1(const void* base, int64_t at) {
    typedef typename ElementOf<TYPE>::type T;
    return static_cast<float>(static_cast<const T*>(base)[at]);
}
// ... of which the first `valid` exist; 0 in the place of the others
template <int TYPE>
__device__ __forceinline__ void load_8_of(const void* base, int64_t at, int valid, float (&v)[8]) {
    if (valid >= 8) {
        load_8<TYPE>(base, at, v);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < valid ? load_1<TYPE>(base, at + e) : 0.0f;
}
// Rounding to 16 bits is to nearest, ties to even.
template <int TYPE, bool STREAM = false>
__device__ __forceinline__ void store_8_of(void* base, int64_t at, int valid, const float (&v)[8]) {
    typedef typename ElementOf<TYPE>::type T;
    T* p = static_cast<T*>(base) + at;
    if (valid >= 8) {
        if constexpr (TYPE == kF32) {
            store_16_once<STREAM>(p, __builtin_bit_cast(i32x4, f32x4{v[0], v[1], v[2], v[3]}));
            store_16_once<STREAM>(p + 4, __builtin_bit_cast(i32x4, f32x4{v[4], v[5], v[6], v[7]}));
        } else {
            typedef T tx8 __attribute__((ext_vector_type(8)));
            tx8 a;
#pragma unroll
            for (int e = 0; e < 8; ++e) a[e] = static_cast<T>(v[e]);
            store_16_once<STREAM>(p, __builtin_bit_cast(i32x4, a));
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < valid) p[e] = static_cast<T>(v[e]);
}
// ... from column `col` (a multiple of eight) on of a row of `width` elements that begins at `at`: the row's last ones, where they are fewer than eight,
// as four, two and one of them.
template <int TYPE, int ROWS>
__device__ __forceinline__ void store_row_8(void* base, int64_t at, int32_t col, int32_t width, const float (&v)[8]) {
    typedef typename ElementOf<TYPE>::type T;
    typedef T tx2 __attribute__((ext_vector_type(2), aligned(sizeof(T))));
    typedef T tx4 __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    if (col + 8 <= width) {
        store_8_of<TYPE, ROWS == kStreamedRows>(base, at + col, 8, v);
    } else if ((ROWS == kRowsWithRest || ROWS == kShortRows) && col < width) {
        T* p = static_cast<T*>(base) + at + col;
        const int rest = width & 7;
        const auto two = [&](int e, float a, float b) { *reinterpret_cast<tx2*>(p + e) = tx2{static_cast<T>(a), static_cast<T>(b)}; };
        // (branches to the end: elements chosen by conditions would make an array in memory of v)
        if (rest & 4) {
            *reinterpret_cast<tx4*>(p) = tx4{static_cast<T>(v[0]), static_cast<T>(v[1]), static_cast<T>(v[2]), static_cast<T>(v[3])};
            if (rest & 2) {
                two(4, v[4], v[5]);
                if (rest & 1) p[6] = static_cast<T>(v[6]);
            } else if (rest & 1) {
                p[4] = static_cast<T>(v[4]);
            }
        } else if (rest & 2) {
            two(0, v[0], v[1]);
            if (rest & 1) p[2] = static_cast<T>(v[2]);
        } else {
            p[0] = static_cast<T>(v[0]);
        }
    }
}
// (the type is an argument of the kernel: the branches are the same for all lanes)
__device__ __forceinline__ void store_1(int type, void* base, int64_t at, float v) {
    if (type == kF32) static_cast<float*>(base)[at] = v;
    else if (type == kF16) static_cast<_Float16*>(base)[at] = static_cast<_Float16>(v);
    else static_cast<__bf16*>(base)[at] = static_cast<__bf16>(v);
}

// The normal distribution's Phi(z) and density at z.  For values that are rounded to 16 bits, by Abramowitz and Stegun, Handbook of
// Mathematical Functions, 7.1.26: erfc(u) = (a1 t + ... + a5 t^5) exp(-u^2), t = 1 / (1 + p u), off by at most 1.5e-7; one exponential serves
// both.  For single precision (PRECISE) by the error function itself: the formula is off by 1.7e-3 of the value at z = -5.  (50 000 x 64 x 512 in
// single precision with GELU: 63 us by the formula, 83 so; SiLU, whose quick exponential and reciprocal are off by 1e-6 far out, 58 and 70;
// 11 264 x 256 x 256 18.0 and 19.4, 17.6 and 18.4.)
template <bool PRECISE>
__device__ __forceinline__ float normal_cdf(float z, float* density) {
    if (PRECISE) {
        *density = 0.39894228040143268f * expf(-0.5f * z * z);
        return 0.5f * erfcf(z * -0.70710678118654752f);
    }
    const float u = fabsf(z) * 0.70710678118654752f, t = __builtin_amdgcn_rcpf(1.0f + 0.3275911f * u), e = __expf(-u * u);
    const float tail = 0.5f * e * t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
    *density = 0.39894228040143268f * e;
    return z < 0.0f ? tail : 1.0f - tail;
}
// 1 / (1 + exp(-z)), and exp(-z)
template <bool PRECISE>
__device__ __forceinline__ float logistic(float z, float* e) {
    *e = PRECISE ? expf(-z) : __expf(-z);
    return PRECISE ? 1.0f / (1.0f + *e) : __builtin_amdgcn_rcpf(1.0f + *e);
}
// GELU or SiLU of eight values (one branch for all of them)
template <bool PRECISE>
__device__ __forceinline__ void act_8(int act, float (&v)[8]) {
    float other;
    if (act == kActGelu) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= normal_cdf<PRECISE>(v[e], &other);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= logistic<PRECISE>(v[e], &other);
    }
}
// (at the infinities, which half precision keeps of a z beyond 65504, the slopes are their limits, 0 and 1)
template <bool PRECISE>
__device__ __forceinline__ float gelu_slope(float z) {
    float density;
    const float phi = normal_cdf<PRECISE>(z, &density);
    return phi + __builtin_amdgcn_fmed3f(z, -128.0f, 128.0f) * density;                // (beyond, the density is 0)
}
template <bool PRECISE>
__device__ __forceinline__ float silu_slope(float z) {
    float e;
    const float p = logistic<PRECISE>(z, &e), q = z > 0.0f ? e * p : 1.0f - p;         // (q: 1 - p, also where p is all but 1)
    return p * (1.0f + __builtin_amdgcn_fmed3f(z, -128.0f, 128.0f) * q);               // (beyond, p or q is 0)
}
// v *= the slopes at z
template <bool PRECISE>
__device__ __forceinline__ void scale_by_slope_8(int act, const float (&z)[8], float (&v)[8]) {
    if (act == kActRelu) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= z[e] > 0.0f ? 1.0f : 0.0f;
    } else if (act == kActGelu) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= gelu_slope<PRECISE>(z[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= silu_slope<PRECISE>(z[e]);
    }
}

// The value of another lane, by moves that need no trip through LDS: STEP 0 and 1 the lane 1 and 2 away (within four), 2 and 3 the
// mirrored one of eight and of sixteen lanes.
template <int STEP>
__device__ __forceinline__ float moved(float v) {
    constexpr int kControl = STEP == 0 ? 0xb1 : STEP == 1 ? 0x4e : STEP == 2 ? 0x141 : 0x140;
    const int bits = __builtin_bit_cast(int, v);
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(bits, bits, kControl, 0xf, 0xf, false));
}
// {the value of the row of 16 (32) lanes that comes first of two, that of the second}
struct TwoFloats {
    float a, b;
};
template <int ROW>
__device__ __forceinline__ TwoFloats both_rows(float v) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    const uint32_t bits = __builtin_bit_cast(uint32_t, v);
    const u32x2 r = ROW == 16 ? __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(bits, bits, false, false))
                              : __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(bits, bits, false, false));
    const uint32_t lo = r.x, hi = r.y;
    return TwoFloats{__builtin_bit_cast(float, lo), __builtin_bit_cast(float, hi)};
}
// A sum, or a maximum that keeps NaN, over the lanes of a group of G (16 or 64), the same bits in all of them.
template <int G, class OP>
__device__ __forceinline__ float group_reduce(float v, OP op) {
    static_assert(G == 16 || G == 64, "a row of lanes, or a wave");
    v = op(v, moved<0>(v));
    v = op(v, moved<1>(v));
    v = op(v, moved<2>(v));
    v = op(v, moved<3>(v));
    if (G == 64) {
        TwoFloats t = both_rows<16>(v);
        v = op(t.a, t.b);
        t = both_rows<32>(v);
        v = op(t.a, t.b);
    }
    return v;
}
template <int G>
__device__ __forceinline__ float group_sum(float v) {
    return group_reduce<G>(v, [](float a, float b) { return a + b; });
}
template <int G>
__device__ __forceinline__ float group_max(float v) {
    return group_reduce<G>(v, [](float a, float b) { return a > b || a != a ? a : b; });
}

// Where the items of a workgroup are, from number `base` on: an item is eight neighbouring columns of a row, items are numbered along the rows
// (of `blocks` items each, at most 2^21).  What is the same for all threads is the scalar unit's; the division by `blocks` goes by its
// reciprocal (off by one at most: at and blocks are below 2^22, which 32-bit floats and 24-bit products hold).
struct ItemPlaces {
    int64_t row0;
    uint32_t rem0, blocks;
    float inverse;
    __device__ __forceinline__ ItemPlaces(int64_t base, uint32_t row_blocks)
        : row0(base / row_blocks), rem0(static_cast<uint32_t>(base % row_blocks)), blocks(row_blocks), inverse(1.0f / static_cast<float>(row_blocks)) {}
    // item i's row is row0 + down
    __device__ __forceinline__ void get(uint32_t i, uint32_t* down, int32_t* col) const {
        const uint32_t at = rem0 + i;
        uint32_t q = static_cast<uint32_t>(static_cast<float>(at) * inverse);
        int32_t left = static_cast<int32_t>(at - (q & 0xffffffu) * (blocks & 0xffffffu));
        if (left < 0) q -= 1, left += static_cast<int32_t>(blocks);
        else if (left >= static_cast<int32_t>(blocks)) q += 1, left -= static_cast<int32_t>(blocks);
        *down = q;
        *col = left * 8;
    }
    // the element of a matrix where its row begins
    __device__ __forceinline__ int64_t row(int64_t ld, uint32_t down) const { return row0 * ld + static_cast<int64_t>(down) * ld; }
};

// Which of a workgroup's rows is a thread's, if LANES share one: the same for a whole wave where it is.  (Where it is not, the lanes of a wave go through
// their rows in step all the same: those that have none left take the last one, and write nothing.)
template <int LANES>
__device__ __forceinline__ int row_of_lanes() {
    const int sub = static_cast<int>(threadIdx.x) / LANES;
    return LANES >= kWave ? __builtin_amdgcn_readfirstlane(sub) : sub;
}

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
    if constexpr (LANES > kWave) {
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
// The sum over a group of lanes (16, or a wave), with the additions in group_sum's order: every step within 16 lanes is one instruction, and for a
// wave two more carry the rows' sums to the last lane (32 instructions fewer for the four sums of a row of the join's gradient).
template <int G>
__device__ __forceinline__ float lanes_sum(float v) {
    static_assert(G == 16 || G == 64, "a row of lanes, or a wave");
    const auto add = [&](auto control) {
        v += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), decltype(control)::value, 0xf, 0xf, true));
    };
    add(std::integral_constant<int, 0xb1>());
    add(std::integral_constant<int, 0x4e>());
    add(std::integral_constant<int, 0x141>());
    add(std::integral_constant<int, 0x140>());
    if (G == 16) return v;
    // (a lane's value may be read by such a move two cycles after it was written)
    asm volatile("s_nop 1\n\tv_add_f32_dpp %0, %0, %0 row_bcast:15 row_mask:0xa bank_mask:0xf\n\ts_nop 1\n\tv_add_f32_dpp %0, %0, %0 row_bcast:31 row_mask:0xc bank_mask:0xf"
        : "+v"(v));
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), kWave - 1));
}
// N sums at once, by one exchange; `s` has room for two of them, which take turns, so that one barrier does.
template <int LANES, int N>
struct RowSums {
    static constexpr int kWaves = LANES < kWave ? 1 : LANES / kWave;
    float (*s)[N][kWaves];                          // [2], in LDS; one row to a workgroup where it is used
    int turn = 0;
    __device__ __forceinline__ void run(float (&v)[N]) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = lanes_sum<(LANES < kWave ? LANES : kWave)>(v[k]);
        if (LANES <= kWave) return;
        if (lane_id() == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) s[turn][k][wave_id()] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) v[k] += s[turn][k][w];
        }
        turn ^= 1;
    }
};
template <int LANES>
__device__ __forceinline__ float row_max(float v, float* s) {
    v = group_max<(LANES < kWave ? LANES : kWave)>(v);
    if constexpr (LANES > kWave) {
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

// A row's finished values to memory at element `at` of y: rounded to TYPE, or (to_scale) to 8 bits with the row's scale.
constexpr float kE4M3Max = 448.0f, kMinScale = 0x1p-126f;
template <int TYPE, int LANES, int CHUNKS>
__device__ __forceinline__ void finish_row(float (&t)[CHUNKS][8], int32_t width, int lane, float* s, void* y, int64_t at, float* to_scale) {
    if (!to_scale) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int col = (c * LANES + lane) * 8;
            store_8_of<TYPE>(y, at + col, width - col, t[c]);
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
    if (lane == 0) *to_scale = scale;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int col = (c * LANES + lane) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float near = t[c][e] * inv;     // t / scale, but for its last bit
            t[c][e] = inv > 0.0f ? __builtin_fmaf(__builtin_fmaf(-near, scale, t[c][e]), inv, near) : near;
        }
        store_8_of_e4m3(y, at + col, width - col, t[c]);
    }
}

// out[c] = the sum over p of part[p][c], p < n_parts, for the 16 columns from `first` on, by a workgroup of kBlock threads.  Four of
// them share a part's columns and 64 go through the parts, so that few loads follow on one another; the order of the additions
// is the same in every call.
constexpr int kSumColumns = 16;
template <class STORE>                            // store(column, sum)
__device__ __forceinline__ void sum_columns(const float* part, int n_parts, int32_t n, int32_t first, STORE store) {
    constexpr int kSubs = kBlock / 4;
    __shared__ float s[kSubs][kSumColumns + 1], s2[16][kSumColumns + 1];
    const int c = threadIdx.x % 4 * 4, sub = threadIdx.x / 4, valid = n - first - c;
    f32x4 t = {0, 0, 0, 0};
#pragma unroll 4
    for (int p = sub; p < n_parts; p += kSubs) t += __builtin_bit_cast(f32x4, load_16_of<4>(part + static_cast<int64_t>(p) * n + first + c, valid));
#pragma unroll
    for (int e = 0; e < 4; ++e) s[sub][c + e] = t[e];
    __syncthreads();
    const int col = threadIdx.x % 16, q = threadIdx.x / 16;
    s2[q][col] = (s[4 * q][col] + s[4 * q + 1][col]) + (s[4 * q + 2][col] + s[4 * q + 3][col]);
    __syncthreads();
    if (q == 0 && first + col < n) {
        float v = 0;
#pragma unroll
        for (int k = 0; k < 16; ++k) v += s2[k][col];
        store(first + col, v);
    }
}
__device__ __forceinline__ void sum_columns(const float* part, int n_parts, int32_t n, int32_t first, void* out, int type) {
    sum_columns(part, n_parts, n, first, [=](int32_t col, float v) { store_1(type, out, col, v); });
}

}  // namespace helios
