// Which elements of a matrix are dropped: 16 bits of a counter-based generator for every element, so that no mask is stored.
#pragma once
#include "layer.hpp"
#include "layer_dev.hpp"
#include "philox.hpp"

namespace helios {

constexpr uint32_t kDropTag = 0x44524f50u;               // tells these counters from the sampler's

__device__ __forceinline__ uint64_t drop_seed(const Drop& d) { return d.seed_dev ? *d.seed_dev : d.seed; }

// The elements of row `row` from column `col` (a multiple of eight) on that are kept, as eight bits.  One counter serves eight
// elements: its ten rounds are 20 products of 32 x 32 bits, which take the vector unit about as long as 80 other instructions, so 32 bits for an
// element would hold memory up (102 million elements in half precision: see dropout_kernel).
__device__ __forceinline__ uint32_t kept_8(const Drop& d, uint64_t seed, int64_t row, int32_t col) {
    const Philox4 w = philox4x32_10(static_cast<uint32_t>(row), static_cast<uint32_t>(col) / 8, d.site, kDropTag, static_cast<uint32_t>(seed),
                                    static_cast<uint32_t>(seed >> 32));
    const uint32_t word[4] = {w.w0, w.w1, w.w2, w.w3};
    uint32_t bits = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        bits |= ((word[k] & 0xffffu) >= d.threshold ? 1u : 0u) << (2 * k);
        bits |= ((word[k] >> 16) >= d.threshold ? 1u : 0u) << (2 * k + 1);
    }
    return bits;
}
// (what is dropped becomes 0 whatever it was: no product)
__device__ __forceinline__ void drop_8(uint32_t kept, float scale, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (kept >> e) & 1u ? v[e] * scale : 0.0f;
}

}  // namespace helios
