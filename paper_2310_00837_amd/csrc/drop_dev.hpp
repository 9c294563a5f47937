// Which elements of a matrix are dropped: 16 bits of a counter-based generator for every element, so that no mask is stored.
#pragma once
#include "layer.hpp"
#include "layer_dev.hpp"
#include "philox.hpp"

namespace helios {

constexpr uint32_t kDropTag = 0x44524f50u;               // tells these counters from the sampler's

__device__ __forceinline__ uint64_t drop_seed(const Drop& d) { return d.seed_dev ? *d.seed_dev : d.seed; }

// Which of the eight elements of row `row` from column `col` (a multiple of eight) on are kept.  One counter serves eight
// elements: its ten rounds are 20 products of 32 x 32 bits, which take the vector unit about as long as 80 other instructions, so 32 bits for an
// element would hold memory up (102 million elements in half precision: see dropout_kernel).
struct Kept8 {
    bool on[8];
};
__device__ __forceinline__ Kept8 kept_8(const Drop& d, uint64_t seed, int64_t row, int32_t col) {
    Kept8 kept;
    if (d.threshold == 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) kept.on[e] = true;
        return kept;
    }
    // (as if the key changed from call to call: the rounds' keys are sums that cost the scalar unit nothing, kept for a loop they are 20 registers)
    int32_t k0 = __builtin_amdgcn_readfirstlane(static_cast<int32_t>(seed)), k1 = __builtin_amdgcn_readfirstlane(static_cast<int32_t>(seed >> 32));
    asm volatile("" : "+s"(k0), "+s"(k1));
    const Philox4 w = philox4x32_10(static_cast<uint32_t>(row), static_cast<uint32_t>(col) / 8, d.site, kDropTag, static_cast<uint32_t>(k0),
                                    static_cast<uint32_t>(k1));
    const uint32_t word[4] = {w.w0, w.w1, w.w2, w.w3};
    // (16 bits against the threshold in the upper half of a word; a threshold of 65536 has no such word)
    const bool some = d.threshold < 65536u;
    const uint32_t least = some ? d.threshold << 16 : 0u;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        kept.on[2 * k] = some && word[k] << 16 >= least;
        kept.on[2 * k + 1] = some && word[k] >= least;
    }
    return kept;
}

}  // namespace helios
