// Token numbers of 32 or 64 bits, and what the kernels that walk over rows and the passes over logits share.
#pragma once
#include "elem.hpp"

namespace grass {
namespace {

// A list of token numbers; a number outside 0 .. V - 1 (compared before it is cut to 32 bits) reads as V.
struct Tokens {
    const void* p;
    bool wide;
    uint32_t V;
    __device__ __forceinline__ uint32_t operator[](int64_t t) const {
        const uint64_t id = wide ? static_cast<const uint64_t*>(p)[t]
                                 : static_cast<uint64_t>(static_cast<int64_t>(static_cast<const int32_t*>(p)[t]));
        return id < V ? static_cast<uint32_t>(id) : V;
    }
};
inline Tokens tokens(const void* p, grass_index idt, int64_t V) { return {p, idt == GRASS_I64, static_cast<uint32_t>(V)}; }

// The grid of a kernel that walks over the work of so many blocks: one workgroup for each, or `most` that take several turns.
inline unsigned walking_grid(int64_t blocks, int64_t most = kMostBlocks) {
    const int64_t forced = test_option(GRASS_TEST_MOST_BLOCKS);
    if (forced > 0 && forced < most) most = forced;
    return static_cast<unsigned>(blocks < most ? blocks : most);
}

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945f;
// scale log2(e), at most the largest number there is (0 times it is 0)
__device__ __forceinline__ float scale_of_powers(float scale) { return fminf(scale * kLog2e, 3.40282347e38f); }
// scale * (x - m) of two logits, also where the difference alone would pass the range of fp32.
__device__ __forceinline__ float scaled_difference(float x, float m, float scale) { return 2.f * (scale * (0.5f * x - 0.5f * m)); }

}  // namespace
}  // namespace grass
