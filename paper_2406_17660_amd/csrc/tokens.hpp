// Token numbers of 32 or 64 bits, and what the passes over logits share.
#pragma once
#include "common.hpp"

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

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945f;
// scale log2(e), at most the largest number there is (0 times it is 0)
__device__ __forceinline__ float scale_of_powers(float scale) { return fminf(scale * kLog2e, 3.40282347e38f); }
// scale * (x - m) of two logits, also where the difference alone would pass the range of fp32.
__device__ __forceinline__ float scaled_difference(float x, float m, float scale) { return 2.f * (scale * (0.5f * x - 0.5f * m)); }

}  // namespace
}  // namespace grass
