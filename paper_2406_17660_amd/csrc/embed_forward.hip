// grass_embed_forward: rows of the embedding by token.
//
// Bound by memory: Y is written once, and a row of E is read from memory once and from the cache for the other
// places of its token.
#include "elem.hpp"
#include "tokens.hpp"

namespace grass {
namespace {

constexpr int kThreads = 256;

template <typename TE, typename TY>
__global__ __launch_bounds__(kThreads) void lookup_kernel(const TE* E, int64_t n, int64_t lde, Tokens ids, int64_t T, float scale,
                                                          TY* Y, int64_t ldy) {
    for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
        const uint32_t v = ids[t];
        const TE* e = E + v * lde;
        for (int64_t c = threadIdx.x; c < n; c += kThreads)
            store_from_f32(Y + t * ldy + c, v < ids.V ? load_as_f32(e + c) * scale : 0.f);
    }
}

template <typename TE, typename TY>
void launch(const void* E, int64_t n, int64_t lde, const Tokens& ids, int64_t T, float scale, void* Y, int64_t ldy, hipStream_t s) {
    const unsigned grid = static_cast<unsigned>(T < kMostBlocks ? T : kMostBlocks);
    lookup_kernel<TE, TY><<<grid, kThreads, 0, s>>>(static_cast<const TE*>(E), n, lde, ids, T, scale, static_cast<TY*>(Y), ldy);
}

}  // namespace

grass_status launch_embed_forward(const void* E, grass_dtype edt, int64_t V, int64_t n, int64_t lde, const void* ids,
                                  grass_index idt, int64_t T, float scale, void* Y, grass_dtype ydt, int64_t ldy,
                                  hipStream_t s) {
    if (T == 0) return GRASS_OK;
    const Tokens tok = tokens(ids, idt, V);
    const auto go = [&](auto from, auto to) { launch<decltype(from), decltype(to)>(E, n, lde, tok, T, scale, Y, ldy, s); };
    if (edt == GRASS_F32) ydt == GRASS_F32 ? go(float{}, float{}) : go(float{}, uint16_t{});
    else ydt == GRASS_F32 ? go(uint16_t{}, float{}) : go(uint16_t{}, uint16_t{});
    return launch_status();
}

}  // namespace grass
