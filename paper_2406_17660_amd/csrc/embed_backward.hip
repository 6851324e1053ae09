// grass_embed_backward: the gradient of the embedding, summed by tokens.
#include "elem.hpp"
#include "tokens.hpp"

namespace grass {
namespace {

constexpr int kThreads = 256;

// A workgroup for each row of dE and 256 columns at a time: it looks through all token numbers in order.
template <typename TY, typename TE>
__global__ __launch_bounds__(kThreads) void sum_kernel(const TY* dY, int64_t lddy, Tokens ids, int64_t T, int64_t n, float scale,
                                                       bool accumulate, TE* dE, int64_t ldde) {
    for (int64_t v = blockIdx.x; v < ids.V; v += gridDim.x)
        for (int64_t c = threadIdx.x; c < n; c += kThreads) {
            float sum = 0.f;
            bool there = false;
            for (int64_t t = 0; t < T; ++t)
                if (ids[t] == v) {
                    sum += load_as_f32(dY + t * lddy + c);
                    there = true;
                }
            TE* out = dE + v * ldde + c;
            if (accumulate) {
                if (there) store_from_f32(out, load_as_f32(out) + sum * scale);
            } else {
                store_from_f32(out, sum * scale);
            }
        }
}

template <typename TY, typename TE>
void launch(const void* dY, int64_t lddy, const Tokens& ids, int64_t T, int64_t n, float scale, bool accumulate, void* dE,
            int64_t ldde, hipStream_t s) {
    const unsigned grid = static_cast<unsigned>(ids.V < kMostBlocks ? ids.V : kMostBlocks);
    sum_kernel<TY, TE><<<grid, kThreads, 0, s>>>(static_cast<const TY*>(dY), lddy, ids, T, n, scale, accumulate, static_cast<TE*>(dE), ldde);
}

}  // namespace

size_t embed_backward_workspace_bytes(int64_t T, int64_t V, int64_t n) { return 0; }

grass_status launch_embed_backward(const void* dY, grass_dtype dt, int64_t lddy, const void* ids, grass_index idt, int64_t T,
                                   int64_t V, int64_t n, float scale, bool accumulate, void* dE, grass_dtype gdt,
                                   int64_t ldde, void* ws, hipStream_t s) {
    if (T == 0 && accumulate) return GRASS_OK;
    const Tokens tok = tokens(ids, idt, V);
    const auto go = [&](auto from, auto to) { launch<decltype(from), decltype(to)>(dY, lddy, tok, T, n, scale, accumulate, dE, ldde, s); };
    if (dt == GRASS_F32) gdt == GRASS_F32 ? go(float{}, float{}) : go(float{}, uint16_t{});
    else gdt == GRASS_F32 ? go(uint16_t{}, float{}) : go(uint16_t{}, uint16_t{});
    return launch_status();
}

}  // namespace grass
