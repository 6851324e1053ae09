// grass_logp_backward: the gradient of the logits from those of log probabilities and entropies.
#include "elem.hpp"
#include "tokens.hpp"

namespace grass {
namespace {

constexpr int kThreads = 256;

struct BackwardArgs {
    const void* logits;
    void* dlogits;
    int64_t T, ldl, lddl;
    int V;
    Tokens targets;
    float scale;
    const float *rmax, *rlog, *dlogp, *entropy, *dentropy;
};

template <typename T>
__global__ __launch_bounds__(kThreads) void backward_kernel(BackwardArgs a) {
    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        const T* x = static_cast<const T*>(a.logits) + t * a.ldl;
        T* dx = static_cast<T*>(a.dlogits) + t * a.lddl;
        const float m = a.rmax[t], log = a.rlog[t], m0 = m == -INFINITY ? 0.f : m;
        const uint32_t target = a.dlogp ? a.targets[t] : a.targets.V;
        const float g = target < a.targets.V && !(m == -INFINITY && log == 0.f) ? a.dlogp[t] : 0.f;
        const float h = a.dentropy ? a.dentropy[t] : 0.f, H = a.dentropy ? a.entropy[t] : 0.f;
        const bool none = g == 0.f && h == 0.f;
        for (int c = threadIdx.x; c < a.V; c += kThreads) {
            float d = 0.f;
            if (!none) {
                const float l = scaled_difference(load_as_f32(x + c), m0, a.scale) - log, p = expf(l);
                d = g * ((static_cast<uint32_t>(c) == target ? 1.f : 0.f) - p);
                if (p != 0.f) d -= h * p * (l + H);
            }
            store_from_f32(dx + c, d * a.scale);
        }
    }
}

}  // namespace

grass_status launch_logp_backward(const void* logits, grass_dtype dt, int64_t T, int64_t V, int64_t ldl, const void* targets,
                                  grass_index idt, float scale, const float* rmax, const float* rlog, const float* dlogp,
                                  const float* entropy, const float* dentropy, void* dlogits, int64_t lddl, hipStream_t s) {
    if (T == 0) return GRASS_OK;
    const BackwardArgs a{logits, dlogits, T, ldl, lddl, static_cast<int>(V), tokens(targets, idt, V), scale, rmax, rlog, dlogp,
                         entropy, dentropy};
    const unsigned grid = static_cast<unsigned>(T < kMostBlocks ? T : kMostBlocks);
    if (dt == GRASS_F32) backward_kernel<float><<<grid, kThreads, 0, s>>>(a);
    else backward_kernel<uint16_t><<<grid, kThreads, 0, s>>>(a);
    return launch_status();
}

}  // namespace grass
