// grass_logp_forward: log probabilities of given tokens, entropies and alternatives.
#include "elem.hpp"
#include "tokens.hpp"

namespace grass {
namespace {

constexpr int kThreads = 256;

struct ForwardArgs {
    const void* logits;
    int64_t T, ldl;
    int V, top;
    Tokens targets;
    float scale;
    float *logp, *entropy, *rmax, *rlog, *top_logp;
    int32_t* top_idx;
};

// Numbers in the order of the logits (both zeros alike); below them 0.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return (u >> 31) ? ~u : u | 0x80000000u;
}

// Largest of a workgroup's values, for every thread.
template <typename N, typename F>
__device__ __forceinline__ N over_block(N v, F f) {
    __shared__ N part[kThreads / kWave];
    for (int o = kWave / 2; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o, kWave));
    __syncthreads();
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
    __syncthreads();
    v = part[0];
    for (int w = 1; w < kThreads / kWave; ++w) v = f(v, part[w]);
    return v;
}

// One row per workgroup at a time: a pass over it for the maximum, one for the sums, one for each alternative.
template <typename T>
__global__ __launch_bounds__(kThreads) void forward_kernel(ForwardArgs a) {
    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        const T* x = static_cast<const T*>(a.logits) + t * a.ldl;
        float m = -INFINITY;
        for (int c = threadIdx.x; c < a.V; c += kThreads) m = fmaxf(m, load_as_f32(x + c));
        m = over_block(m, [](float p, float q) { return fmaxf(p, q); });
        const float m0 = m == -INFINITY ? 0.f : m;
        float sum = 0.f, mean = 0.f;
        for (int c = threadIdx.x; c < a.V; c += kThreads) {
            const float d = scaled_difference(load_as_f32(x + c), m0, a.scale), e = expf(d);
            sum += e;
            if (e > 0.f) mean += e * d;
        }
        const auto add = [](float p, float q) { return p + q; };
        sum = over_block(sum, add);
        mean = over_block(mean, add);
        const bool none = sum == 0.f;
        const float log = none ? 0.f : logf(sum);
        if (threadIdx.x == 0) {
            if (a.rmax) a.rmax[t] = m;
            if (a.rlog) a.rlog[t] = log;
            if (a.entropy) a.entropy[t] = none ? 0.f : log - mean / sum;
            if (a.logp) {
                const uint32_t j = a.targets[t];
                a.logp[t] = j < a.targets.V ? scaled_difference(load_as_f32(x + j), m0, a.scale) - log : 0.f;
            }
        }
        uint64_t before = ~uint64_t{0};
        for (int k = 0; k < a.top; ++k) {
            uint64_t best = 0;
            for (int c = threadIdx.x; c < a.V; c += kThreads) {
                const float z = load_as_f32(x + c);
                const uint64_t key = static_cast<uint64_t>(order_of(z)) << 32 | static_cast<uint32_t>(~c);
                if (z > -INFINITY && key < before && key > best) best = key;
            }
            best = over_block(best, [](uint64_t p, uint64_t q) { return p > q ? p : q; });
            if (threadIdx.x == 0) {
                const int c = static_cast<int>(~static_cast<uint32_t>(best));
                a.top_idx[t * a.top + k] = best && log == log ? c : -1;
                a.top_logp[t * a.top + k] = log != log ? NAN : best ? scaled_difference(load_as_f32(x + c), m0, a.scale) - log : -INFINITY;
            }
            before = best;
        }
    }
}

}  // namespace

size_t logp_forward_workspace_bytes(int64_t T, int64_t V, int64_t top, grass_dtype dt) { return 0; }

grass_status launch_logp_forward(const void* logits, grass_dtype dt, int64_t T, int64_t V, int64_t ldl, const void* targets,
                                 grass_index idt, float scale, float* logp, float* entropy, float* rmax, float* rlog,
                                 int64_t top, float* top_logp, int32_t* top_idx, void* ws, hipStream_t s) {
    if (T == 0) return GRASS_OK;
    const ForwardArgs a{logits, T, ldl, static_cast<int>(V), static_cast<int>(top), tokens(targets, idt, V), scale,
                        logp, entropy, rmax, rlog, top_logp, top_idx};
    const unsigned grid = static_cast<unsigned>(T < kMostBlocks ? T : kMostBlocks);
    if (dt == GRASS_F32) forward_kernel<float><<<grid, kThreads, 0, s>>>(a);
    else forward_kernel<uint16_t><<<grid, kThreads, 0, s>>>(a);
    return launch_status();
}

}  // namespace grass
