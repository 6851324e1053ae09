// grass_logp_backward: the gradient of the logits from those of log probabilities and entropies.
//
// Measured: 32768 x 32000 bf16, a tenth of the rows without a target, 688 us (3.99 GB, 5.8 TB/s); 513 x 50001 fp32 with the entropy's
// gradient, in any position, 36.8 (5.6 TB/s).
//
// Bound by memory: the logits are read once and their gradient is written once, rows without a gradient only written.
// With c = scale log2(e) and w = x c - (rmax c + rlog log2(e)), p = 2^w, the gradient of logit j is
//   p (k0 + k1 w) [+ scale dlogp at the target],  k1 = -scale dentropy ln(2),  k0 = -scale (dlogp + dentropy entropy).
#include "elem.hpp"
#include "tokens.hpp"

namespace grass {
namespace {

struct BackwardArgs {
    const void* logits;
    void* dlogits;
    int64_t T, ldl, lddl;
    int V, pieces;
    Tokens targets;
    float scale;
    const float *rmax, *rlog, *dlogp, *entropy, *dentropy;
};

// TPR threads take V vectors each of a row, in blocks of 256: a piece of it where the row has more.
template <int TPR_, int V_>
struct Shape {
    static constexpr int TPR = TPR_, V = V_, kRows = 256 / TPR_;
};

template <typename T, typename S, bool kEntropy, bool kOnce>
__global__ __launch_bounds__(256) void backward_kernel(BackwardArgs a) {
    constexpr int TPR = S::TPR, V = S::V, N = 16 / sizeof(T);
    const int lane = threadIdx.x % TPR;
    const int group = TPR >= kWave ? __builtin_amdgcn_readfirstlane(threadIdx.x / TPR) : threadIdx.x / TPR;
    const int64_t items = a.T * a.pieces;
    for (int64_t item = static_cast<int64_t>(blockIdx.x) * S::kRows + group; item < items; item += static_cast<int64_t>(gridDim.x) * S::kRows) {
        const int64_t t = a.pieces == 1 ? item : item / a.pieces;
        const int64_t first = (item - t * a.pieces) * (TPR * V * N);
        const T* x0 = static_cast<const T*>(a.logits) + t * a.ldl;
        T* d0 = static_cast<T*>(a.dlogits) + t * a.lddl;
        const float m = a.rmax[t], log = a.rlog[t], m0 = m == -INFINITY ? 0.f : m;
        const uint32_t target = a.dlogp ? a.targets[t] : a.targets.V;
        const float g = target < a.targets.V && !(m == -INFINITY && log == 0.f) ? a.dlogp[t] * a.scale : 0.f;
        const float h = kEntropy ? a.dentropy[t] * a.scale : 0.f, H = kEntropy ? a.entropy[t] : 0.f;
        const bool none = g == 0.f && h == 0.f;
        Raw<T, N> x[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int64_t at = first + (v * TPR + lane) * N;
            x[v].zero();
            if (none) continue;
            if (at + N <= a.V) x[v].template load_as<kOnce>(x0 + at);
            else x[v].load_some(x0 + at, at < a.V ? static_cast<int>(a.V - at) : 0);
        }
        // b is rounded; by how much is known, and p is 2^off times the 2^w that is formed.  Where the product with c
        // is large, or beyond fp32, the difference is formed first.
        constexpr float kRest = 1.44269504088896341 - 1.44269504088896341f;
        const float c = scale_of_powers(a.scale), mc = m0 * c, l2 = log * kLog2e, b = -(mc + l2);
        const bool near = fabsf(mc) <= 0x1p20f;
        float off = fmaf(log, kLog2e, -l2) + log * kRest;
        if (near) {
            const float back = -b - mc;  // what of the sum is l2, and what each of the two lost
            off += fmaf(m0, c, -mc) + ((mc - (-b - back)) + (l2 - back));
        }
        const float factor = __builtin_amdgcn_exp2f(-off);
        const float k1 = -h * kLn2 * factor, k0 = -(g + h * (H - off * kLn2)) * factor;
        const auto vector = [&](int v, auto power) {
            const int64_t at = first + (v * TPR + lane) * N;
            float d[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float w = power(x[v].get(i)), e = __builtin_amdgcn_exp2f(w);
                // (0 times minus infinity is 0 here; multiplied by e first, as k1 w + k0 may be beyond fp32)
                d[i] = kEntropy ? fmaf(e * k1, fmaxf(w, -200.f), e * k0) : e * k0;
            }
            const int64_t place = static_cast<int64_t>(target) - at;
            if (place >= 0 && place < N) {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (i == place) d[i] += g;
            }
            x[v].set(d);
        };
        if (!none) {
            if (near) {
#pragma unroll
                for (int v = 0; v < V; ++v) vector(v, [&](float z) { return fmaf(z, c, b); });
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v) vector(v, [&](float z) { return (z - m0) * c - l2; });
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int64_t at = first + (v * TPR + lane) * N;
            if (at + N <= a.V) x[v].template store_as<kOnce>(d0 + at);
            else x[v].store_some(d0 + at, at < a.V ? static_cast<int>(a.V - at) : 0);
        }
    }
}

template <typename T>
void launch(BackwardArgs a, hipStream_t s) {
    constexpr int N = 16 / sizeof(T);
    const int64_t vectors = (a.V + N - 1) / N;
    const bool once = 2.0 * a.T * a.V * sizeof(T) > kStreamed;
    const auto go = [&](auto shape) {
        typedef decltype(shape) S;
        a.pieces = static_cast<int>((vectors + S::TPR * S::V - 1) / (S::TPR * S::V));
        const int64_t blocks = (a.T * a.pieces + S::kRows - 1) / S::kRows;
        const unsigned grid = walking_grid(blocks);
        if (a.dentropy) once ? backward_kernel<T, S, true, true><<<grid, 256, 0, s>>>(a) : backward_kernel<T, S, true, false><<<grid, 256, 0, s>>>(a);
        else once ? backward_kernel<T, S, false, true><<<grid, 256, 0, s>>>(a) : backward_kernel<T, S, false, false><<<grid, 256, 0, s>>>(a);
    };
    // The fewest threads and vectors that hold a row, so that few lanes are idle, and up to four vectors a thread.  us with the shape
    // taken / the next one: 131072 x 128 bf16 14.4 / 53.2, 32768 x 512 15.8 / 45.2 (16 threads in pieces 15.1), 8192 x 2048 15.1 / 17.2,
    // 262144 x 2048 559 / 531, 4096 x 4096 12.5 / 18.0 (one vector 15.4), 65536 x 8192 342 with four vectors, 344 with two, 559 with one.
    if (vectors <= 16) go(Shape<16, 1>{});
    else if (vectors <= 64) go(Shape<64, 1>{});
    else if (vectors <= 256) go(Shape<256, 1>{});
    else if (vectors <= 512) go(Shape<256, 2>{});
    else go(Shape<256, 4>{});
}

}  // namespace

grass_status launch_logp_backward(const void* logits, grass_dtype dt, int64_t T, int64_t V, int64_t ldl, const void* targets,
                                  grass_index idt, float scale, const float* rmax, const float* rlog, const float* dlogp,
                                  const float* entropy, const float* dentropy, void* dlogits, int64_t lddl, hipStream_t s) {
    if (T == 0) return GRASS_OK;
    const BackwardArgs a{logits, dlogits, T, ldl, lddl, static_cast<int>(V), 1, tokens(targets, idt, V), scale, rmax, rlog, dlogp,
                         entropy, dentropy};
    if (dt == GRASS_F32) launch<float>(a, s);
    else launch<uint16_t>(a, s);
    return launch_status();
}

}  // namespace grass
