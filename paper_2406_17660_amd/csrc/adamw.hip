// grass_adamw_plan, grass_adamw_step, grass_grad_norm: AdamW and the gradients' norm over many tensors.
//
// All of it is bound by memory: every array is read once and written once.  The plan cuts the
// tensors into chunks of 2048 elements and holds for each the addresses where it starts, so that a
// workgroup finds its work with one 64-byte load whatever the number and sizes of the tensors;
// chunks of one combination of types lie together and take one launch.  A thread handles eight consecutive
// elements, or four (twice, beside 8-bit moments) where an fp32 array is among those written; the 16 or 32 lanes that hold a block of 128
// lie in one row of a wavefront or two, which exchange values without LDS.  Measured on large tensors: 6.0 TB/s
// with fp32 moments (65.6M values of bf16 W and G: 240 us), 6.3 to 6.4 with 8-bit ones (262M: 415 to 424 us), 6.5
// for the norm (262M bf16 gradients: 81 us); a step of 65 tensors of 4096 takes its kernel 3.5 us.
#include "adam.hpp"
#include "elem.hpp"

namespace grass {
namespace {

constexpr int kChunk = 2048;
constexpr int kThreads = kChunk / 8;  // of the norm's kernels
constexpr int kQBlock = 128;  // elements that share a scale

// What of a chunk starts on 16 bytes: W, G, M and V; G.
constexpr uint32_t kAllOn16 = 1, kGradientOn16 = 2;

struct alignas(16) Chunk {
    void* W;
    const void* G;
    void* M;
    void* V;
    float* mscale;
    float* vscale;
    int32_t elems;
    int32_t gdt;
    float weight_decay;
    uint32_t aligned;  // kAllOn16, kGradientOn16
};
static_assert(sizeof(Chunk) == 64, "one load of sixteen dwords");

constexpr int kStepGroups = 8;  // by W's, G's and the moments' type; two more for gradients alone

int group_of(const grass_adamw_tensor& a) {
    if (!a.W) return kStepGroups + (a.gdt == GRASS_F32 ? 0 : 1);
    return (a.wdt == GRASS_F32 ? 0 : 4) + (a.gdt == GRASS_F32 ? 0 : 2) + (a.moments == GRASS_MOMENTS_F32 ? 0 : 1);
}

grass_dtype gradient_of(int group) {  // the type of G
    if (group >= kStepGroups) return group == kStepGroups ? GRASS_F32 : GRASS_BF16;
    return group & 2 ? GRASS_BF16 : GRASS_F32;
}

// The pieces a tensor is cut into: itself where its rows follow one another, else its rows.
struct Pieces {
    int64_t count, elems;
};
Pieces pieces_of(const grass_adamw_tensor& a) {
    const bool dense = a.rows <= 1 || (a.ldg == a.cols && (!a.W || a.ldw == a.cols));
    if (a.rows == 0 || a.cols == 0) return {0, 0};
    return dense ? Pieces{1, a.rows * a.cols} : Pieces{a.rows, a.cols};
}

struct StepArgs {
    const Chunk* chunks;
    AdamParams adam;
    uint32_t t;
    const float* grad_scale;
};

// Moments of N consecutive elements of a thread, V times over a chunk.  fp32: four, so that a wavefront's
// access is one piece of memory, and no more, in workgroups of 512 (65.6M values 236 to 242 us, with
// twice four in 256 244 to 246) ...
struct MomentsF32 {
    static constexpr int N = 4, V = 1;
    float m[N], v[N];
    template <bool kOnce>
    __device__ __forceinline__ void load(const Chunk& c, int at, int left) {
        Raw<float, N> a, b;
        const float *pm = static_cast<const float*>(c.M) + at, *pv = static_cast<const float*>(c.V) + at;
        if (left >= N) {
            a.load_as<kOnce>(pm);
            b.load_as<kOnce>(pv);
        } else {
            a.load_some(pm, left);
            b.load_some(pv, left);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            m[i] = a.get(i);
            v[i] = b.get(i);
        }
    }
    template <bool kOnce>
    __device__ __forceinline__ void store(const Chunk& c, int at, int left, uint32_t) const {
        Raw<float, N> a, b;
        a.set(m);
        b.set(v);
        float *pm = static_cast<float*>(c.M) + at, *pv = static_cast<float*>(c.V) + at;
        if (left >= N) {
            a.store_as<kOnce>(pm);
            b.store_as<kOnce>(pv);
        } else {
            a.store_some(pm, left);
            b.store_some(pv, left);
        }
    }
};

// The largest of the 16 lanes of a row, in every one of them.
template <int kRotate>
__device__ __forceinline__ uint32_t row_rotate(uint32_t x) {
    return static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(x), 0x120 + kRotate, 0xF, 0xF, true));
}
__device__ __forceinline__ uint32_t row_max(uint32_t x) {
    x = max(x, row_rotate<8>(x));
    x = max(x, row_rotate<4>(x));
    x = max(x, row_rotate<2>(x));
    return max(x, row_rotate<1>(x));
}

// The largest of the LANES (16 or 32) consecutive lanes that hold a block, in every one of them.
template <int LANES>
__device__ __forceinline__ uint32_t block_max(uint32_t x) {
    static_assert(LANES == 16 || LANES == 32, "one row of 16 lanes or two");
    x = row_max(x);
    if constexpr (LANES == 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        x = max(r[0], r[1]);
    }
    return x;
}

constexpr uint32_t kInf = 0x7F800000u;

// One kind of 8-bit moment: kMan bits of mantissa, scale 2^(e - kTop).  Scaled by a further
// 2^(bias - 127) the type's numbers, subnormal ones too, are the fp32 numbers whose bits are the code
// followed by zeros; so a value becomes a code by cutting its bits after adding u's bits to them.
// kLeast: the least code of a value that is not zero.  1 for V: what lies below its block's smallest code
// would be cut to zero on most steps, while M's own cut leaves some of M, and a step that then divides M by
// the root of nothing but its own gradient is thousands of lr long.
template <int kMan, int kTop, int kBias, uint32_t kLeast>
struct Code8 {
    static constexpr int kCut = 23 - kMan;
    // the exponent of the block's largest value from its lanes' N values each (all of them get the same)
    template <int N>
    __device__ static __forceinline__ uint32_t exponent(const float (&x)[N]) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t b = __float_as_uint(x[i]) & 0x7FFFFFFFu;
            top = max(top, b < kInf ? b : 0u);
        }
        return max(block_max<kQBlock / N>(top) >> 23, 24u);
    }
    __device__ static __forceinline__ float scale(uint32_t e) { return __uint_as_float((e - kTop) << 23); }
    __device__ static __forceinline__ uint32_t code(float x, float inv_scale, uint32_t word) {
        const float y = (x * inv_scale) * __uint_as_float(kBias << 23);
        const uint32_t b = __float_as_uint(x);
        const uint32_t cut = ((__float_as_uint(y) & 0x7FFFFFFFu) + (word >> (32 - kCut))) >> kCut;
        const uint32_t c = kLeast ? max(cut, min(b & 0x7FFFFFFFu, kLeast)) : cut;
        return ((b & 0x7FFFFFFFu) < kInf ? c : 0x7Fu) | (b >> 31 << 7);
    }
    // codes of N values; word: u's bits at the first of them
    template <int N>
    __device__ static __forceinline__ void codes(const float (&x)[N], uint32_t e, uint32_t word, uint32_t (&r)[N / 4]) {
        const float inv = __uint_as_float((254u + kTop - e) << 23);
#pragma unroll
        for (int i = 0; i < N / 4; ++i) r[i] = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) r[i / 4] |= code(x[i], inv, word + i * 0x9E3779B1u) << (8 * (i & 3));
    }
};
typedef Code8<3, 7, 7, 0> CodeM;     // e4m3
typedef Code8<2, 14, 15, 1> CodeV;   // e5m2

// N codes from any byte on, four to a word.
typedef uint32_t word_any_t __attribute__((aligned(1)));
template <bool kOnce, int N>
__device__ __forceinline__ void load_codes(const void* p, int at, int left, uint32_t (&r)[N / 4]) {
    const uint8_t* q = static_cast<const uint8_t*>(p) + at;
    if (left >= N) {
        if constexpr (N == 8) {
            const raw2_any_t* whole = reinterpret_cast<const raw2_any_t*>(q);
            const raw2_t a = kOnce ? __builtin_nontemporal_load(whole) : *whole;
            r[0] = a[0];
            r[1] = a[1];
        } else {
            const word_any_t* whole = reinterpret_cast<const word_any_t*>(q);
            r[0] = kOnce ? __builtin_nontemporal_load(whole) : *whole;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < N / 4; ++i) r[i] = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < left) r[i / 4] |= static_cast<uint32_t>(q[i]) << (8 * (i & 3));
}
template <bool kOnce, int N>
__device__ __forceinline__ void store_codes(void* p, int at, int left, const uint32_t (&r)[N / 4]) {
    uint8_t* q = static_cast<uint8_t*>(p) + at;
    if (left >= N) {
        if constexpr (N == 8) {
            const raw2_t a = {r[0], r[1]};
            raw2_any_t* whole = reinterpret_cast<raw2_any_t*>(q);
            if constexpr (kOnce) __builtin_nontemporal_store(a, whole);
            else *whole = a;
        } else {
            word_any_t* whole = reinterpret_cast<word_any_t*>(q);
            if constexpr (kOnce) __builtin_nontemporal_store(r[0], whole);
            else *whole = r[0];
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < left) q[i] = static_cast<uint8_t>(r[i / 4] >> (8 * (i & 3)));
}

// ... and 8 bits: eight at a time, or four where W is fp32, whose accesses are whole pieces then (66M values of
// fp32 W and G: 172 us, 190 with eight; 262M of bf16: 482, with eight 419).  Every lane of the wavefront takes
// part in store(), those without elements too.
template <int N_>
struct MomentsQ8 {
    static constexpr int N = N_, V = 8 / N_;
    float m[N], v[N];
    template <bool kOnce>
    __device__ __forceinline__ void load(const Chunk& c, int at, int left) {
        uint32_t a[N / 4], b[N / 4];
        load_codes<kOnce, N>(c.M, at, left, a);
        load_codes<kOnce, N>(c.V, at, left, b);
        const float sm = left > 0 ? c.mscale[at / kQBlock] : 0.f, sv = left > 0 ? c.vscale[at / kQBlock] : 0.f;
#pragma unroll
        for (int w = 0; w < N / 4; ++w) {
            const f32x2_t m0 = __builtin_amdgcn_cvt_pk_f32_fp8(a[w], false), m1 = __builtin_amdgcn_cvt_pk_f32_fp8(a[w], true);
            const f32x2_t v0 = __builtin_amdgcn_cvt_pk_f32_bf8(b[w], false), v1 = __builtin_amdgcn_cvt_pk_f32_bf8(b[w], true);
            m[4 * w] = m0.x * sm; m[4 * w + 1] = m0.y * sm; m[4 * w + 2] = m1.x * sm; m[4 * w + 3] = m1.y * sm;
            v[4 * w] = v0.x * sv; v[4 * w + 1] = v0.y * sv; v[4 * w + 2] = v1.x * sv; v[4 * w + 3] = v1.y * sv;
        }
    }
    template <bool kOnce>
    __device__ __forceinline__ void store(const Chunk& c, int at, int left, uint32_t t) const {
        const uint32_t em = CodeM::exponent(m), ev = CodeV::exponent(v);
        const uint32_t j = static_cast<uint32_t>(at % kQBlock) * 0x9E3779B1u;
        uint32_t a[N / 4], b[N / 4];
        CodeM::codes(m, em, j + t * 0x6A09E667u, a);
        CodeV::codes(v, ev, j + t * 0xBB67AE85u, b);
        if (left <= 0) return;
        store_codes<kOnce, N>(c.M, at, left, a);
        store_codes<kOnce, N>(c.V, at, left, b);
        if (at % kQBlock == 0) {
            c.mscale[at / kQBlock] = CodeM::scale(em);
            c.vscale[at / kQBlock] = CodeV::scale(ev);
        }
    }
};

template <typename Moments>
constexpr int kStepThreads = kChunk / (Moments::N * Moments::V);

template <bool kOnce, typename W, typename G, typename Moments>
__device__ __forceinline__ void step_chunk(const Chunk& c, const AdamParams& p, uint32_t t, float grad_scale) {
    constexpr int N = Moments::N, V = Moments::V;
    Raw<W, N> w[V];
    Raw<G, N> g[V];
    Moments s[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int at = (k * kStepThreads<Moments> + threadIdx.x) * N, left = c.elems - at;
        const W* pw = static_cast<const W*>(c.W) + at;
        const G* pg = static_cast<const G*>(c.G) + at;
        if (left >= N) {
            w[k].template load_as<kOnce>(pw);
            g[k].template load_as<kOnce>(pg);
        } else {
            w[k].load_some(pw, left);
            g[k].load_some(pg, left);
        }
        s[k].template load<kOnce>(c, at, left);
    }
    const float keep = 1.0f - p.lr * c.weight_decay;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int at = (k * kStepThreads<Moments> + threadIdx.x) * N, left = c.elems - at;
        float out[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            {
#pragma clang fp contract(off)
                const float x = g[k].get(i) * grad_scale;
                const float m0 = p.b1 * s[k].m[i], m1 = p.one_minus_b1 * x;
                const float v0 = p.b2 * s[k].v[i], v1 = p.one_minus_b2 * x;
                s[k].m[i] = m0 + m1;
                s[k].v[i] = v0 + v1 * x;
            }
            // hardware square root and reciprocal, as in adam_elem
            const float step = p.lr * (s[k].m[i] * p.inv_c1) *
                               __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(s[k].v[i] * p.inv_c2) + p.eps);
            out[i] = w[k].get(i) * keep - step;
        }
        s[k].template store<kOnce>(c, at, left, t);
        w[k].set(out);
        W* pw = static_cast<W*>(c.W) + at;
        if (left >= N) w[k].template store_as<kOnce>(pw);
        else w[k].store_some(pw, left);
    }
}

// One chunk per workgroup.  The streaming hint only where every access is one whole piece: lines that two
// lanes share are then read twice.  At any size: between two steps of a model the arrays leave the cache.  With the hint and without,
// us, three sets of arrays in turn: bf16 W and G, 8-bit moments 1M values 4.8 and 4.7, 4M 10.3 and 11.6, 34M 59.5 and 65.2; fp32
// moments 1M 5.2 and 5.1, 4M 17.1 and 15.5, 17M 61.9 and 71.0, 67M 250 and 275.  What a step alone leaves in the cache and
// repeats there is faster without (17M bf16, fp32 moments, one set 59.7 and 53.3).
template <typename W, typename G, typename Moments>
__global__ __launch_bounds__(kStepThreads<Moments>) void adamw_kernel(StepArgs a) {
    const Chunk c = a.chunks[blockIdx.x];
    const AdamParams p = resolve(a.adam);
    const uint32_t t = p.step_scalars ? static_cast<uint32_t>(p.step_scalars[3]) : a.t;
    const float grad_scale = a.grad_scale ? *a.grad_scale : 1.0f;
    if (grad_scale != grad_scale) return;
    if (c.aligned & kAllOn16) step_chunk<true, W, G, Moments>(c, p, t, grad_scale);
    else step_chunk<false, W, G, Moments>(c, p, t, grad_scale);
}

// Workgroups that walk the chunks for the norm: 262M bf16 values 81.0 us, with 1024 of them 107, 1536 83.3, 4096 84.2; 66M fp32
// ones 44.1, 49.9, 43.8, 44.4.
constexpr int kNormBlocks = 2048;

// A thread's part of the gradients of a chunk, as it lies in memory: eight bf16 values in a row (in the
// first half), or twice four fp32 values.
struct Gradients {
    Raw<float, 4> x[2];
    template <bool kOnce>
    __device__ __forceinline__ void load(const Chunk& c, int tid) {
        if (c.gdt == GRASS_F32) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int at = (k * kThreads + tid) * 4, left = c.elems - at;
                const float* p = static_cast<const float*>(c.G) + at;
                if (left >= 4) x[k].load_as<kOnce>(p);
                else x[k].load_some(p, left);
            }
        } else {
            const int at = tid * 8, left = c.elems - at;
            const uint16_t* p = static_cast<const uint16_t*>(c.G) + at;
            Raw<uint16_t, 8> h;
            if (left >= 8) h.load_as<kOnce>(p);
            else h.load_some(p, left);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[0].w[i] = h.w[i];
        }
    }
    __device__ __forceinline__ double squares(const Chunk& c) const {
        double s = 0.0;
        if (c.gdt == GRASS_F32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) s += static_cast<double>(x[i / 4].get(i & 3)) * static_cast<double>(x[i / 4].get(i & 3));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double v = __uint_as_float((i & 1) ? x[0].w[i / 2] & 0xFFFF0000u : x[0].w[i / 2] << 16);
                s += v * v;
            }
        }
        return s;
    }
};

// Sum over a block of B threads, in thread 0.
template <int B>
__device__ __forceinline__ double block_sum(double s) {
    __shared__ double part[B / kWave];
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) s += __shfl_xor(s, o, kWave);
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = s;
    __syncthreads();
    s = part[0];
#pragma unroll
    for (int w = 1; w < B / kWave; ++w) s += part[w];
    return s;
}

// Squares of the chunks first, first + step, ...: a thread's part of two at a time, whose loads are under
// way together.
template <bool kOnce>
__device__ __forceinline__ double squares_of(const Chunk* __restrict__ chunks, int64_t count, int64_t first, int64_t step) {
    const int tid = threadIdx.x % kThreads;
    double s = 0.0;
    for (int64_t k = first; k < count; k += 2 * step) {
        const bool two = k + step < count;
        const Chunk c0 = chunks[k], c1 = chunks[two ? k + step : k];
        Gradients g0, g1;
        if (kOnce && (c0.aligned & c1.aligned & kGradientOn16)) {
            g0.load<true>(c0, tid);
            g1.load<true>(c1, tid);
        } else {
            g0.load<false>(c0, tid);
            g1.load<false>(c1, tid);
        }
        s += g0.squares(c0);
        if (two) s += g1.squares(c1);
    }
    return s;
}

__device__ __forceinline__ void write_norm(double s, float max_norm, float* out) {
    const double norm = sqrt(s);
    out[0] = static_cast<float>(norm);
    const double factor = norm > static_cast<double>(max_norm) ? static_cast<double>(max_norm) / norm : 1.0;
    out[1] = s <= 1.7976931348623157e308 ? static_cast<float>(factor) : __uint_as_float(0x7FC00000u);
}

// kOnce: from kStreamed bytes on, read with the streaming hint where accesses are whole
// pieces (262M bf16 values 88.5 -> 83.4 us; it costs where they are not: 7M values in 300 tensors 8.8 -> 9.6).
template <bool kOnce>
__global__ __launch_bounds__(kThreads) void grad_squares_kernel(const Chunk* __restrict__ chunks, int64_t count, double* part) {
    const double s = block_sum<kThreads>(squares_of<kOnce>(chunks, count, blockIdx.x, gridDim.x));
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// (1024 threads: two of the most sums each, 4.2 us with 256 threads)
constexpr int kJoinThreads = 1024;
__global__ __launch_bounds__(kJoinThreads) void grad_norm_kernel(const double* __restrict__ part, int count, float max_norm, float* out) {
    double s = 0.0;
    for (int k = threadIdx.x; k < count; k += kJoinThreads) s += part[k];
    s = block_sum<kJoinThreads>(s);
    if (threadIdx.x == 0) write_norm(s, max_norm, out);
}

// Few chunks: one block of four times the threads takes them all, in one launch.  32 chunks take it 5.0 us, 64 8.1;
// the two kernels take 2.8 and 1.7 and what goes between them, and 2.8 more of the host.
constexpr int kFewThreads = 4 * kThreads;
constexpr int64_t kFewChunks = 32;
__global__ __launch_bounds__(kFewThreads) void grad_norm_few_kernel(const Chunk* __restrict__ chunks, int count, float max_norm, float* out) {
    const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads);
    const double s = block_sum<kFewThreads>(squares_of<false>(chunks, count, group, kFewThreads / kThreads));
    if (threadIdx.x == 0) write_norm(s, max_norm, out);
}

int64_t chunks_in(const grass_adamw_layout& layout) {
    int64_t n = 0;
    for (int i = 0; i < GRASS_ADAMW_GROUPS; ++i) n += layout.chunks[i];
    return n;
}

int norm_blocks(const grass_adamw_layout& layout) {
    const int64_t n = chunks_in(layout);
    return static_cast<int>(n < kNormBlocks ? n : kNormBlocks);
}

}  // namespace

void adamw_count(int count, const grass_adamw_tensor* tensors, grass_adamw_layout* layout) {
    *layout = grass_adamw_layout{};
    for (int i = 0; i < count; ++i) {
        const Pieces p = pieces_of(tensors[i]);
        layout->chunks[group_of(tensors[i])] += p.count * ((p.elems + kChunk - 1) / kChunk);
    }
}

size_t adamw_plan_bytes(const grass_adamw_layout& layout) { return static_cast<size_t>(chunks_in(layout)) * sizeof(Chunk); }

void adamw_lay_out(int count, const grass_adamw_tensor* tensors, const grass_adamw_layout& layout, void* plan) {
    Chunk* next[GRASS_ADAMW_GROUPS];
    Chunk* at = static_cast<Chunk*>(plan);
    for (int i = 0; i < GRASS_ADAMW_GROUPS; ++i) {
        next[i] = at;
        at += layout.chunks[i];
    }
    for (int i = 0; i < count; ++i) {
        const grass_adamw_tensor& a = tensors[i];
        const Pieces p = pieces_of(a);
        Chunk*& out = next[group_of(a)];
        const int64_t wsize = a.wdt == GRASS_F32 ? 4 : 2, gsize = a.gdt == GRASS_F32 ? 4 : 2;
        const bool q8 = a.moments == GRASS_MOMENTS_Q8;
        for (int64_t r = 0; r < p.count; ++r)
            for (int64_t e = 0; e < p.elems; e += kChunk) {
                Chunk c{};
                c.G = static_cast<const char*>(a.G) + (r * a.ldg + e) * gsize;
                c.elems = static_cast<int32_t>(p.elems - e < kChunk ? p.elems - e : kChunk);
                c.gdt = a.gdt;
                c.aligned = aligned_to(c.G, 16) ? kGradientOn16 : 0;
                if (a.W) {
                    const int64_t s = r * a.cols + e;
                    c.W = static_cast<char*>(a.W) + (r * a.ldw + e) * wsize;
                    c.M = static_cast<char*>(a.M) + s * (q8 ? 1 : 4);
                    c.V = static_cast<char*>(a.V) + s * (q8 ? 1 : 4);
                    c.mscale = q8 ? a.mscale + s / kQBlock : nullptr;
                    c.vscale = q8 ? a.vscale + s / kQBlock : nullptr;
                    c.weight_decay = a.weight_decay;
                    if (aligned_to(c.W, 16) && aligned_to(c.G, 16) && aligned_to(c.M, 16) && aligned_to(c.V, 16))
                        c.aligned |= kAllOn16;
                }
                *out++ = c;
            }
    }
}

bool adamw_steps(const grass_adamw_layout& layout) {
    for (int i = kStepGroups; i < GRASS_ADAMW_GROUPS; ++i)
        if (layout.chunks[i] != 0) return false;
    return true;
}

void adamw_step_scalars(float lr, float b1, float b2, int64_t t, float out[4]) {
    adam_step_scalars(lr, b1, b2, t, out);
    out[3] = static_cast<float>(t % (1 << 24));
}

grass_status launch_adamw(const void* plan, const grass_adamw_layout& layout, float lr, float b1, float b2,
                          float eps, int64_t t, const float* step_scalars, const float* grad_scale, hipStream_t s) {
    if (chunks_in(layout) == 0) return GRASS_OK;
    StepArgs a{static_cast<const Chunk*>(plan), make_params(lr, b1, b2, eps, t, step_scalars),
               static_cast<uint32_t>(t % (1 << 24)), grad_scale};
    for (int i = 0; i < kStepGroups; ++i) {
        // a grid has fewer than 2^32 threads
        for (int64_t left = layout.chunks[i]; left > 0;) {
            const int64_t now = left < (int64_t{1} << 22) ? left : int64_t{1} << 22;
            const unsigned grid = static_cast<unsigned>(now);
            const auto go = [&](auto w, auto g, auto moments) {
                typedef decltype(moments) Moments;
                adamw_kernel<decltype(w), decltype(g), Moments><<<grid, kStepThreads<Moments>, 0, s>>>(a);
            };
            switch (i) {
                case 0: go(float{}, float{}, MomentsF32{}); break;
                case 1: go(float{}, float{}, MomentsQ8<4>{}); break;
                case 2: go(float{}, uint16_t{}, MomentsF32{}); break;
                case 3: go(float{}, uint16_t{}, MomentsQ8<4>{}); break;
                case 4: go(uint16_t{}, float{}, MomentsF32{}); break;
                case 5: go(uint16_t{}, float{}, MomentsQ8<8>{}); break;
                case 6: go(uint16_t{}, uint16_t{}, MomentsF32{}); break;
                case 7: go(uint16_t{}, uint16_t{}, MomentsQ8<8>{}); break;
            }
            a.chunks += now;
            left -= now;
        }
    }
    return launch_status();
}

size_t grad_norm_workspace_bytes(const grass_adamw_layout& layout) {
    return static_cast<size_t>(norm_blocks(layout)) * sizeof(double);
}

grass_status launch_grad_norm(const void* plan, const grass_adamw_layout& layout, float max_norm, float* out,
                              void* ws, hipStream_t s) {
    const int blocks = norm_blocks(layout);
    double* part = static_cast<double*>(ws);
    if (blocks <= kFewChunks) {
        grad_norm_few_kernel<<<1, kFewThreads, 0, s>>>(static_cast<const Chunk*>(plan), blocks, max_norm, out);
        return launch_status();
    }
    double bytes = 0;
    for (int i = 0; i < GRASS_ADAMW_GROUPS; ++i)
        bytes += static_cast<double>(layout.chunks[i]) * kChunk * (gradient_of(i) == GRASS_F32 ? 4 : 2);
    (bytes > kStreamed ? grad_squares_kernel<true> : grad_squares_kernel<false>)
        <<<static_cast<unsigned>(blocks), kThreads, 0, s>>>(static_cast<const Chunk*>(plan), chunks_in(layout), part);
    grad_norm_kernel<<<1, kJoinThreads, 0, s>>>(part, blocks, max_norm, out);
    return launch_status();
}

}  // namespace grass
