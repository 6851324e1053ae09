// N consecutive elements (4 or 8) of an fp32 or bf16 array in any position: 8- or 16-byte accesses on
// the elements' own alignment, which the memory system takes on any, or single elements where fewer
// than N are there.  Sums over lanes that share a row.  Used by the norms and by AdamW.
#pragma once
#include "common.hpp"

namespace grass {
namespace {

typedef uint32_t raw2_t __attribute__((ext_vector_type(2)));
typedef uint32_t raw4_t __attribute__((ext_vector_type(4)));
typedef raw2_t raw2_any_t __attribute__((aligned(1)));
typedef raw4_t raw4_any_t __attribute__((aligned(2)));

// Nearest even, NaN stays NaN; two values per instruction.
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const f32x2_t x = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2_t));
}

// The elements as they lie in memory.  kOnce: the streaming hint, for what is not read again soon.
template <typename T, int N>
struct Raw {
    static constexpr bool kHalf = sizeof(T) == 2;
    static constexpr int kWords = N * sizeof(T) / 4, kQuads = kWords / 4;
    uint32_t w[kWords];

    template <bool kOnce>
    __device__ __forceinline__ void load_as(const T* p) {
        if constexpr (kWords == 2) {
            const raw2_any_t* q = reinterpret_cast<const raw2_any_t*>(p);
            const raw2_t a = kOnce ? __builtin_nontemporal_load(q) : *q;
            w[0] = a[0];
            w[1] = a[1];
        } else {
#pragma unroll
            for (int k = 0; k < kQuads; ++k) {
                const raw4_any_t* q = reinterpret_cast<const raw4_any_t*>(p + k * (16 / sizeof(T)));
                const raw4_t a = kOnce ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
                for (int i = 0; i < 4; ++i) w[4 * k + i] = a[i];
            }
        }
    }
    template <bool kOnce>
    __device__ __forceinline__ void store_as(T* p) const {
        if constexpr (kWords == 2) {
            const raw2_t a = {w[0], w[1]};
            raw2_any_t* q = reinterpret_cast<raw2_any_t*>(p);
            if constexpr (kOnce) __builtin_nontemporal_store(a, q);
            else *q = a;
        } else {
#pragma unroll
            for (int k = 0; k < kQuads; ++k) {
                const raw4_t a = {w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]};
                raw4_any_t* q = reinterpret_cast<raw4_any_t*>(p + k * (16 / sizeof(T)));
                if constexpr (kOnce) __builtin_nontemporal_store(a, q);
                else *q = a;
            }
        }
    }
    __device__ __forceinline__ void load(const T* p) { load_as<false>(p); }
    __device__ __forceinline__ void store(T* p) const { store_as<false>(p); }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int k = 0; k < kWords; ++k) w[k] = 0;
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (kHalf) return __uint_as_float((i & 1) ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
        else return __uint_as_float(w[i]);
    }
    __device__ __forceinline__ void set(const float (&x)[N]) {
        if constexpr (kHalf) {
#pragma unroll
            for (int k = 0; k < kWords; ++k) w[k] = pack_bf16(x[2 * k], x[2 * k + 1]);
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) w[k] = __float_as_uint(x[k]);
        }
    }
    __device__ __forceinline__ T element(int i) const {
        if constexpr (kHalf) return static_cast<T>(w[i / 2] >> (16 * (i & 1)));
        else return __uint_as_float(w[i]);
    }
    // elements 0 .. count - 1 (none where count <= 0), the others as zeros
    __device__ __forceinline__ void load_some(const T* p, int count) {
        zero();
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < count) {
                if constexpr (kHalf) w[i / 2] |= static_cast<uint32_t>(p[i]) << (16 * (i & 1));
                else w[i] = __float_as_uint(p[i]);
            }
    }
    __device__ __forceinline__ void store_some(T* p, int count) const {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < count) p[i] = element(i);
    }
};

// A row of `bytes` bytes, the same one for all lanes of a wavefront, through which a read behind its end gives
// zeros and a write behind its end does nothing: no branches around accesses, so that the compiler
// knows how many of them are under way and waits for no more than it needs.  Starts and lengths are
// multiples of 16 bytes.
struct RowWindow {
    __amdgpu_buffer_rsrc_t r;
    __device__ __forceinline__ RowWindow(const void* base, uint32_t bytes) {
        const uint64_t p = reinterpret_cast<uint64_t>(base);
        const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(p));
        const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(p >> 32));
        r = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>((static_cast<uint64_t>(hi) << 32) | lo), 0,
                                              __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
    }
    template <bool kOnce>
    __device__ __forceinline__ void load(uint32_t (&w)[4], uint32_t at) const {
        const raw4_t a = __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, kOnce ? 2 : 0);  // 2: the streaming hint
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = a[i];
    }
    template <bool kOnce>
    __device__ __forceinline__ void store(const uint32_t (&w)[4], uint32_t at) const {
        const raw4_t a = {w[0], w[1], w[2], w[3]};
        __builtin_amdgcn_raw_buffer_store_b128(a, r, at, 0, kOnce ? 2 : 0);
    }
};

template <int kCtrl>
__device__ __forceinline__ float dpp(float x) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), kCtrl, 0xF, 0xF, true));
}

// Sum over the LANES (16, 32 or 64) consecutive lanes that share a row; each of them gets it, bit for bit the
// same.  Exchanges inside rows of 16 lanes are part of the addition; rows of 16 and halves of the
// wavefront are swapped between two copies.
template <int LANES>
__device__ __forceinline__ float sum_lanes(float v) {
    static_assert(LANES == 16 || LANES == 32 || LANES == 64, "whole rows of 16 lanes");
    v += dpp<0xB1>(v);   // lanes 1 0 3 2 of each four
    v += dpp<0x4E>(v);   // lanes 2 3 0 1
    v += dpp<0x141>(v);  // mirrored in each eight
    v += dpp<0x140>(v);  // mirrored in each sixteen
    if constexpr (LANES >= 32) {
        const uint32_t a = __float_as_uint(v);
        const auto r = __builtin_amdgcn_permlane16_swap(a, a, false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if constexpr (LANES == 64) {
        const uint32_t b = __float_as_uint(v);
        const auto h = __builtin_amdgcn_permlane32_swap(b, b, false, false);
        v = __uint_as_float(h[0]) + __uint_as_float(h[1]);
    }
    return v;
}

// The same for N sums over a row that TPR threads of a block of B share: beyond a wavefront the
// wavefronts' sums meet in LDS, one barrier a call; `at` alternates between two places, so that a call
// does not overwrite what a slower wavefront still reads.  Every thread of the block must take part.
template <int TPR, int B, int N>
struct RowSum {
    float (*part)[B / kWave][N];
    int at = 0;
    __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = sum_lanes<TPR < kWave ? TPR : kWave>(v[k]);
        if constexpr (TPR > kWave) {
            constexpr int kWaves = TPR / kWave;
            const int wave = threadIdx.x / kWave;
            if (threadIdx.x % kWave == 0)
#pragma unroll
                for (int k = 0; k < N; ++k) part[at][wave][k] = v[k];
            __syncthreads();
            const int first = wave / kWaves * kWaves;
#pragma unroll
            for (int k = 0; k < N; ++k) {
                v[k] = part[at][first][k];
#pragma unroll
                for (int w = 1; w < kWaves; ++w) v[k] += part[at][first + w][k];
            }
            at ^= 1;
        }
    }
};

// Where a thread's vector v of a row of n values starts, for rows of at least N values that TPR threads
// share: every vector is read and written whole.  The one that would end behind the row is the row's
// last N values instead, whose first `skip` are the thread before's too: both compute and write the
// same there, and sums leave them out here.  A vector without values of its own (skip = N) is another
// copy of the row's last.  The first kFull vectors of every thread lie inside the row whatever n is.
struct Span {
    int at, skip;
};
template <int TPR, int kFull, int N>
__device__ __forceinline__ Span span(int v, int lane, int n) {
    const int c = (v * TPR + lane) * N;
    if (v < kFull || c + N <= n) return {c, 0};
    return {n - N, c < n ? c - (n - N) : N};
}

// Threads that share a row, each with V vectors of 16 bytes of which the row fills kFull, in blocks of 512.
template <int TPR_, int V_, int kFull_>
struct RowShape {
    static constexpr int TPR = TPR_, V = V_, kFull = kFull_, B = 512;
};
constexpr int kWidestRow = 16384;  // values of a row that stay in registers
// The shape for a row of n values, as a call of f with it.  Two vectors per thread, so that a workgroup
// has 16 KB of each array under way, or three where two of twice as many threads would leave a quarter of them and
// more without work and three(threads of such a row) says so; more for the widest rows, one for the narrowest.
template <typename T, typename Three, typename F>
void by_shape(int64_t n, Three&& three, F&& f) {
    const int64_t vectors = (n * static_cast<int64_t>(sizeof(T)) + 15) / 16;
    if (vectors <= 16) f(RowShape<16, 1, 0>{});
    else if (vectors <= 32) f(RowShape<32, 1, 0>{});
    else if (vectors <= 64) f(RowShape<64, 1, 0>{});
    else if (vectors <= 128) f(RowShape<64, 2, 1>{});
    else if (vectors <= 192 && three(64)) f(RowShape<64, 3, 2>{});
    else if (vectors <= 256) f(RowShape<128, 2, 1>{});
    else if (vectors <= 384 && three(128)) f(RowShape<128, 3, 2>{});
    else if (vectors <= 512) f(RowShape<256, 2, 1>{});
    else if (vectors <= 768 && three(256)) f(RowShape<256, 3, 2>{});
    else if (vectors <= 1024) f(RowShape<512, 2, 1>{});
    else if (vectors <= 1536) f(RowShape<512, 3, 2>{});
    else if (vectors <= 2048) f(RowShape<512, 4, 3>{});
    else if constexpr (sizeof(T) == 4) {
        if (vectors <= 3072) f(RowShape<512, 6, 4>{});
        else f(RowShape<512, 8, 6>{});
    }
}
template <typename T>
bool in_registers(int64_t n) { return n >= static_cast<int64_t>(16 / sizeof(T)) && n <= kWidestRow; }

constexpr int kUnits = 256;                         // compute units
// Bytes of a call from which its accesses carry the streaming hint: half the last-level cache, from where on
// little of it is still there for whatever reads it next.  Backward of 201 MB 41.7 -> 37.6 us with the hint,
// of 67 MB 13.7 -> 14.4.
constexpr double kStreamed = 128.0 * (1 << 20);
constexpr int64_t kMostBlocks = int64_t{1} << 20;   // of kernels that walk the rest themselves

}  // namespace
}  // namespace grass
