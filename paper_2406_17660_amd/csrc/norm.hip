// grass_norm_forward, grass_norm_backward: layer norm and RMS norm.
//
// Both directions are bound by memory: forward reads X (and R) once and writes Y (and H), backward
// reads dY and H (and dR) and writes dX.  A row of up to 16384 values stays in the registers of the
// lanes that own it (16 lanes to four wavefronts), so it is read once although its statistics are
// needed before its first output; wider rows are read once per pass.  Eight consecutive elements per
// lane and access, in any position.
#include <type_traits>

#include "elem8.hpp"

namespace grass {
namespace {

constexpr int kBlock = 256;
constexpr int kUnits = 256;  // compute units

// Sum over the TPR consecutive lanes that share a row; every one of them gets it.
template <int TPR>
__device__ __forceinline__ float sum_lanes(float v) {
    constexpr int W = TPR < kWave ? TPR : kWave;
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    return v;
}

// The same for N sums over a row that TPR > 64 threads share: wavefront sums meet in LDS, one barrier a
// call; `at` alternates between two places, so that a call does not overwrite what a slower wavefront
// still reads.  Every thread of the block must take part.
template <int TPR, int N>
struct RowSum {
    float (*part)[kBlock / kWave][N];
    int at = 0;
    __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = sum_lanes<TPR>(v[k]);
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

template <typename T>
struct Matrix {
    T* p;
    int64_t ld;
    __device__ __forceinline__ T* row(int64_t t) const { return p + t * ld; }
};

template <typename T>
__device__ __forceinline__ void load_part(Raw8<T>& x, const T* p, int left) {
    if (left >= 8) x.load(p);
    else if (left > 0) x.load_some(p, left);
    else x.zero();
}
template <typename T>
__device__ __forceinline__ void store_part(const Raw8<T>& x, T* p, int left) {
    if (left >= 8) x.store(p);
    else if (left > 0) x.store_some(p, left);
}

struct ForwardArgs {
    const void *X, *R, *gain, *bias;
    void *H, *Y;
    int64_t ldx, ldr, ldh, ldy, T;
    int n;
    float eps;
    float *mean, *rstd;
};

// One row per TPR threads, V vectors of eight each.
template <typename T, typename G, bool kCentre, int TPR, int V>
__global__ __launch_bounds__(kBlock) void forward_kernel(ForwardArgs a) {
    __shared__ float part[2][kBlock / kWave][1];
    RowSum<TPR, 1> row_sum{part};
    const int l = threadIdx.x % TPR;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * (kBlock / TPR) + threadIdx.x / TPR;
    const bool there = t < a.T;
    const int n = there ? a.n : 0;
    const T* x = static_cast<const T*>(a.X) + t * a.ldx;
    Raw8<T> raw[V];
#pragma unroll
    for (int v = 0; v < V; ++v) load_part(raw[v], x + (v * TPR + l) * 8, n - (v * TPR + l) * 8);
    if (a.R) {
        const T* r = static_cast<const T*>(a.R) + t * a.ldr;
        T* h = static_cast<T*>(a.H) + t * a.ldh;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            Raw8<T> b;
            load_part(b, r + (v * TPR + l) * 8, n - (v * TPR + l) * 8);
            float s[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] = raw[v].get(i) + b.get(i);
            raw[v].set(s);
            store_part(raw[v], h + (v * TPR + l) * 8, n - (v * TPR + l) * 8);
        }
    }
    float mean = 0.f;
    if constexpr (kCentre) {
        float s[1] = {0.f};
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) s[0] += raw[v].get(i);
        row_sum(s);
        mean = s[0] / static_cast<float>(a.n);
    }
    float q[1] = {0.f};
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float d = raw[v].get(i) - mean;
            if (kCentre && (v * TPR + l) * 8 + i >= n) d = 0.f;
            q[0] += d * d;
        }
    row_sum(q);
    const float rstd = 1.0f / sqrtf(q[0] / static_cast<float>(a.n) + a.eps);
    if (there && l == 0) {
        if (kCentre && a.mean) a.mean[t] = mean;
        if (a.rstd) a.rstd[t] = rstd;
    }
    T* y = static_cast<T*>(a.Y) + t * a.ldy;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int c = (v * TPR + l) * 8;
        if (c >= n) continue;
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = (raw[v].get(i) - mean) * rstd;
        Raw8<G> w;
        if (a.gain) {
            load_part(w, static_cast<const G*>(a.gain) + c, n - c);
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] *= w.get(i);
        }
        if (a.bias) {
            load_part(w, static_cast<const G*>(a.bias) + c, n - c);
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] += w.get(i);
        }
        raw[v].set(o);
        store_part(raw[v], y + c, n - c);
    }
}

// Rows of any width, one per block: the sum, the squares about the mean and the outputs are a pass
// each over the row (over H, where there is a residual branch: every lane reads what it wrote).
template <typename T, typename G, bool kCentre>
__global__ __launch_bounds__(kBlock) void forward_wide_kernel(ForwardArgs a) {
    __shared__ float part[2][kBlock / kWave][1];
    RowSum<kBlock, 1> row_sum{part};
    const int64_t t = blockIdx.x;
    const int n = a.n;
    const T* x = static_cast<const T*>(a.X) + t * a.ldx;
    const T* h = a.R ? static_cast<const T*>(a.H) + t * a.ldh : x;
    float s[1] = {0.f};
    if (kCentre || a.R)
        for (int64_t c = threadIdx.x * 8; c < n; c += kBlock * 8) {
            const int left = static_cast<int>(n - c < 8 ? n - c : 8);
            Raw8<T> u;
            load_part(u, x + c, left);
            if (a.R) {
                Raw8<T> b;
                load_part(b, static_cast<const T*>(a.R) + t * a.ldr + c, left);
                float z[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) z[i] = u.get(i) + b.get(i);
                u.set(z);
                store_part(u, static_cast<T*>(a.H) + t * a.ldh + c, left);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) s[0] += u.get(i);
        }
    float mean = 0.f;
    if constexpr (kCentre) {
        row_sum(s);
        mean = s[0] / static_cast<float>(n);
    }
    float q[1] = {0.f};
    for (int64_t c = threadIdx.x * 8; c < n; c += kBlock * 8) {
        const int left = static_cast<int>(n - c < 8 ? n - c : 8);
        Raw8<T> u;
        load_part(u, h + c, left);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) {
                const float d = u.get(i) - mean;
                q[0] += d * d;
            }
    }
    row_sum(q);
    const float rstd = 1.0f / sqrtf(q[0] / static_cast<float>(a.n) + a.eps);
    if (threadIdx.x == 0) {
        if (kCentre && a.mean) a.mean[t] = mean;
        if (a.rstd) a.rstd[t] = rstd;
    }
    for (int64_t c = threadIdx.x * 8; c < n; c += kBlock * 8) {
        const int left = static_cast<int>(n - c < 8 ? n - c : 8);
        Raw8<T> u;
        load_part(u, h + c, left);
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = (u.get(i) - mean) * rstd;
        Raw8<G> w;
        if (a.gain) {
            load_part(w, static_cast<const G*>(a.gain) + c, left);
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] *= w.get(i);
        }
        if (a.bias) {
            load_part(w, static_cast<const G*>(a.bias) + c, left);
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] += w.get(i);
        }
        u.set(o);
        store_part(u, static_cast<T*>(a.Y) + t * a.ldy + c, left);
    }
}

struct BackwardArgs {
    const void *dY, *H, *dR, *gain;
    void* dX;
    int64_t lddy, ldh, lddr, lddx, T;
    int n;
    const float *mean, *rstd;
    float* part;  // [gridDim.x][2][n]: sums of dY * xh and of dY over a block's rows, or nullptr
    bool want_bias;
};

// A block's row groups (TPR threads each) take rows blockIdx, blockIdx + gridDim, ...; a thread keeps
// the sums of its own 8 * V columns in registers over all of them.
template <typename T, typename G, bool kCentre, int TPR, int V>
__global__ __launch_bounds__(kBlock) void backward_kernel(BackwardArgs a) {
    constexpr int kRows = kBlock / TPR;
    __shared__ float red[2][kBlock / kWave][2];
    __shared__ float sums[kBlock * 8];
    RowSum<TPR, 2> row_sum{red};
    const int l = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const float inv_n = 1.0f / static_cast<float>(a.n);
    Raw8<G> gain[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (a.gain) {
            load_part(gain[v], static_cast<const G*>(a.gain) + (v * TPR + l) * 8, a.n - (v * TPR + l) * 8);
        } else {
            const float ones[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
            gain[v].set(ones);
        }
    }
    float dgain[V][8], dbias[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) dgain[v][i] = dbias[v][i] = 0.f;
    // (the same number of turns for every thread: they meet at the barriers of row_sum)
    for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * kRows; t0 < a.T; t0 += static_cast<int64_t>(gridDim.x) * kRows) {
        const int64_t t = t0 + group;
        const bool there = t < a.T;
        const int n = there ? a.n : 0;
        const T* dy = static_cast<const T*>(a.dY) + t * a.lddy;
        const T* h = static_cast<const T*>(a.H) + t * a.ldh;
        Raw8<T> y[V], x[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            load_part(y[v], dy + (v * TPR + l) * 8, n - (v * TPR + l) * 8);
            load_part(x[v], h + (v * TPR + l) * 8, n - (v * TPR + l) * 8);
        }
        const float mean = kCentre && there ? a.mean[t] : 0.f;
        const float rstd = there ? a.rstd[t] : 0.f;
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int v = 0; v < V; ++v)
            if ((v * TPR + l) * 8 < n) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float d = y[v].get(i), xh = (x[v].get(i) - mean) * rstd, z = d * gain[v].get(i);
                    s[0] += z * xh;
                    if (kCentre) s[1] += z;
                    dgain[v][i] += d * xh;
                    dbias[v][i] += d;
                }
            }
        row_sum(s);
        const float c0 = s[0] * inv_n, c1 = s[1] * inv_n;
        T* dx = static_cast<T*>(a.dX) + t * a.lddx;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = (v * TPR + l) * 8;
            if (c >= n) continue;
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float xh = (x[v].get(i) - mean) * rstd, z = y[v].get(i) * gain[v].get(i);
                o[i] = rstd * (kCentre ? z - c1 - xh * c0 : z - xh * c0);
            }
            if (a.dR) {
                Raw8<T> b;
                load_part(b, static_cast<const T*>(a.dR) + t * a.lddr + c, n - c);
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] += b.get(i);
            }
            x[v].set(o);
            store_part(x[v], dx + c, n - c);
        }
    }
    if (!a.part) return;
    float* part = a.part + static_cast<int64_t>(blockIdx.x) * 2 * a.n;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        if (q == 1 && !a.want_bias) break;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) sums[(group * TPR + l) * 8 + i] = q ? dbias[v][i] : dgain[v][i];
            __syncthreads();
            for (int c = threadIdx.x; c < TPR * 8; c += kBlock) {
                float s = sums[c];
#pragma unroll
                for (int r = 1; r < kRows; ++r) s += sums[r * TPR * 8 + c];
                if (v * TPR * 8 + c < a.n) part[static_cast<int64_t>(q) * a.n + v * TPR * 8 + c] = s;
            }
        }
    }
}

// Rows of any width.  First the columns' sums (a block: 2048 columns of every gridDim.y-th row) ...
template <typename T>
__global__ __launch_bounds__(kBlock) void backward_wide_sums_kernel(BackwardArgs a, bool centre) {
    const int64_t c = (static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x) * 8;
    if (c >= a.n) return;
    const int left = static_cast<int>(a.n - c < 8 ? a.n - c : 8);
    float dgain[8] = {}, dbias[8] = {};
    for (int64_t t = blockIdx.y; t < a.T; t += gridDim.y) {
        Raw8<T> y, x;
        load_part(y, static_cast<const T*>(a.dY) + t * a.lddy + c, left);
        load_part(x, static_cast<const T*>(a.H) + t * a.ldh + c, left);
        const float mean = centre ? a.mean[t] : 0.f, rstd = a.rstd[t];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            dgain[i] += y.get(i) * ((x.get(i) - mean) * rstd);
            dbias[i] += y.get(i);
        }
    }
    float* part = a.part + static_cast<int64_t>(blockIdx.y) * 2 * a.n + c;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) {
            part[i] = dgain[i];
            if (a.want_bias) part[a.n + i] = dbias[i];
        }
}

// ... then dX, a row per block and a pass over it for each of the sums and the outputs.
template <typename T, typename G, bool kCentre>
__global__ __launch_bounds__(kBlock) void backward_wide_kernel(BackwardArgs a) {
    __shared__ float red[2][kBlock / kWave][2];
    RowSum<kBlock, 2> row_sum{red};
    const int64_t t = blockIdx.x;
    const float mean = kCentre ? a.mean[t] : 0.f, rstd = a.rstd[t];
    const float inv_n = 1.0f / static_cast<float>(a.n);
    float s[2] = {0.f, 0.f};
    float c0 = 0.f, c1 = 0.f;
    for (int pass = 0; pass < 2; ++pass) {
        for (int64_t c = threadIdx.x * 8; c < a.n; c += kBlock * 8) {
            const int left = static_cast<int>(a.n - c < 8 ? a.n - c : 8);
            Raw8<T> y, x;
            Raw8<G> w;
            load_part(y, static_cast<const T*>(a.dY) + t * a.lddy + c, left);
            load_part(x, static_cast<const T*>(a.H) + t * a.ldh + c, left);
            if (a.gain) load_part(w, static_cast<const G*>(a.gain) + c, left);
            Raw8<T> b;
            b.zero();
            if (pass && a.dR) load_part(b, static_cast<const T*>(a.dR) + t * a.lddr + c, left);
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float xh = (x.get(i) - mean) * rstd, z = y.get(i) * (a.gain ? w.get(i) : 1.f);
                if (!pass && i < left) {
                    s[0] += z * xh;
                    if (kCentre) s[1] += z;
                }
                o[i] = rstd * (kCentre ? z - c1 - xh * c0 : z - xh * c0) + b.get(i);
            }
            if (pass) {
                x.set(o);
                store_part(x, static_cast<T*>(a.dX) + t * a.lddx + c, left);
            }
        }
        if (!pass) {
            row_sum(s);
            c0 = s[0] * inv_n;
            c1 = s[1] * inv_n;
        }
    }
}

// dgain and dbias from the blocks' sums (64 columns per block, its four wavefronts take every fourth
// of the P rows).  P = 0 writes zeros.
__global__ __launch_bounds__(kBlock) void column_sums_kernel(const float* __restrict__ part, int P, int n,
                                                             float* dgain, float* dbias) {
    __shared__ float sums[kBlock / kWave][kWave];
    float* out = blockIdx.y ? dbias : dgain;
    if (!out) return;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * kWave + lane;
    float s = 0.f;
    if (c < n) {
        const float* p = part + static_cast<int64_t>(blockIdx.y) * n + c;
#pragma unroll 8
        for (int k = wave; k < P; k += kBlock / kWave) s += p[static_cast<int64_t>(k) * 2 * n];
    }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < n) out[c] = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
}

constexpr int kWidest = 16384;  // widest row that stays in registers

// Threads that share a row and vectors of eight per thread, for rows of n values.
struct Shape {
    int tpr, v;
};
Shape shape_for(int64_t n) {
    const int64_t vectors = (n + 7) / 8;
    if (vectors <= 16) return {16, 1};
    if (vectors <= 64) return {64, 1};
    if (vectors <= 128) return {64, 2};
    if (vectors <= 256) return {64, 4};
    if (vectors <= 512) return {256, 2};
    if (vectors <= 1024) return {256, 4};
    return {256, 8};
}

template <typename T, typename G, bool kCentre>
void forward_launch(const ForwardArgs& a, hipStream_t s) {
    if (a.n > kWidest) {
        forward_wide_kernel<T, G, kCentre><<<static_cast<unsigned>(a.T), kBlock, 0, s>>>(a);
        return;
    }
    const Shape f = shape_for(a.n);
    const int rows = kBlock / f.tpr;
    const unsigned grid = static_cast<unsigned>((a.T + rows - 1) / rows);
    if (f.tpr == 16) forward_kernel<T, G, kCentre, 16, 1><<<grid, kBlock, 0, s>>>(a);
    else if (f.tpr == 64 && f.v == 1) forward_kernel<T, G, kCentre, 64, 1><<<grid, kBlock, 0, s>>>(a);
    else if (f.tpr == 64 && f.v == 2) forward_kernel<T, G, kCentre, 64, 2><<<grid, kBlock, 0, s>>>(a);
    else if (f.tpr == 64) forward_kernel<T, G, kCentre, 64, 4><<<grid, kBlock, 0, s>>>(a);
    else if (f.v == 2) forward_kernel<T, G, kCentre, 256, 2><<<grid, kBlock, 0, s>>>(a);
    else if (f.v == 4) forward_kernel<T, G, kCentre, 256, 4><<<grid, kBlock, 0, s>>>(a);
    else forward_kernel<T, G, kCentre, 256, 8><<<grid, kBlock, 0, s>>>(a);
}

// Blocks of the backward pass, each of which leaves one row of column sums.
int backward_blocks(int64_t T, int64_t n) {
    const int rows = n > kWidest ? 1 : kBlock / shape_for(n).tpr;
    const int64_t want = (T + rows - 1) / rows;
    return static_cast<int>(want < 4 * kUnits ? want : 4 * kUnits);
}

template <typename T, typename G, bool kCentre>
void backward_launch(const BackwardArgs& a, hipStream_t s) {
    const unsigned grid = static_cast<unsigned>(backward_blocks(a.T, a.n));
    if (a.n > kWidest) {
        if (a.part) {
            const dim3 g(static_cast<unsigned>((a.n + int64_t{kBlock} * 8 - 1) / (kBlock * 8)), grid);
            backward_wide_sums_kernel<T><<<g, kBlock, 0, s>>>(a, kCentre);
        }
        backward_wide_kernel<T, G, kCentre><<<static_cast<unsigned>(a.T), kBlock, 0, s>>>(a);
        return;
    }
    const Shape f = shape_for(a.n);
    if (f.tpr == 16) backward_kernel<T, G, kCentre, 16, 1><<<grid, kBlock, 0, s>>>(a);
    else if (f.tpr == 64 && f.v == 1) backward_kernel<T, G, kCentre, 64, 1><<<grid, kBlock, 0, s>>>(a);
    else if (f.tpr == 64 && f.v == 2) backward_kernel<T, G, kCentre, 64, 2><<<grid, kBlock, 0, s>>>(a);
    else if (f.tpr == 64) backward_kernel<T, G, kCentre, 64, 4><<<grid, kBlock, 0, s>>>(a);
    else if (f.v == 2) backward_kernel<T, G, kCentre, 256, 2><<<grid, kBlock, 0, s>>>(a);
    else if (f.v == 4) backward_kernel<T, G, kCentre, 256, 4><<<grid, kBlock, 0, s>>>(a);
    else backward_kernel<T, G, kCentre, 256, 8><<<grid, kBlock, 0, s>>>(a);
}

// The kernel for a combination of types, by one call with the types' tags.
template <typename F>
void by_types(grass_dtype dt, grass_dtype gdt, grass_norm kind, F&& f) {
    const auto with_kind = [&](auto t, auto g) {
        kind == GRASS_NORM_LAYER ? f(t, g, std::true_type{}) : f(t, g, std::false_type{});
    };
    const auto with_gain = [&](auto t) { gdt == GRASS_F32 ? with_kind(t, float{}) : with_kind(t, uint16_t{}); };
    dt == GRASS_F32 ? with_gain(float{}) : with_gain(uint16_t{});
}

}  // namespace

grass_status launch_norm_forward(grass_norm kind, const void* X, int64_t ldx, const void* R, int64_t ldr,
                                 grass_dtype dt, int64_t T, int64_t n, const void* gain, const void* bias,
                                 grass_dtype gdt, float eps, void* H, int64_t ldh, void* Y, int64_t ldy,
                                 float* mean, float* rstd, hipStream_t s) {
    if (T == 0) return GRASS_OK;
    constexpr int64_t kMost = int64_t{1} << 22;  // rows of a launch: a grid has fewer than 2^32 threads
    const int64_t size = dt == GRASS_F32 ? 4 : 2;
    const auto rows_from = [&](const void* p, int64_t ld, int64_t t) {
        return p ? static_cast<const char*>(p) + t * ld * size : nullptr;
    };
    for (int64_t t0 = 0; t0 < T; t0 += kMost) {
        const ForwardArgs a{rows_from(X, ldx, t0), rows_from(R, ldr, t0), gain, bias,
                            const_cast<char*>(rows_from(H, ldh, t0)), const_cast<char*>(rows_from(Y, ldy, t0)),
                            ldx, ldr, ldh, ldy, T - t0 < kMost ? T - t0 : kMost, static_cast<int>(n), eps,
                            mean ? mean + t0 : nullptr, rstd ? rstd + t0 : nullptr};
        by_types(dt, gdt, kind, [&](auto t, auto g, auto centre) {
            forward_launch<decltype(t), decltype(g), decltype(centre)::value>(a, s);
        });
    }
    return launch_status();
}

size_t norm_backward_workspace_bytes(int64_t T, int64_t n) {
    return static_cast<size_t>(backward_blocks(T, n)) * 2 * n * sizeof(float);
}

grass_status launch_norm_backward(grass_norm kind, const void* dY, int64_t lddy, const void* H, int64_t ldh,
                                  const void* dR, int64_t lddr, grass_dtype dt, int64_t T, int64_t n,
                                  const void* gain, grass_dtype gdt, const float* mean, const float* rstd,
                                  void* dX, int64_t lddx, float* dgain, float* dbias, void* ws, hipStream_t s) {
    const bool sums = dgain || dbias;
    if (T == 0 && !sums) return GRASS_OK;
    if (T > 0) {
        const BackwardArgs a{dY, H, dR, gain, dX, lddy, ldh, lddr, lddx, T, static_cast<int>(n), mean, rstd,
                             sums ? static_cast<float*>(ws) : nullptr, dbias != nullptr};
        by_types(dt, gdt, kind, [&](auto t, auto g, auto centre) {
            backward_launch<decltype(t), decltype(g), decltype(centre)::value>(a, s);
        });
    }
    if (sums) {
        const dim3 grid(static_cast<unsigned>((n + kWave - 1) / kWave), 2);
        column_sums_kernel<<<grid, kBlock, 0, s>>>(static_cast<const float*>(ws), backward_blocks(T, n),
                                                   static_cast<int>(n), dgain, dbias);
    }
    return launch_status();
}

}  // namespace grass
