// grass_norm_forward: layer norm and RMS norm.
//
// Bound by memory: X (and R) are read once and Y (and H) are written once.  A row stays in the registers of
// the threads that share it from its sums to its outputs; gain and bias stay there for all rows that a
// workgroup takes.  Measured: 131072 x 4096 bf16 with R 716 to 726 us (5.9 to 6.0 TB/s); one row of 4096 2.9 us.
#include <type_traits>

#include "elem.hpp"

namespace grass {
namespace {

struct ForwardArgs {
    const void *X, *R, *gain, *bias;
    void *H, *Y;
    int64_t ldx, ldr, ldh, ldy, T;
    int n;
    bool centre, gain_bf16;
    float eps;
    float *mean, *rstd;
};

// N values of gain or bias from column `at` on; `without` where there is none.
template <int N>
__device__ __forceinline__ void load_vector(const void* p, bool bf16, int at, float without, float (&g)[N]) {
    if (!p) {
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] = without;
    } else if (bf16) {
        Raw<uint16_t, N> r;
        r.load(static_cast<const uint16_t*>(p) + at);
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] = r.get(i);
    } else {
        Raw<float, N> r;
        r.load(static_cast<const float*>(p) + at);
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] = r.get(i);
    }
}

// What a thread holds of a row.  kWindow: rows of whole 16-byte vectors that start on 16 bytes, through
// windows; else rows in any position.
template <typename T, int TPR, int V, bool kWindow, bool kAdd, bool kOnce>
struct Row {
    static constexpr int N = 16 / sizeof(T);
    Raw<T, N> x[V], b[kAdd ? V : 1];
    __device__ __forceinline__ void load(const ForwardArgs& a, int64_t t, int lane, const Span (&at)[V]) {
        const uint32_t bytes = t < a.T ? static_cast<uint32_t>(a.n) * sizeof(T) : 0u;
        t = t < a.T ? t : a.T - 1;
        const T* x0 = static_cast<const T*>(a.X) + t * a.ldx;
        const T* r0 = static_cast<const T*>(a.R) + t * a.ldr;
        if constexpr (kWindow) {
            const RowWindow wx(x0, bytes);
#pragma unroll
            for (int v = 0; v < V; ++v) wx.template load<kOnce>(x[v].w, (v * TPR + lane) * 16);
            if constexpr (kAdd) {
                const RowWindow wb(r0, bytes);
#pragma unroll
                for (int v = 0; v < V; ++v) wb.template load<kOnce>(b[v].w, (v * TPR + lane) * 16);
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                x[v].template load_as<kOnce>(x0 + at[v].at);
                if constexpr (kAdd) b[v].template load_as<kOnce>(r0 + at[v].at);
            }
        }
    }
};

// A block's B / TPR row groups take rows from blockIdx on, gridDim apart.  While a thread works on its part
// of one row, its part of the next is on its way.
template <typename T, typename Shape, bool kWindow, bool kAdd, bool kOnce>
__global__ __launch_bounds__(Shape::B) void forward_kernel(ForwardArgs a) {
    constexpr int TPR = Shape::TPR, V = Shape::V, B = Shape::B, N = 16 / sizeof(T), kRows = B / TPR;
    typedef Row<T, TPR, V, kWindow, kAdd, kOnce> RowPart;
    __shared__ float red[2][B / kWave][1];
    RowSum<TPR, B, 1> row_sum{red};
    const int l = threadIdx.x % TPR;
    const int group = TPR >= kWave ? __builtin_amdgcn_readfirstlane(threadIdx.x / TPR) : threadIdx.x / TPR;
    const float n = static_cast<float>(a.n);
    const int64_t step = static_cast<int64_t>(gridDim.x) * kRows;
    int64_t t0 = static_cast<int64_t>(blockIdx.x) * kRows;
    Span at[V];
#pragma unroll
    for (int v = 0; v < V; ++v) at[v] = span<TPR, Shape::kFull, N>(v, l, a.n);
    RowPart even, odd;
    even.load(a, t0 + group, l, at);
    float gain[V][N], bias[V][N];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        load_vector<N>(a.gain, a.gain_bf16, at[v].at, 1.f, gain[v]);
        load_vector<N>(a.bias, a.gain_bf16, at[v].at, 0.f, bias[v]);
    }
    const auto work = [&](RowPart& row, int64_t t) {
        const bool there = kRows == 1 || t < a.T;
        if constexpr (kAdd) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float s[N];
#pragma unroll
                for (int i = 0; i < N; ++i) s[i] = row.x[v].get(i) + row.b[v].get(i);
                row.x[v].set(s);
            }
        }
        float mean = 0.f;
        if (a.centre) {
            float s[1] = {0.f};
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < N; ++i) s[0] += kWindow || i >= at[v].skip ? row.x[v].get(i) : 0.f;
            row_sum(s);
            mean = s[0] / n;
        }
        float q[1] = {0.f};
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float d = i >= at[v].skip ? row.x[v].get(i) - mean : 0.f;
                q[0] += d * d;
            }
        // (behind row_sum all threads of the row have what they read of it, so that H and Y may lie over it)
        row_sum(q);
        const float rstd = 1.0f / sqrtf(q[0] / n + a.eps);
        if (there && l == 0) {
            if (a.centre && a.mean) a.mean[t] = mean;
            if (a.rstd) a.rstd[t] = rstd;
        }
        T* h = static_cast<T*>(a.H) + t * a.ldh;
        T* y = static_cast<T*>(a.Y) + t * a.ldy;
        const uint32_t bytes = there ? static_cast<uint32_t>(a.n) * sizeof(T) : 0u;
        const RowWindow wh(h, bytes), wy(y, bytes);
        if (!kWindow && !there) return;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if constexpr (kAdd) {
                if constexpr (kWindow) wh.template store<kOnce>(row.x[v].w, (v * TPR + l) * 16);
                else row.x[v].template store_as<kOnce>(h + at[v].at);
            }
            float o[N];
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] = (row.x[v].get(i) - mean) * rstd * gain[v][i] + bias[v][i];
            Raw<T, N> out;
            out.set(o);
            if constexpr (kWindow) wy.template store<kOnce>(out.w, (v * TPR + l) * 16);
            else out.template store_as<kOnce>(y + at[v].at);
        }
    };
    // (the same number of turns for every thread: they meet at the barriers of row_sum)
    for (;; t0 += 2 * step) {
        odd.load(a, t0 + step + group, l, at);
        work(even, t0 + group);
        if (t0 + step >= a.T) break;
        even.load(a, t0 + 2 * step + group, l, at);
        work(odd, t0 + step + group);
        if (t0 + 2 * step >= a.T) break;
    }
}

constexpr int kWide = 256;  // threads of the kernel for rows of any width

// Rows of any width, one per block at a time: the sum, the squares about the mean and the outputs are a pass
// each over the row (over H, where there is a residual branch: every thread reads what it wrote).
template <typename T>
__global__ __launch_bounds__(kWide) void forward_wide_kernel(ForwardArgs a) {
    __shared__ float red[2][kWide / kWave][1];
    RowSum<kWide, kWide, 1> row_sum{red};
    const int n = a.n;
    const auto load = [&](Raw<T, 8>& u, const T* p, int left) {
        if (left == 8) u.load(p);
        else u.load_some(p, left);
    };
    const auto store = [&](const Raw<T, 8>& u, T* p, int left) {
        if (left == 8) u.store(p);
        else u.store_some(p, left);
    };
    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        const T* x = static_cast<const T*>(a.X) + t * a.ldx;
        const T* h = a.R ? static_cast<const T*>(a.H) + t * a.ldh : x;
        float s[1] = {0.f};
        if (a.centre || a.R)
            for (int64_t c = threadIdx.x * 8; c < n; c += kWide * 8) {
                const int left = static_cast<int>(n - c < 8 ? n - c : 8);
                Raw<T, 8> u;
                load(u, x + c, left);
                if (a.R) {
                    Raw<T, 8> b;
                    load(b, static_cast<const T*>(a.R) + t * a.ldr + c, left);
                    float z[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) z[i] = u.get(i) + b.get(i);
                    u.set(z);
                    store(u, static_cast<T*>(a.H) + t * a.ldh + c, left);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) s[0] += u.get(i);
            }
        float mean = 0.f;
        if (a.centre) {
            row_sum(s);
            mean = s[0] / static_cast<float>(n);
        }
        float q[1] = {0.f};
        for (int64_t c = threadIdx.x * 8; c < n; c += kWide * 8) {
            const int left = static_cast<int>(n - c < 8 ? n - c : 8);
            Raw<T, 8> u;
            load(u, h + c, left);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) {
                    const float d = u.get(i) - mean;
                    q[0] += d * d;
                }
        }
        row_sum(q);
        const float rstd = 1.0f / sqrtf(q[0] / static_cast<float>(n) + a.eps);
        if (threadIdx.x == 0) {
            if (a.centre && a.mean) a.mean[t] = mean;
            if (a.rstd) a.rstd[t] = rstd;
        }
        for (int64_t c = threadIdx.x * 8; c < n; c += kWide * 8) {
            const int left = static_cast<int>(n - c < 8 ? n - c : 8);
            Raw<T, 8> u;
            load(u, h + c, left);
            float g[8], b[8], o[8];
            if (left == 8) {
                load_vector<8>(a.gain, a.gain_bf16, static_cast<int>(c), 1.f, g);
                load_vector<8>(a.bias, a.gain_bf16, static_cast<int>(c), 0.f, b);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const auto value = [&](const void* p, float without) {
                        if (!p || i >= left) return without;
                        return a.gain_bf16 ? bf16_to_f32(static_cast<const uint16_t*>(p)[c + i]) : static_cast<const float*>(p)[c + i];
                    };
                    g[i] = value(a.gain, 1.f);
                    b[i] = value(a.bias, 0.f);
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = (u.get(i) - mean) * rstd * g[i] + b[i];
            u.set(o);
            store(u, static_cast<T*>(a.Y) + t * a.ldy + c, left);
        }
    }
}

// Blocks for so many groups of rows.  Short of kStreamed bytes two per compute unit, which walk the rest; from there
// on as many as take so many turns, 16 in whole multiples of that (a few blocks beyond them would be a round of their own).
int64_t forward_blocks(int64_t groups, bool once, int turns) {
    const int64_t some = 2 * kUnits;
    if (groups < some || !once) return groups < some ? groups : some;
    const int64_t more = turns < 16 ? groups / turns : groups / (16 * some) * some;
    return more > some ? more : some;
}

// Turns of a block where the call streams: few where what it starts with (gain, bias, the first row's way) is small against a
// turn.  TB/s at 1.2 GB with 2, 4 and 16 turns.  fp32: 512 values 5.98 5.94 5.59, 4096 6.18 6.05 6.01, 3001 5.42 5.41 5.13,
// with R 512 5.96 5.74 5.56.  bf16 with R: 512 5.98 5.68 5.30, 4096 6.02 5.76 5.88, 200 5.51 5.29 4.65, 500 (no window) 5.22 4.91 4.37,
// 2601 (no window) 3.99 4.33 4.97.  bf16 without: 512 5.83 6.11 5.38, 2048 6.11 6.08 5.83, 200 4.98 5.33 4.97, 501 5.02 5.16 4.54,
// 2601 3.74 4.09 4.76, 2200 (three vectors) 4.17 4.69 5.27; 64, which half of a row's lanes have no part of, 3.48 3.90 4.34 (80, with
// five eighths at work, 4.21 4.44 3.99 at 180 MB and 4.16 4.75 4.94).
template <typename T, typename S>
int forward_turns(int64_t n, bool add, bool window) {
    if (sizeof(T) == 4) return 2;
    const bool two = S::V <= 2;
    if (add) return window || (two && S::TPR <= kWave) ? 2 : 16;
    if (two && window && S::TPR >= kWave && S::TPR <= 2 * kWave) return 2;  // (shorter rows take no windows)
    return two && S::TPR <= kWave && n * sizeof(T) * 8 >= S::TPR * S::V * 16 * 5 ? 4 : 16;
}

// Three vectors a thread put more rows into a workgroup.  With R, two / three us: rows of 64 lanes 2320 x 1293 bf16 8.8 / 9.9,
// 6050 x 1033 14.5 / 12.5, so from two workgroups per compute unit (`many`) on; wider ones 3038 x 2057 14.5 / 15.0, 1249 x 5001
// 12.7 / 13.6, 60768 x 2057 242 / 222, 24995 x 5001 233 / 199, so where the call streams.  Without R at any number of rows: 5808 x 1033
// 9.6 / 8.1, 242013 x 1033 258 / 204, 12019 x 520 fp32 11.6 / 8.6; rows of 128 and 256 lanes win and lose a tenth by how many turns are left.
constexpr bool three_vectors(int tpr, bool add, bool streamed, bool many) {
    return !add || (tpr == 64 ? many : streamed);
}

template <typename T>
void launch(const ForwardArgs& a, hipStream_t s) {
    if (!in_registers<T>(a.n)) {
        forward_wide_kernel<T><<<static_cast<unsigned>(a.T < kMostBlocks ? a.T : kMostBlocks), kWide, 0, s>>>(a);
        return;
    }
    const auto on16 = [](const void* p, int64_t ld) { return aligned_to(p, 16) && ld * sizeof(T) % 16 == 0; };
    const bool window = a.n * sizeof(T) % 16 == 0 && on16(a.X, a.ldx) && on16(a.Y, a.ldy) &&
                        (!a.R || (on16(a.R, a.ldr) && on16(a.H, a.ldh)));
    const bool once = static_cast<double>(a.T) * a.n * sizeof(T) * (a.R ? 4 : 2) > kStreamed;
    const auto three = [&](int tpr) { return three_vectors(tpr, a.R != nullptr, once, a.T >= 2 * kUnits * (512 / tpr)); };
    by_shape<T>(a.n, three, [&](auto shape) {
        typedef decltype(shape) S;
        constexpr int64_t kRows = S::B / S::TPR;
        // (a grid has fewer than 2^32 threads)
        const int64_t blocks = forward_blocks((a.T + kRows - 1) / kRows, once, forward_turns<T, S>(a.n, a.R != nullptr, window));
        const unsigned grid = static_cast<unsigned>(blocks < kMostBlocks ? blocks : kMostBlocks);
        const auto go = [&](auto win, auto add, auto stream) {
            constexpr bool kAdd = decltype(add)::value, kOnce = decltype(stream)::value;
            // (kernels that the rule leaves without calls are not built)
            if constexpr (S::V != 3 || S::TPR == 512 || three_vectors(S::TPR, kAdd, kOnce, true))
                forward_kernel<T, S, decltype(win)::value, kAdd, kOnce><<<grid, S::B, 0, s>>>(a);
        };
        const auto with_add = [&](auto win, auto add) { once ? go(win, add, std::true_type{}) : go(win, add, std::false_type{}); };
        const auto with_window = [&](auto win) { a.R ? with_add(win, std::true_type{}) : with_add(win, std::false_type{}); };
        if constexpr (S::TPR >= kWave)
            if (window) return with_window(std::true_type{});
        with_window(std::false_type{});
    });
}

}  // namespace

grass_status launch_norm_forward(grass_norm kind, const void* X, int64_t ldx, const void* R, int64_t ldr,
                                 grass_dtype dt, int64_t T, int64_t n, const void* gain, const void* bias,
                                 grass_dtype gdt, float eps, void* H, int64_t ldh, void* Y, int64_t ldy,
                                 float* mean, float* rstd, hipStream_t s) {
    if (T == 0) return GRASS_OK;
    const ForwardArgs a{X, R, gain, bias, H, Y, ldx, ldr, ldh, ldy, T, static_cast<int>(n),
                        kind == GRASS_NORM_LAYER, gdt == GRASS_BF16, eps, mean, rstd};
    dt == GRASS_F32 ? launch<float>(a, s) : launch<uint16_t>(a, s);
    return launch_status();
}

}  // namespace grass
