// grass_norm_backward: layer norm and RMS norm.
//
// Bound by memory: dY and H (and dR) are read once and dX is written once.  A row stays in the
// registers of the threads that share it between the two sums it needs and its outputs; the sums of
// dgain and dbias over the rows stay in the registers of the threads that own the columns, for all
// rows that a workgroup takes, and a second kernel adds the workgroups' sums.  Measured: 131072 x 4096 bf16 with
// dR 718 us (6.0 TB/s), 65536 x 512 bf16 37.6 us (5.4 TB/s with the second kernel), 2047 x 5461 bf16 20.5 us.
#include <type_traits>

#include "elem.hpp"

namespace grass {
namespace {

struct BackwardArgs {
    const void *dY, *H, *dR, *gain;
    void* dX;
    int64_t lddy, ldh, lddr, lddx, T;
    int n;
    bool centre, gain_bf16, want_bias;
    const float *mean, *rstd;
    float* part;  // [blocks][2][n]: sums of dY * xh and of dY over a block's rows, or nullptr
    unsigned column_blocks;  // the first blocks of the grid add up columns instead of taking rows
    float *dgain, *dbias;    // what they write
};

template <int N>
__device__ __forceinline__ void load_gain(const BackwardArgs& a, int at, float (&g)[N]) {
    if (!a.gain) {
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] = 1.f;
    } else if (a.gain_bf16) {
        Raw<uint16_t, N> r;
        r.load(static_cast<const uint16_t*>(a.gain) + at);
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] = r.get(i);
    } else {
        Raw<float, N> r;
        r.load(static_cast<const float*>(a.gain) + at);
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] = r.get(i);
    }
}

// What a thread holds of a row.  kWindow: rows of whole 16-byte vectors that start on 16 bytes, through
// windows; else rows in any position.
template <typename T, int TPR, int V, bool kWindow, bool kAdd, bool kOnce>
struct Row {
    static constexpr int N = 16 / sizeof(T);
    Raw<T, N> y[V], x[V], b[kAdd ? V : 1];
    float mean, rstd;
    __device__ __forceinline__ void load(const BackwardArgs& a, int64_t t, int lane, const Span (&at)[V]) {
        const uint32_t bytes = t < a.T ? static_cast<uint32_t>(a.n) * sizeof(T) : 0u;
        t = t < a.T ? t : a.T - 1;
        const T* dy = static_cast<const T*>(a.dY) + t * a.lddy;
        const T* h = static_cast<const T*>(a.H) + t * a.ldh;
        const T* dr = static_cast<const T*>(a.dR) + t * a.lddr;
        mean = (a.centre ? a.mean : a.rstd)[t];
        rstd = a.rstd[t];
        if constexpr (kWindow) {
            const RowWindow wy(dy, bytes), wx(h, bytes);
#pragma unroll
            for (int v = 0; v < V; ++v) wy.template load<kOnce>(y[v].w, (v * TPR + lane) * 16);
#pragma unroll
            for (int v = 0; v < V; ++v) wx.template load<kOnce>(x[v].w, (v * TPR + lane) * 16);
            if constexpr (kAdd) {
                const RowWindow wb(dr, bytes);
#pragma unroll
                for (int v = 0; v < V; ++v) wb.template load<kOnce>(b[v].w, (v * TPR + lane) * 16);
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                y[v].template load_as<kOnce>(dy + at[v].at);
                x[v].template load_as<kOnce>(h + at[v].at);
                if constexpr (kAdd) b[v].template load_as<kOnce>(dr + at[v].at);
            }
        }
    }
};

// Few rows: dgain and dbias of 16 vectors of columns, whole, by one block, whose groups of 16 lanes take
// rows in turn.  (That reads dY and H twice, and spares the second kernel and what goes between the two.)
constexpr int kColumnLanes = 16;
template <typename T, int B>
__device__ __forceinline__ void add_columns_up(const BackwardArgs& a, float* sums) {
    constexpr int N = 16 / sizeof(T), kColumns = kColumnLanes * N, kGroups = B / kColumnLanes;
    const int group = threadIdx.x / kColumnLanes, lane = threadIdx.x % kColumnLanes;
    const int64_t first = static_cast<int64_t>(blockIdx.x) * kColumns;
    // (the row's last piece may be shorter than a vector, which then starts before it)
    const Span at = span<kColumnLanes, 0, N>(0, lane, static_cast<int>(a.n - first < kColumns ? a.n - first : kColumns));
    const T* dy = static_cast<const T*>(a.dY) + first + at.at;
    const T* h = static_cast<const T*>(a.H) + first + at.at;
    float dgain[N] = {}, dbias[N] = {};
#pragma unroll 4
    for (int64_t t = group; t < a.T; t += kGroups) {
        Raw<T, N> y, x;
        y.load(dy + t * a.lddy);
        x.load(h + t * a.ldh);
        const float mean = a.centre ? a.mean[t] : 0.f, rstd = a.rstd[t];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            dgain[i] += y.get(i) * ((x.get(i) - mean) * rstd);
            dbias[i] += y.get(i);
        }
    }
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        float* out = q ? a.dbias : a.dgain;
        if (!out) continue;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i >= at.skip) sums[group * kColumns + lane * N + i - at.skip] = q ? dbias[i] : dgain[i];
        __syncthreads();
        for (int c = threadIdx.x; c < kColumns; c += B) {
            float s = sums[c];
#pragma unroll
            for (int g = 1; g < kGroups; ++g) s += sums[g * kColumns + c];
            if (first + c < a.n) out[first + c] = s;
        }
    }
}

// A block's B / TPR row groups take every so many-th row.  While a thread works on its part of one row, its
// part of the next is on its way.
template <typename T, typename Shape, bool kWindow, bool kAdd, bool kOnce>
__global__ __launch_bounds__(Shape::B) void backward_kernel(BackwardArgs a) {
    constexpr int TPR = Shape::TPR, V = Shape::V, B = Shape::B, N = 16 / sizeof(T), kRows = B / TPR;
    typedef Row<T, TPR, V, kWindow, kAdd, kOnce> RowPart;
    __shared__ float red[2][B / kWave][2];
    __shared__ float sums[B * N];
    if (blockIdx.x < a.column_blocks) return add_columns_up<T, B>(a, sums);
    const unsigned block = blockIdx.x - a.column_blocks, blocks = gridDim.x - a.column_blocks;
    RowSum<TPR, B, 2> row_sum{red};
    const int l = threadIdx.x % TPR;
    const int group = TPR >= kWave ? __builtin_amdgcn_readfirstlane(threadIdx.x / TPR) : threadIdx.x / TPR;
    const float inv_n = 1.0f / static_cast<float>(a.n);
    Span at[V];
    float gain[V][N], dgain[V][N], dbias[V][N];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        at[v] = span<TPR, Shape::kFull, N>(v, l, a.n);
        load_gain<N>(a, at[v].at, gain[v]);
#pragma unroll
        for (int i = 0; i < N; ++i) dgain[v][i] = dbias[v][i] = 0.f;
    }
    const int64_t step = static_cast<int64_t>(blocks) * kRows;
    int64_t t0 = static_cast<int64_t>(block) * kRows;
    const auto work = [&](RowPart& row, int64_t t) {
        const bool there = kRows == 1 || t < a.T;
        const float mean = a.centre ? row.mean : 0.f, rstd = row.rstd;
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int skip = there ? at[v].skip : N;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const bool own = kWindow || i >= skip;  // (behind a window's end there are zeros)
                const float d = own ? row.y[v].get(i) : 0.f;
                const float xh = own ? (row.x[v].get(i) - mean) * rstd : 0.f, z = d * gain[v][i];
                s[0] += z * xh;
                s[1] += z;
                dgain[v][i] += d * xh;
                dbias[v][i] += d;
            }
        }
        // Behind row_sum all threads of the row have what they read of it, so that dX may lie over it: dY and H,
        // which are in the sums, and dR, which is waited for here where two threads write the same elements.
        if constexpr (kAdd && !kWindow && TPR > kWave) {
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(row.b[v].w[i]));
        }
        row_sum(s);
        const float c0 = s[0] * inv_n, c1 = a.centre ? s[1] * inv_n : 0.f;
        T* dx = static_cast<T*>(a.dX) + t * a.lddx;
        const RowWindow window(dx, there ? static_cast<uint32_t>(a.n) * sizeof(T) : 0u);
        if (!kWindow && !there) return;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float o[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float xh = (row.x[v].get(i) - mean) * rstd;
                o[i] = rstd * (row.y[v].get(i) * gain[v][i] - c1 - xh * c0);
                if constexpr (kAdd) o[i] += row.b[v].get(i);
            }
            Raw<T, N> out;
            out.set(o);
            if constexpr (kWindow) window.template store<kOnce>(out.w, (v * TPR + l) * 16);
            else out.template store_as<kOnce>(dx + at[v].at);
        }
    };
    // (the same number of turns for every thread: they meet at the barriers of row_sum)
    if constexpr (V <= 3) {
        RowPart even, odd;
        even.load(a, t0 + group, l, at);
        for (;; t0 += 2 * step) {
            odd.load(a, t0 + step + group, l, at);
            work(even, t0 + group);
            if (t0 + step >= a.T) break;
            even.load(a, t0 + 2 * step + group, l, at);
            work(odd, t0 + step + group);
            if (t0 + 2 * step >= a.T) break;
        }
    } else {  // the widest rows: no registers for a second one, and enough of the first under way
        for (; t0 < a.T; t0 += step) {
            RowPart row;
            row.load(a, t0 + group, l, at);
            work(row, t0 + group);
        }
    }
    if (!a.part) return;
    float* part = a.part + static_cast<int64_t>(block) * 2 * a.n;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        if (q == 1 && !a.want_bias) break;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float(&own)[N] = q ? dbias[v] : dgain[v];
            const int skip = at[v].skip;
            if constexpr (kRows == 1) {  // the thread has seen all of the block's rows
                float* p = part + static_cast<int64_t>(q) * a.n + at[v].at;
                Raw<float, N> r;
                r.set(own);
                if (skip == 0) r.store(p);
                else
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        if (i >= skip) p[i] = own[i];
            } else {
                __syncthreads();
                // a column's sums stand where its own thread's element would without the shift at the row's end
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (kWindow || i >= skip) sums[(group * TPR + l) * N + i - (kWindow ? 0 : skip)] = own[i];
                __syncthreads();
                for (int c = threadIdx.x; c < TPR * N; c += B) {
                    float s = sums[c];
#pragma unroll
                    for (int r = 1; r < kRows; ++r) s += sums[r * TPR * N + c];
                    if (v * TPR * N + c < a.n) part[static_cast<int64_t>(q) * a.n + v * TPR * N + c] = s;
                }
            }
        }
    }
}

constexpr int kWide = 256;  // threads of the kernels for rows of any width

// Rows of any width.  First the columns' sums (a block: 2048 columns of every gridDim.y-th row) ...
template <typename T>
__global__ __launch_bounds__(kWide) void backward_wide_sums_kernel(BackwardArgs a) {
    const int64_t c = (static_cast<int64_t>(blockIdx.x) * kWide + threadIdx.x) * 8;
    if (c >= a.n) return;
    const int left = static_cast<int>(a.n - c < 8 ? a.n - c : 8);
    float dgain[8] = {}, dbias[8] = {};
    for (int64_t t = blockIdx.y; t < a.T; t += gridDim.y) {
        Raw<T, 8> y, x;
        const T *dy = static_cast<const T*>(a.dY) + t * a.lddy + c, *h = static_cast<const T*>(a.H) + t * a.ldh + c;
        if (left == 8) {
            y.load(dy);
            x.load(h);
        } else {
            y.load_some(dy, left);
            x.load_some(h, left);
        }
        const float mean = a.centre ? a.mean[t] : 0.f, rstd = a.rstd[t];
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

// ... then dX, a row per block at a time and a pass over it for each of the sums and the outputs.
template <typename T>
__global__ __launch_bounds__(kWide) void backward_wide_kernel(BackwardArgs a) {
    __shared__ float red[2][kWide / kWave][2];
    RowSum<kWide, kWide, 2> row_sum{red};
    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        const float mean = a.centre ? a.mean[t] : 0.f, rstd = a.rstd[t];
        float s[2] = {0.f, 0.f};
        float c0 = 0.f, c1 = 0.f;
        for (int pass = 0; pass < 2; ++pass) {
            for (int64_t c = threadIdx.x * 8; c < a.n; c += kWide * 8) {
                const int left = static_cast<int>(a.n - c < 8 ? a.n - c : 8);
                const T *dy = static_cast<const T*>(a.dY) + t * a.lddy + c, *h = static_cast<const T*>(a.H) + t * a.ldh + c;
                const T* dr = static_cast<const T*>(a.dR) + t * a.lddr + c;
                const bool add = pass && a.dR;
                Raw<T, 8> y, x, b;
                b.zero();
                float g[8];
                if (left == 8) {
                    y.load(dy);
                    x.load(h);
                    if (add) b.load(dr);
                    load_gain<8>(a, static_cast<int>(c), g);
                } else {
                    y.load_some(dy, left);
                    x.load_some(h, left);
                    if (add) b.load_some(dr, left);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        g[i] = 1.f;
                        if (a.gain && i < left)
                            g[i] = a.gain_bf16 ? bf16_to_f32(static_cast<const uint16_t*>(a.gain)[c + i])
                                               : static_cast<const float*>(a.gain)[c + i];
                    }
                }
                float o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float xh = (x.get(i) - mean) * rstd, z = y.get(i) * g[i];
                    if (!pass && i < left) {
                        s[0] += z * xh;
                        s[1] += z;
                    }
                    o[i] = rstd * (z - c1 - xh * c0) + b.get(i);
                }
                if (!pass) continue;
                x.set(o);
                T* dx = static_cast<T*>(a.dX) + t * a.lddx + c;
                if (left == 8) x.store(dx);
                else x.store_some(dx, left);
            }
            if (pass) break;
            row_sum(s);
            c0 = s[0] / static_cast<float>(a.n);
            c1 = a.centre ? s[1] / static_cast<float>(a.n) : 0.f;
        }
    }
}

// dgain and dbias from the P blocks' sums.  A block: 64 columns, of those from `first` on; its sixteen wavefronts
// take every sixteenth row each, all of them under way at once, however many there are (a loop over P asked for
// them one by one where P was not 256: 2000 x 500 bf16 10.8 us with both kernels, so 7.3).  P = 0 writes zeros.
constexpr int kSumWaves = 16, kSumRows = kUnits / kSumWaves;
constexpr int64_t kMostColumns = int64_t{1} << 27;  // of one launch
__global__ __launch_bounds__(kSumWaves* kWave) void column_sums_kernel(const float* __restrict__ part, int P, int n,
                                                                       int first, float* dgain, float* dbias) {
    __shared__ float sums[kSumWaves][kWave];
    float* out = blockIdx.y ? dbias : dgain;
    if (!out) return;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int64_t c = first + static_cast<int64_t>(blockIdx.x) * kWave + lane;
    float s = 0.f;
    if (c < n) {
        const float* p = part + static_cast<int64_t>(blockIdx.y) * n + c;
        float x[kSumRows];
#pragma unroll
        for (int j = 0; j < kSumRows; ++j) {
            const int k = wave + j * kSumWaves;
            x[j] = k < P ? p[static_cast<int64_t>(k) * 2 * n] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < kSumRows; ++j) s += x[j];
    }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || c >= n) return;
    s = sums[0][lane];
#pragma unroll
    for (int w = 1; w < kSumWaves; ++w) s += sums[w][lane];
    out[c] = s;
}

// Three vectors a thread (which hold sums and gain of their own: 228 registers where two take 153), two / three us.  Rows of 64
// lanes: bf16 161342 x 1033 253 / 210, 34090 x 1100 with dR 57 / 61, 18151 x 1033 with dR 42 / 38, fp32 109649 x 760 170 / 194: bf16 without
// dR or on odd 2-byte boundaries.  Of 128: bf16 81024 x 2057 262 / 211, 1537 x 2601 13.7 / 13.9, fp32 80671 x 1033 199 / 180: all.  Of 256:
// bf16 30519 x 5461 226 / 191, 1525 x 5461 18.2 / 19.7, in windows 11904 x 4200 59.9 / 60.9, fp32 37810 x 2204 195 / 177, 1890 x 2204
// 13.9 / 14.9: where the call streams and its rows are fp32 or start anywhere.
template <typename T>
constexpr bool three_vectors(int tpr, bool streamed, bool window, bool on_words, bool add) {
    if (tpr == 64) return sizeof(T) == 2 && (!add || !on_words);
    return tpr == 128 || (streamed && (sizeof(T) == 4 || !window));
}

// Blocks, each of which leaves one row of column sums: one per compute unit.  With 128, 192, 256, 384 and 512 of them, both kernels:
// 2047 x 5461 bf16 28.5 24.4 21.9 27.5 28.0 us, 65536 x 512 52.3 41.5 38.1 44.5 42.5, 30000 x 1293 fp32 105.9 87.4 85.3 92.3 87.8.
int blocks_of(int64_t T, int64_t rows_each) {
    const int64_t want = (T + rows_each - 1) / rows_each;
    return static_cast<int>(want < kUnits ? want : kUnits);
}

// The most blocks that a call may take: of the shape with the fewest rows to a block.
template <typename T>
int most_blocks(int64_t rows, int64_t n) {
    int64_t rows_each = 1;
    if (in_registers<T>(n))
        by_shape<T>(n, [](int) { return false; }, [&](auto shape) { rows_each = decltype(shape)::B / decltype(shape)::TPR; });
    return blocks_of(rows, rows_each);
}

// Rows up to which dgain and dbias are added up beside dX in one launch.  180 rows, one launch and two, in a graph: 4096
// bf16 5.0 and 9.0 us, 7162 fp32 7.0 and 11.5, 250 bf16 4.5 and 5.8; 546 rows: 9.6 and 12.3, 14.6 and 17.8, 6.5 and 5.9;
// 1000 rows: 13.9 and 13.0, 26.5 and 25.4, 8.5 and 6.1.  (Outside a graph the second launch costs the host another 3 us.)
constexpr int64_t kFewRows = 768;

// The number of blocks whose sums wait to be added; 0 where dgain and dbias are done with (or not wanted).
template <typename T>
int launch(BackwardArgs a, hipStream_t s) {
    if (!in_registers<T>(a.n)) {
        const int blocks = a.part ? blocks_of(a.T, 1) : 0;
        if (a.part) {
            const dim3 g(static_cast<unsigned>((a.n + int64_t{kWide} * 8 - 1) / (kWide * 8)), static_cast<unsigned>(blocks));
            backward_wide_sums_kernel<T><<<g, kWide, 0, s>>>(a);
        }
        backward_wide_kernel<T><<<static_cast<unsigned>(a.T < kMostBlocks ? a.T : kMostBlocks), kWide, 0, s>>>(a);
        return blocks;
    }
    const auto all_on = [&](size_t bytes) {  // every row starts on so many bytes
        const auto on = [&](const void* p, int64_t ld) { return aligned_to(p, bytes) && ld * sizeof(T) % bytes == 0; };
        return on(a.dY, a.lddy) && on(a.H, a.ldh) && on(a.dX, a.lddx) && (!a.dR || on(a.dR, a.lddr));
    };
    const bool window = a.n * sizeof(T) % 16 == 0 && all_on(16);
    const bool once = static_cast<double>(a.T) * a.n * sizeof(T) * (a.dR ? 4 : 3) > kStreamed;
    const auto three = [&](int tpr) { return three_vectors<T>(tpr, once, window, all_on(4), a.dR != nullptr); };
    const auto run = [&](unsigned column_blocks, bool rows_too) {
        a.column_blocks = column_blocks;
        int blocks = 0;
        by_shape<T>(a.n, three, [&](auto shape) {
            typedef decltype(shape) S;
            blocks = rows_too ? blocks_of(a.T, S::B / S::TPR) : 0;
            const unsigned row_blocks = static_cast<unsigned>(blocks);
            const auto go = [&](auto win, auto add, auto stream) {
                constexpr bool kWindow = decltype(win)::value, kAdd = decltype(add)::value, kOnce = decltype(stream)::value;
                // (windows start on words; kernels that the rule leaves without calls are not built)
                if constexpr (S::V != 3 || S::TPR == 512 || three_vectors<T>(S::TPR, kOnce, kWindow, kWindow, kAdd))
                    backward_kernel<T, S, kWindow, kAdd, kOnce><<<column_blocks + row_blocks, S::B, 0, s>>>(a);
            };
            const auto with_add = [&](auto win, auto add) { once ? go(win, add, std::true_type{}) : go(win, add, std::false_type{}); };
            const auto with_window = [&](auto win) { a.dR ? with_add(win, std::true_type{}) : with_add(win, std::false_type{}); };
            if constexpr (S::TPR >= kWave)
                if (window) return with_window(std::true_type{});
            with_window(std::false_type{});
        });
        return blocks;
    };
    if (!a.part || a.T > kFewRows) {
        const int blocks = run(0, true);
        return a.part ? blocks : 0;
    }
    a.part = nullptr;
    constexpr int kColumns = kColumnLanes * 16 / static_cast<int>(sizeof(T));
    const unsigned columns = static_cast<unsigned>((a.n + kColumns - 1) / kColumns);
    if (a.dX != a.dY && a.dX != a.H) {
        run(columns, true);
    } else {  // dX overwrites what the columns' sums read
        run(columns, false);
        run(0, true);
    }
    return 0;
}

}  // namespace

size_t norm_backward_workspace_bytes(int64_t T, int64_t n, grass_dtype dt) {
    return static_cast<size_t>(dt == GRASS_F32 ? most_blocks<float>(T, n) : most_blocks<uint16_t>(T, n)) * 2 * n * sizeof(float);
}

grass_status launch_norm_backward(grass_norm kind, const void* dY, int64_t lddy, const void* H, int64_t ldh,
                                  const void* dR, int64_t lddr, grass_dtype dt, int64_t T, int64_t n,
                                  const void* gain, grass_dtype gdt, const float* mean, const float* rstd,
                                  void* dX, int64_t lddx, float* dgain, float* dbias, void* ws, hipStream_t s) {
    const bool sums = dgain || dbias;
    if (T == 0 && !sums) return GRASS_OK;
    int blocks = 0;  // without tokens dgain and dbias are sums of nothing
    if (T > 0) {
        const BackwardArgs a{dY, H, dR, gain, dX, lddy, ldh, lddr, lddx, T, static_cast<int>(n),
                             kind == GRASS_NORM_LAYER, gdt == GRASS_BF16, dbias != nullptr, mean, rstd,
                             sums ? static_cast<float*>(ws) : nullptr, 0, dgain, dbias};
        blocks = dt == GRASS_F32 ? launch<float>(a, s) : launch<uint16_t>(a, s);
        if (blocks == 0) return launch_status();
    }
    // (a grid has fewer than 2^32 threads: 16 of them for each column here)
    for (int64_t first = 0; first < n; first += kMostColumns) {
        const int64_t columns = n - first < kMostColumns ? n - first : kMostColumns;
        const dim3 grid(static_cast<unsigned>((columns + kWave - 1) / kWave), 2);
        column_sums_kernel<<<grid, kSumWaves * kWave, 0, s>>>(static_cast<const float*>(ws), blocks,
                                                              static_cast<int>(n), static_cast<int>(first), dgain, dbias);
    }
    return launch_status();
}

}  // namespace grass
