// grass_logp_forward: log probabilities of given tokens, entropies and alternatives.
//
// Measured: 32768 x 32000 bf16 303 us (7.0 TB/s); 256 x 128000 fp32 with entropies and 20 alternatives 41 (without alternatives
// 27), 1025 x 50001 bf16 in any position with 5 alternatives 39; one row of 32000 bf16 with 20 alternatives 10.0 (kernel 9.3).
//
// Bound by memory: a row is read once and stays in the registers of the threads that share it, for its maximum, its
// sums and its alternatives.  With c = scale log2(e) and d = (x - rmax) c, s = sum 2^d and u = sum 2^d d give
// rlog = ln s and entropy = ln s - ln(2) u / s.
#include <type_traits>

#include "elem.hpp"
#include "tokens.hpp"

namespace grass {
namespace {

struct ForwardArgs {
    const void* logits;
    int64_t T, ldl;
    int V, top, parts;
    Tokens targets;
    float scale;
    float *logp, *entropy, *rmax, *rlog, *top_logp;
    int32_t* top_idx;
    // of rows in parts: maximum, s and u of each part, and its alternatives
    float4* part;
    uint64_t* part_top;
};

// Numbers in the order of the logits (both zeros alike), above 0; and the logit again.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return (u >> 31) ? ~u : u | 0x80000000u;
}
constexpr uint32_t kMasked = 0x007FFFFFu;  // of minus infinity
__device__ __forceinline__ float logit_of(uint32_t order) {
    return __uint_as_float((order >> 31) ? order & 0x7FFFFFFFu : ~order);
}
// An alternative: in the order of the logits, then of the tokens, the lower one first.
__device__ __forceinline__ uint64_t key_of(uint32_t order, int token) {
    return static_cast<uint64_t>(order) << 32 | static_cast<uint32_t>(~token);
}

// The largest of three.  (As a builtin, each operand from memory is first made a quiet NaN if it is a signalling one.
// Here the result may be any where an operand is NaN: the sums of such a row are NaN.)
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// Threads that share a row, V vectors of 16 bytes each, in blocks of B; alternatives are chosen among up to kCap logits.  Eight wavefronts
// a SIMD fit in all shapes without alternatives, and in those of 256 and 512 threads with them, where the bf16 ones of eight vectors keep
// two registers in memory; of 64 threads with alternatives six fit (LDS), with eight vectors five (registers).
template <int TPR_, int V_>
struct Shape {
    static constexpr int TPR = TPR_, V = V_, B = TPR_ < 256 ? 256 : TPR_, kRows = B / TPR_, kCap = TPR_ < 256 ? 512 : 1024;
};

// A barrier of the threads that share a row, and their exchange of pairs of values over wavefronts.
template <typename S>
struct Group {
    static constexpr int kWaves = S::TPR / kWave;
    __device__ static __forceinline__ void sync() {
        if constexpr (kWaves > 1) __syncthreads();
        else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    // f and g over the wavefronts' values; `room` is not written again before the next sync but one
    template <typename F, typename G>
    __device__ static __forceinline__ void over_waves(float2* room, float& a, float& b, F f, G g) {
        if constexpr (kWaves > 1) {
            if (threadIdx.x % kWave == 0) room[threadIdx.x / kWave] = {a, b};
            sync();
            a = room[0].x;
            b = room[0].y;
#pragma unroll
            for (int w = 1; w < kWaves; ++w) {
                a = f(a, room[w].x);
                b = g(b, room[w].y);
            }
        }
    }
    __device__ static __forceinline__ int count(int* room, int v) {
#pragma unroll
        for (int o = kWave / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
        if constexpr (kWaves > 1) {
            sync();
            if (threadIdx.x % kWave == 0) room[threadIdx.x / kWave] = v;
            sync();
            v = 0;
            for (int w = 0; w < kWaves; ++w) v += room[w];
        }
        return v;
    }
};

// f of a lane's value and of another's 2^kStep lanes away, where lanes that were together in the steps before have the same value.
template <int kStep, typename F>
__device__ __forceinline__ float fold(float v, F f) {
    if constexpr (kStep < 4) {
        constexpr int kCtrl = kStep == 0 ? 0xB1 : kStep == 1 ? 0x4E : kStep == 2 ? 0x141 : 0x140;  // (as in sum_lanes)
        return f(v, dpp<kCtrl>(v));
    } else {
        const uint32_t a = __float_as_uint(v);
        const auto r = kStep == 4 ? __builtin_amdgcn_permlane16_swap(a, a, false, false) : __builtin_amdgcn_permlane32_swap(a, a, false, false);
        return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
}
template <typename F>
__device__ __forceinline__ void over_lanes(F step) {
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
    step(std::integral_constant<int, 2>{});
    step(std::integral_constant<int, 3>{});
    step(std::integral_constant<int, 4>{});
    step(std::integral_constant<int, 5>{});
}

struct Sums {
    float m, s, u;  // the largest logit, sum 2^d and sum 2^d d
};

// What a row's sums and alternatives come to, written by the threads that share the row (`lane` of `threads`).
struct Row {
    float m, m0, log;
    __device__ __forceinline__ Row(const ForwardArgs& a, const Sums& z, int64_t t, float given, bool there, int lane) : m(z.m) {
        m0 = m == -INFINITY ? 0.f : m;
        const bool none = z.s == 0.f;
        log = none ? 0.f : logf(z.s);
        if (lane == 0) {
            if (a.rmax) a.rmax[t] = m;
            if (a.rlog) a.rlog[t] = log;
            if (a.entropy) a.entropy[t] = none ? 0.f : log - kLn2 * z.u / z.s;
            if (a.logp) a.logp[t] = there ? scaled_difference(given, m0, a.scale) - log : 0.f;
        }
    }
    // the alternative of rank r (0: none)
    __device__ __forceinline__ void alternative(const ForwardArgs& a, int64_t t, int r, uint64_t key) const {
        const float x = logit_of(static_cast<uint32_t>(key >> 32));
        const bool spoiled = log != log;
        a.top_idx[t * a.top + r] = key && !spoiled ? static_cast<int32_t>(~static_cast<uint32_t>(key)) : -1;
        a.top_logp[t * a.top + r] = spoiled ? NAN : key ? scaled_difference(x, m0, a.scale) - log : -INFINITY;
    }
};

// The rank of each of `count` keys in LDS among them, by comparing it with all of them: out(rank, key) for ranks below
// `top`, and out(rank, 0) for those that are left.  Where there are fewer keys than threads, several compare for each; ranks:
// room for as many as there are keys, zeros, and zeros again afterwards (sync() between its uses).
template <typename Sync, typename F>
__device__ __forceinline__ void rank_keys(const uint64_t* keys, int* ranks, int count, int top, int lane, int threads, Sync sync, F out) {
    int each = 1;
    while (2 * each * count <= threads && each < 16) each *= 2;
    for (int i = lane / each; i < count; i += threads / each) {
        const uint64_t key = keys[i];
        int r = 0;
#pragma unroll 4
        for (int j = lane % each; j < count; j += each) r += keys[j] > key;
        if (each == 1) ranks[i] = r;
        else if (r) atomicAdd(&ranks[i], r);
    }
    sync();
    for (int i = lane; i < count; i += threads) {
        const int r = ranks[i];
        ranks[i] = 0;
        if (r < top) out(r, keys[i]);
    }
    for (int r = count + lane; r < top; r += threads) out(r, uint64_t{0});
}

// Leaves the keys of the `top` largest logits, and of those that equal the last of them, of `count` in LDS: comparing all with all would
// take the square of their number.  The last one's value is found bit by bit, by every wavefront for itself.
template <typename S>
__device__ __forceinline__ int keep_best(uint64_t* keys, int& found, int count, int top, int lane) {
    uint32_t value = 0;
    for (uint32_t bit = 0x80000000u; bit; bit >>= 1) {
        int n = 0;
        for (int i = threadIdx.x % kWave; i - static_cast<int>(threadIdx.x % kWave) < count; i += kWave)
            n += __popcll(__ballot(i < count && static_cast<uint32_t>(keys[i < count ? i : 0] >> 32) >= (value | bit)));
        if (n >= top) value |= bit;
        if (n == top) break;
    }
    constexpr int kMine = S::kCap / S::TPR;
    uint64_t mine[kMine];
#pragma unroll
    for (int k = 0; k < kMine; ++k) mine[k] = lane + k * S::TPR < count ? keys[lane + k * S::TPR] : 0;
    Group<S>::sync();
    if (lane == 0) found = 0;
    Group<S>::sync();
#pragma unroll
    for (int k = 0; k < kMine; ++k)
        if (static_cast<uint32_t>(mine[k] >> 32) >= value && mine[k]) keys[atomicAdd(&found, 1)] = mine[k];
    Group<S>::sync();
    return found;
}

// A row, or a part of one: where it starts, how many logits it has, and the token of the first.
template <typename T, typename S>
struct Piece {
    static constexpr int N = 16 / sizeof(T);
    int64_t item, t;
    int first, len;
    const T* x0;
    __device__ __forceinline__ Piece(const ForwardArgs& a, int64_t at) : item(at) {
        t = a.parts == 1 ? item : item / a.parts;
        const int part = a.parts == 1 ? 0 : static_cast<int>(item - t * a.parts);
        const auto start = [&](int p) { return p == a.parts ? a.V : static_cast<int>(static_cast<int64_t>(a.V) * p / a.parts) & ~7; };
        first = start(part);
        len = start(part + 1) - first;
        x0 = static_cast<const T*>(a.logits) + t * a.ldl + first;
    }
    // Where vector v of a thread starts: at the last N logits where fewer are left.  Those that another vector has, or
    // none, count as masked.
    __device__ __forceinline__ int at(int v, int lane) const {
        const int c = (v * S::TPR + lane) * N;
        return c + N <= len ? c : len > N ? len - N : 0;
    }
    template <bool kOnce>
    __device__ __forceinline__ void load(int v, int lane, Raw<T, N>& x) const {
        if (len >= N) x.template load_as<kOnce>(x0 + at(v, lane));
        else x.load_some(x0, len);
    }
    __device__ __forceinline__ void mask(int v, int lane, Raw<T, N>& x) const {
        const int c = (v * S::TPR + lane) * N, from = at(v, lane);
        if (c > from || len < N) {
            float z[N];
#pragma unroll
            for (int i = 0; i < N; ++i) z[i] = from + i >= c && from + i < len ? x.get(i) : -INFINITY;
            x.set(z);
        }
    }
};

template <typename T, typename S, bool kTop, bool kEntropy, bool kOnce>
__global__ __launch_bounds__(S::B) __attribute__((amdgpu_waves_per_eu(8))) void forward_kernel(ForwardArgs a) {
    constexpr int TPR = S::TPR, V = S::V, N = 16 / sizeof(T);
    typedef Group<S> G;
    typedef Raw<T, N> Vector;
    __shared__ float2 room[2][G::kWaves];
    __shared__ uint64_t keys[S::kRows][kTop ? S::kCap : 1];
    __shared__ float sets[2 * kWave];
    __shared__ int found[S::kRows], counts[G::kWaves], ranks[S::kRows][kTop ? S::kCap : 1];
    const int lane = threadIdx.x % TPR, wave0 = __builtin_amdgcn_readfirstlane(lane);
    const int group = S::kRows == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
    // `lane` again, so that what an earlier step made of it is not kept: each thread has the registers of eight wavefronts to a SIMD.
    const auto lane_again = [&] {
        int l = lane;
        asm volatile("" : "+v"(l));
        return l;
    };
    if constexpr (kTop) {
        for (int i = lane; i < S::kCap; i += TPR) ranks[group][i] = 0;
        G::sync();
    }
    const auto work = [&](int64_t item) {
        const Piece<T, S> row(a, item);
        const int64_t t = row.t;
        Vector x[V];
        // Whether the wavefront has logits of vector v at all.
        const auto some = [&](int v) { return (v * TPR + wave0) * N < row.len; };
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (some(v)) row.template load<kOnce>(v, lane, x[v]);
        uint32_t target = a.targets.V;
        float given = 0.f;
        if (lane == 0) {
            if (a.logp && a.parts == 1) target = a.targets[t];
            if (target < a.targets.V) given = load_as_f32(row.x0 + target);
            found[group] = 0;
        }
        const int masking = lane_again();
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (some(v)) row.mask(v, masking, x[v]);
        // The largest logit, of kSets sets for each lane of a wavefront where there are alternatives.
        constexpr int kSets = !kTop ? 1 : TPR > kWave ? 2 : V < 2 ? V : 2, kOwn = TPR > kWave ? 1 : kSets;
        float q[kSets];
#pragma unroll
        for (int k = 0; k < kSets; ++k) q[k] = -INFINITY;
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (some(v))
#pragma unroll
                for (int i = 0; i < N; i += 2) q[v % kOwn] = max3(q[v % kOwn], x[v].get(i), x[v].get(i + 1));
        float m = q[0];
#pragma unroll
        for (int k = 1; k < kOwn; ++k) m = fmaxf(m, q[k]);
        const float own = m;
        float least = -INFINITY;
        const auto larger = [](float p, float q) { return fmaxf(p, q); };
        const auto plus = [](float p, float q) { return p + q; };
        if constexpr (kTop) {
            // As many of the sets as `top` have a logit not below the `top`-th largest of their maxima, so that no alternative is
            // below it; and with twice as many sets as alternatives or more, few other logits are above: 64 sets left 300 of 32000
            // for 64 alternatives, 128 leave 90.  It is found bit by bit (down to some, below which hardly any differ).
            if constexpr (TPR > kWave) {
                constexpr int kSet = TPR / (kSets * kWave);  // threads
                over_lanes([&](auto step) {
                    constexpr int kStep = decltype(step)::value;
                    if constexpr ((1 << kStep) < kSet) m = fold<kStep>(m, larger);
                });
                if (lane % kSet == 0) sets[lane / kSet] = m;
                G::sync();
#pragma unroll
                for (int k = 0; k < kSets; ++k) {
                    q[k] = sets[k * kWave + threadIdx.x % kWave];
                    m = fmaxf(m, q[k]);
                }
            }
            constexpr int kBits = sizeof(T) == 2 ? 16 : 20;
            uint32_t order[kSets], bound = 0;
#pragma unroll
            for (int k = 0; k < kSets; ++k) order[k] = order_of(q[k]);
            for (uint32_t bit = 0x80000000u; bit >> (32 - kBits); bit >>= 1) {
                int n = 0;
#pragma unroll
                for (int k = 0; k < kSets; ++k) n += __popcll(__ballot(order[k] >= (bound | bit)));
                if (n >= a.top) bound |= bit;
                if (n == a.top && n < kSets * kWave) break;  // (where all sets are alternatives', many a bound is below all)
            }
            if (bound > kMasked) {  // the least of the maxima that are not below it
                least = INFINITY;
#pragma unroll
                for (int k = 0; k < kSets; ++k) least = order[k] >= bound ? fminf(least, q[k]) : least;
                over_lanes([&](auto step) { least = fold<decltype(step)::value>(least, [](float p, float q) { return fminf(p, q); }); });
            }
            over_lanes([&](auto step) { m = fold<decltype(step)::value>(m, larger); });
            if constexpr (TPR == kWave) G::sync();  // (found is 0 for all)
        } else {
            float none = 0.f;
            over_lanes([&](auto step) { m = fold<decltype(step)::value>(m, larger); });
            G::over_waves(room[0], m, none, larger, plus);
        }
        const float m0 = m == -INFINITY ? 0.f : m, c = scale_of_powers(a.scale), b = -(m0 * c);
        // 2^(x c + b) is off by a factor of 2^off, the rounding of b, which is known.  Where that is large, or the
        // product beyond fp32, the difference is formed first.
        const bool near = fabsf(b) <= 0x1p20f;
        const float off = near ? fmaf(m0, c, b) : 0.f;
        float s = 0.f, u = 0.f;
        const auto sums = [&](auto power) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!some(v)) continue;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    // (what the pass before made of a logit is not kept: it would take a register for each)
                    if (i % (4 / sizeof(T)) == 0) asm volatile("" : "+v"(x[v].w[i * sizeof(T) / 4]));
                    const float d = power(x[v].get(i)), e = __builtin_amdgcn_exp2f(d);
                    s += e;
                    if constexpr (kEntropy) u = fmaf(e, fmaxf(d, -200.f), u);  // (0 times minus infinity is 0 here)
                }
            }
        };
        if constexpr (kTop) {  // (one loop: what is left of the registers goes to the alternatives)
            const float z0 = near ? 0.f : m0, b0 = near ? b : 0.f;
            sums([&](float z) { return fmaf(z - z0, c, b0); });
            asm volatile("" : "+v"(s), "+v"(u));  // (and not behind them)
        } else {
            if (near) sums([&](float z) { return fmaf(z, c, b); });
            else sums([&](float z) { return (z - m0) * c; });
        }
        const auto keep = [&](float z, int token) {
            const int to = atomicAdd(&found[group], 1);
            if (to < S::kCap) keys[group][to] = key_of(order_of(z), token);
        };
        if (kTop && own >= least && own > -INFINITY) {  // (few threads)
            const int place = lane_again();
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!some(v)) continue;
#pragma unroll
                for (int k = 0; k < Vector::kWords; ++k) asm volatile("" : "+v"(x[v].w[k]));
                float best = -INFINITY;
#pragma unroll
                for (int i = 0; i < N; i += 2) best = max3(best, x[v].get(i), x[v].get(i + 1));
                if (best < least) continue;
                const int token = row.first + row.at(v, place);
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (x[v].get(i) >= least && x[v].get(i) > -INFINITY) keep(x[v].get(i), token + i);
            }
        }
        s = sum_lanes<kWave>(s);
        if constexpr (kEntropy) u = sum_lanes<kWave>(u);
        G::over_waves(room[1], s, u, plus, plus);
        if constexpr (G::kWaves == 1) G::sync();
        const float back = __builtin_amdgcn_exp2f(-off);
        s *= back;
        const Sums z{m, s, u * back - off * s};
        int count = kTop ? found[group] : 0;
        if (kTop && count > S::kCap) {
            // More logits at the bound and above than there is room for, as where many are alike.  Those above it may be enough; else
            // the value of the last alternative is found, where it is not the bound, and its token among equals, bit by bit.
            // (Read again: with the row's registers in these loops others would not do.  Looking for the token in one vector at a
            // time takes half the time here and more registers, 51 us for 39 at 1025 x 50001; as a function of its own 45.)
            const int place = lane_again();
            const auto each = [&](auto f) {
#pragma unroll 1
                for (int v = 0; v < V; ++v) {
                    Vector y;
                    row.template load<false>(v, place, y);
                    row.mask(v, place, y);
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        if (y.get(i) > -INFINITY) f(y.get(i), row.first + row.at(v, place) + i);
                }
            };
            const auto how_many = [&](auto f) {
                int n = 0;
                each([&](float z, int token) { n += f(order_of(z), token); });
                return G::count(counts, n);
            };
            uint32_t value = order_of(least);
            int above = how_many([&](uint32_t q, int) { return q > value; });
            if (above > S::kCap) {
                value = 0;
                for (uint32_t bit = 0x80000000u; bit; bit >>= 1)
                    if (how_many([&](uint32_t q, int) { return q >= (value | bit); }) >= a.top) value |= bit;
                above = how_many([&](uint32_t q, int) { return q > value; });
            }
            int last = above < a.top ? 0 : -1;
            for (int bit = above < a.top ? 1 << (31 - __clz(a.V)) : 0; bit; bit >>= 1)
                if (how_many([&](uint32_t q, int j) { return q == value && j < (last | bit); }) < a.top - above) last |= bit;
            if (lane == 0) found[group] = 0;
            G::sync();
            each([&](float z, int token) {
                const uint32_t q = order_of(z);
                if (q > value || (q == value && token <= last)) keep(z, token);
            });
            G::sync();
            count = found[group];
        }
        if constexpr (kTop)
            if (count > 2 * a.top) count = keep_best<S>(keys[group], found[group], count, a.top, lane);
        if (a.parts == 1) {
            const Row out(a, z, t, given, target < a.targets.V, lane);
            if constexpr (kTop)
                rank_keys(keys[group], ranks[group], count, a.top, lane, TPR, G::sync, [&](int r, uint64_t key) { out.alternative(a, t, r, key); });
        } else {
            if (lane == 0) a.part[item] = {z.m, z.s, z.u, 0.f};
            if constexpr (kTop)
                rank_keys(keys[group], ranks[group], count, a.top, lane, TPR, G::sync,
                          [&](int r, uint64_t key) { a.part_top[item * a.top + r] = key; });
        }
        G::sync();  // the next row's threads write what this one's read
    };
    const int64_t items = a.T * a.parts, step = static_cast<int64_t>(gridDim.x) * S::kRows;
    for (int64_t item = static_cast<int64_t>(blockIdx.x) * S::kRows + group; item < items; item += step) work(item);
}

// Rows in parts, one per workgroup at a time.  The parts' alternatives go through LDS as many at a time as there is room for.
constexpr int kJoin = 256, kJoinKeys = 2048;

template <typename T>
__global__ __launch_bounds__(kJoin) void join_kernel(ForwardArgs a) {
    typedef Group<Shape<kJoin, 1>> G;
    __shared__ float2 room[3][G::kWaves];
    __shared__ uint64_t keys[kJoinKeys], best[GRASS_LOGP_MOST_TOP], bounds[G::kWaves];
    __shared__ int ranks[kJoinKeys], found;
    for (int i = threadIdx.x; i < kJoinKeys; i += kJoin) ranks[i] = 0;
    const auto larger = [](float p, float q) { return fmaxf(p, q); };
    const auto plus = [](float p, float q) { return p + q; };
    const int lane = threadIdx.x;
    const float c = scale_of_powers(a.scale);
    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        uint32_t target = a.targets.V;
        float given = 0.f;
        if (lane == 0) {
            if (a.logp) target = a.targets[t];
            if (target < a.targets.V) given = load_as_f32(static_cast<const T*>(a.logits) + t * a.ldl + target);
        }
        const float4* part = a.part + t * a.parts;
        float m = -INFINITY, none = 0.f;
        for (int p = lane; p < a.parts; p += kJoin) m = fmaxf(m, part[p].x);
#pragma unroll
        for (int o = kWave / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, kWave));
        G::over_waves(room[0], m, none, larger, plus);
        float s = 0.f, u = 0.f;
        for (int p = lane; p < a.parts; p += kJoin) {
            const float4 q = part[p];
            if (q.y == 0.f) continue;  // all masked
            const float d = q.x == m ? 0.f : (q.x - m) * c, w = __builtin_amdgcn_exp2f(d);
            s += w * q.y;
            if (w > 0.f) u += w * (q.z + d * q.y);
        }
        s = sum_lanes<kWave>(s);
        u = sum_lanes<kWave>(u);
        G::over_waves(room[1], s, u, plus, plus);
        const Row out(a, {m, s, u}, t, given, target < a.targets.V, lane);
        if (a.top) {
            const uint64_t* from = a.part_top + t * a.parts * a.top;
            const int64_t all = static_cast<int64_t>(a.parts) * a.top;
            // no alternative is behind the last one of any part that has as many
            uint64_t bound = 1;
            for (int p = lane; p < a.parts; p += kJoin) {
                const uint64_t last = from[static_cast<int64_t>(p + 1) * a.top - 1];
                bound = last > bound ? last : bound;
            }
#pragma unroll
            for (int o = kWave / 2; o > 0; o >>= 1) {
                const uint64_t other = __shfl_xor(bound, o, kWave);
                bound = other > bound ? other : bound;
            }
            if (lane % kWave == 0) bounds[lane / kWave] = bound;
            if (lane == 0) found = 0;
            G::sync();
            for (int w = 0; w < G::kWaves; ++w) bound = bounds[w] > bound ? bounds[w] : bound;
            for (int64_t at = 0; at < all; at += kJoin) {
                if (at + lane < all) {
                    const uint64_t key = from[at + lane];
                    if (key >= bound) keys[atomicAdd(&found, 1)] = key;
                }
                G::sync();
                const int count = found;
                if (count > kJoinKeys - kJoin && at + kJoin < all) {  // no room for as many again: the best of them
                    rank_keys(keys, ranks, count, a.top, lane, kJoin, G::sync, [&](int r, uint64_t key) { best[r] = key; });
                    G::sync();
                    if (lane < a.top) keys[lane] = best[lane];
                    if (lane == 0) found = a.top;
                }
                G::sync();
            }
            rank_keys(keys, ranks, found, a.top, lane, kJoin, G::sync, [&](int r, uint64_t key) { out.alternative(a, t, r, key); });
        }
        G::sync();
    }
}

// The widest row of one part, and how many parts a row has.
template <typename T>
constexpr int kWidest = 8 * 512 * (16 / sizeof(T));
template <typename T>
int parts_of(int64_t V) {
    return V <= kWidest<T> ? 1 : static_cast<int>((V + kWidest<T> - 16) / (kWidest<T> - 15));  // (see launch)
}
int parts_of(int64_t V, grass_dtype dt) { return dt == GRASS_F32 ? parts_of<float>(V) : parts_of<uint16_t>(V); }

// us with the largest parts at 512 threads / 1024 / 256: 1025 x 50001 bf16 with 5 alternatives 51 / 69 / 55, 256 x 128000 fp32 with 20
// 55 / 63 / 98, 32768 x 32000 bf16 304 / - / 367 (all before later steps).  One row of 32000 bf16 by 1024 threads 11.0 us, by 512 9.6.
// Otherwise the fewest threads and vectors that hold a row.  us of 32768 bf16 rows without / with entropies and 20 alternatives by the
// shape taken, and by a larger one: 2048 logits 31 / 63, by 256 threads 50 / 136; 4096 46 / 95, by 256 threads 60 / 154; 8192 97 / 187, by
// 512 threads 128 / 296; 16384 162 / 261, by 512 threads 179 / 352; 18000 with five vectors 201 / 365, with eight 203 / 385; 20480 212 / 380
// and 217 / 400.
template <typename T, typename F>
void by_width(int64_t len, F&& f) {
    const int64_t vectors = (len * static_cast<int64_t>(sizeof(T)) + 15) / 16;
    if (vectors <= 64) f(Shape<64, 1>{});
    else if (vectors <= 128) f(Shape<64, 2>{});
    else if (vectors <= 256) f(Shape<64, 4>{});
    else if (vectors <= 512) f(Shape<64, 8>{});
    else if (vectors <= 1024) f(Shape<256, 4>{});
    else if (vectors <= 2048) f(Shape<256, 8>{});
    else if (vectors <= 2560) f(Shape<512, 5>{});
    else f(Shape<512, 8>{});
}

template <typename T>
void launch(const ForwardArgs& a, hipStream_t s) {
    // (parts start on multiples of 8 logits: one has up to 7 more than its share)
    const int64_t len = a.parts == 1 ? a.V : (a.V + a.parts - 1) / a.parts + 7;
    by_width<T>(len, [&](auto shape) {
        typedef decltype(shape) S;
        const int64_t blocks = (a.T * a.parts + S::kRows - 1) / S::kRows;
        const unsigned grid = walking_grid(blocks);
        const bool once = static_cast<double>(a.T) * a.V * sizeof(T) > kStreamed;
        const auto go = [&](auto top, auto entropy, auto stream) {
            forward_kernel<T, S, decltype(top)::value, decltype(entropy)::value, decltype(stream)::value><<<grid, S::B, 0, s>>>(a);
        };
        const auto with_entropy = [&](auto top, auto entropy) { once ? go(top, entropy, std::true_type{}) : go(top, entropy, std::false_type{}); };
        const auto with_top = [&](auto top) { a.entropy ? with_entropy(top, std::true_type{}) : with_entropy(top, std::false_type{}); };
        a.top ? with_top(std::true_type{}) : with_top(std::false_type{});
    });
    if (a.parts > 1) join_kernel<T><<<walking_grid(a.T), kJoin, 0, s>>>(a);
}

}  // namespace

size_t logp_forward_workspace_bytes(int64_t T, int64_t V, int64_t top, grass_dtype dt) {
    const int parts = parts_of(V, dt);
    return parts == 1 ? 0 : static_cast<size_t>(T) * parts * (16 + 8 * top);
}

grass_status launch_logp_forward(const void* logits, grass_dtype dt, int64_t T, int64_t V, int64_t ldl, const void* targets,
                                 grass_index idt, float scale, float* logp, float* entropy, float* rmax, float* rlog,
                                 int64_t top, float* top_logp, int32_t* top_idx, void* ws, hipStream_t s) {
    if (T == 0) return GRASS_OK;
    const int parts = parts_of(V, dt);
    float4* part = static_cast<float4*>(ws);
    const ForwardArgs a{logits, T, ldl, static_cast<int>(V), static_cast<int>(top), parts, tokens(targets, idt, V), scale,
                        logp, entropy, rmax, rlog, top_logp, top_idx,
                        part, parts == 1 ? nullptr : reinterpret_cast<uint64_t*>(part + T * parts)};
    if (dt == GRASS_F32) launch<float>(a, s);
    else launch<uint16_t>(a, s);
    return launch_status();
}

}  // namespace grass
