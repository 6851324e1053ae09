// grass_embed_backward: the gradient of the embedding, summed by tokens.
//
// The places of the batch are ordered by token (stably, so that a token's places stay in order), and the rows of dY are then
// read once in that order, each piece of kPiece places by a wavefront (one for each 16 bytes times 64 of a row) that adds the rows of a
// token up in registers.  Tokens of up to kPiece places are summed and stored by the wavefront whose piece has the first of them;
// longer ones, the frequent ones, leave a partial sum a piece, which a second kernel adds up in order.  All sums are fp32, and
// their order depends on the tokens alone.
//
// Bound by memory: dY is read once, dE written once.  Measured, whole calls: 131072 x 4096 bf16 into 32000 bf16 rows 313 us (1.34 GB,
// 4.3 TB/s; the sums 265, ordering 28, frequent tokens 19); 65536 x 512 bf16 into fp32 rows 55 us (the sums 25, ordering 25,
// frequent tokens 5.5); 2047 x 5461 bf16 added to fp32 rows 28.
#include "elem.hpp"
#include "tokens.hpp"

namespace grass {
namespace {

// ------------------------------------------------------------------------------ places by token
// A radix sort by up to kMostBits bits of the token at a time, from the lowest on: per pass one kernel counts each
// workgroup's digits, and one finds from all counts where its own places go.
struct Place {
    uint32_t token, t;
};
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / kWave, kMostBits = 9, kMostBins = 1 << kMostBits;

struct SortArgs {
    Tokens ids;         // of the first pass
    const Place* from;  // of the others
    Place* to;
    int64_t T, chunk;   // places of a workgroup: a multiple of kSortThreads
    int shift, bits, blocks;
    uint32_t* counts;   // blocks x 2^bits
    uint8_t* present;   // NULL, or a byte for each token: whether it occurs
    uint32_t* found;    // how many tokens have more places than a piece: 0 here; and how many places are listed
};

__device__ __forceinline__ Place place_at(const SortArgs& a, int64_t i) {
    return a.from ? a.from[i] : Place{a.ids[i], static_cast<uint32_t>(i)};
}

// The lanes of a wavefront whose digit is this lane's; lanes without a place match none.
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, int bits, bool there) {
    uint64_t same = __ballot(there);
    for (int b = 0; b < bits; ++b) {
        const bool set = digit >> b & 1;
        const uint64_t with = __ballot(set);
        same &= set ? with : ~with;
    }
    return same;
}

// 64 places of a wavefront at a time: what each lane has, and which of them have its digit.
struct Step {
    Place p;
    uint32_t digit;
    uint64_t same;
    bool there;
    __device__ __forceinline__ bool leads() const { return there && (same & ((uint64_t{1} << threadIdx.x % kWave) - 1)) == 0; }
    __device__ __forceinline__ int before() const { return __popcll(same & ((uint64_t{1} << threadIdx.x % kWave) - 1)); }
};
__device__ __forceinline__ Step step_of(Place p, bool there, int shift, int bits) {
    Step s;
    s.p = p;
    s.there = there;
    s.digit = p.token >> shift & ((1u << bits) - 1);
    s.same = same_digit(s.digit, bits, there);
    return s;
}

// Where the place of a step goes; the counter of its digit, which the wavefront's lanes share, moves on.  In the next step another
// lane may lead the digit: the fences keep its access behind this one's (they cost no instruction; a wavefront's accesses to LDS are
// served in order).
__device__ __forceinline__ uint32_t take_place(uint32_t* next, const Step& s) {
    const uint32_t at = next[s.digit];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (s.leads()) next[s.digit] = at + __popcll(s.same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    return at + s.before();
}
// The same for a step that is only counted.
__device__ __forceinline__ void count_place(uint32_t* next, const Step& s) {
    if (s.leads()) next[s.digit] += __popcll(s.same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// f(step) over the wavefront's share of the workgroup's chunk, as often as asked.  kSteps: its steps where they stay in
// registers; 0: any number of them, read again each time.
template <int kSteps>
struct Share {
    const SortArgs& a;
    int64_t start, share;
    Place p[kSteps ? kSteps : 1];
    Step step[kSteps ? kSteps : 1];
    __device__ __forceinline__ explicit Share(const SortArgs& args) : a(args) {
        share = a.chunk / kSortWaves;
        start = blockIdx.x * a.chunk + threadIdx.x / kWave * share;
        if constexpr (kSteps > 0)
#pragma unroll
            for (int k = 0; k < kSteps; ++k) p[k] = fetch(start + k * kWave);
    }
    __device__ __forceinline__ void arrive() {
        if constexpr (kSteps > 0)
#pragma unroll
            for (int k = 0; k < kSteps; ++k) step[k] = made(p[k], start + k * kWave);
    }
    __device__ __forceinline__ Place fetch(int64_t at) const {
        const int64_t i = at + threadIdx.x % kWave;
        return i < a.T ? place_at(a, i) : Place{0, 0};
    }
    __device__ __forceinline__ Step made(Place p, int64_t at) const {
        return step_of(p, at + threadIdx.x % kWave < a.T, a.shift, a.bits);
    }
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        if constexpr (kSteps > 0) {
#pragma unroll
            for (int k = 0; k < kSteps; ++k) f(step[k]);
        } else {
            for (int64_t at = start; at < start + share && at < a.T; at += kWave) f(made(fetch(at), at));
        }
    }
};

template <int kSteps>
__global__ __launch_bounds__(kSortThreads) void count_kernel(SortArgs a) {
    __shared__ uint32_t count[kMostBins];
    const uint32_t bins = 1u << a.bits;
    Share<kSteps> mine(a);
    if (threadIdx.x < bins) count[threadIdx.x] = 0;
    if (!a.from) {  // what later kernels start from
        if (blockIdx.x == 0 && threadIdx.x == 0) {
            a.found[0] = 0;
            a.found[1] = static_cast<uint32_t>(a.T);
        }
        if (a.present)
            for (int64_t v = (static_cast<int64_t>(blockIdx.x) * kSortThreads + threadIdx.x) * 16; v < a.ids.V;
                 v += static_cast<int64_t>(gridDim.x) * kSortThreads * 16)
                *reinterpret_cast<uint4*>(a.present + v) = {0, 0, 0, 0};
    }
    __syncthreads();
    mine.arrive();
    mine.each([&](const Step& s) {
        if (s.leads()) atomicAdd(&count[s.digit], __popcll(s.same));
    });
    __syncthreads();
    if (threadIdx.x < bins) a.counts[blockIdx.x * bins + threadIdx.x] = count[threadIdx.x];
}

// Where each wavefront's places of each digit go: next[wave][digit] holds how many it has, and then where the first goes.  n: how many
// of digit threadIdx.x there are in all, b: those of the workgroups before (threads below `bins`).
__device__ __forceinline__ void places_of_digits(uint32_t (&next)[kSortWaves][kMostBins], uint32_t (&sums)[kSortWaves], uint32_t bins, uint32_t n, uint32_t b) {
    const int wave = threadIdx.x / kWave;
    const uint32_t upto = wave_inclusive_scan(threadIdx.x < bins ? n : 0u);
    if (threadIdx.x % kWave == kWave - 1) sums[wave] = upto;
    __syncthreads();
    if (threadIdx.x < bins) {
        uint32_t at = upto - n + b, c[kSortWaves];
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) c[w] = next[w][threadIdx.x];
#pragma unroll
        for (int w = 0; w < kMostBins / kWave; ++w) at += w < wave ? sums[w] : 0;
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            next[w][threadIdx.x] = at;
            at += c[w];
        }
    }
    __syncthreads();
}

template <int kSteps>
__global__ __launch_bounds__(kSortThreads) void scatter_kernel(SortArgs a) {
    __shared__ uint32_t next[kSortWaves][kMostBins], before[kSortThreads], all[kSortThreads], sums[kSortWaves];
    const uint32_t bins = 1u << a.bits, wave = threadIdx.x / kWave;
    Share<kSteps> mine(a);
    // all counts of a digit, and those of the workgroups before this one, by several threads
    const uint32_t digit = threadIdx.x & (bins - 1), groups = kSortThreads / bins, group = threadIdx.x / bins;
    uint32_t b = 0, n = 0;
#pragma unroll 16
    for (uint32_t k = group; k < static_cast<uint32_t>(a.blocks); k += groups) {
        const uint32_t c = a.counts[k * bins + digit];
        n += c;
        b += k < blockIdx.x ? c : 0;
    }
    before[threadIdx.x] = b;
    all[threadIdx.x] = n;
    for (uint32_t k = group; k < kSortWaves; k += groups) next[k][digit] = 0;
    mine.arrive();
    __syncthreads();
    mine.each([&](const Step& s) { count_place(next[wave], s); });
    if (threadIdx.x < bins)
        for (uint32_t g = 1; g < groups; ++g) {
            b += before[threadIdx.x + g * bins];
            n += all[threadIdx.x + g * bins];
        }
    places_of_digits(next, sums, bins, n, b);
    mine.each([&](const Step& s) {
        const uint32_t at = take_place(next[wave], s);
        if (!s.there) return;
        a.to[at] = s.p;
        if (!a.from && a.present && s.p.token < a.ids.V) a.present[s.p.token] = 1;
    });
}

// The same in one kernel, where tokens and places are not too many: each workgroup takes kRange tokens, looks through all places
// for them, and counts those of lower tokens on the way, so that it knows where its own go.  What is no token is not listed.  A
// wavefront looks through a share of the places and lists what it finds, up to kList of them; with more it looks again.
constexpr int kRange = 256, kList = 384, kLook = 8;

__global__ __launch_bounds__(kSortThreads) void order_kernel(SortArgs a) {
    __shared__ uint32_t next[kSortWaves][kMostBins], sums[kSortWaves], lower;
    __shared__ uint32_t list[kSortWaves][kList];  // place from the share's first on, and token from the range's first on in 8 bits
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const uint32_t lo = blockIdx.x * kRange, V = a.ids.V;
    const uint32_t range = V - lo < kRange ? V - lo : kRange;
    const int64_t share = (a.T + kSortThreads - 1) / kSortThreads * kWave, start = wave * share;
    const int64_t end = start + share < a.T ? start + share : a.T;
    for (uint32_t k = threadIdx.x / kRange; k < kSortWaves; k += kSortThreads / kRange) next[k][threadIdx.x % kRange] = 0;
    if (threadIdx.x == 0) {
        lower = 0;
        if (blockIdx.x == 0) a.found[0] = 0;
    }
    uint32_t below = 0, n = 0;
    const auto look = [&](auto type) {
        typedef decltype(type) Id;
        const Id* ids = static_cast<const Id*>(a.ids.p);
        const auto fetch = [&](int64_t at, Id (&id)[kLook]) {
#pragma unroll
            for (int k = 0; k < kLook; ++k) {
                const int64_t i = at + k * kWave + lane;
                id[k] = ids[i < end ? i : end - 1];
            }
        };
        const auto one = [&](Id id, int64_t first, uint64_t there) {
            const uint32_t low = static_cast<uint32_t>(id);
            // (a negative number of 32 bits is above V; one of 64 has bits above the lower 32, like all that are too large)
            if constexpr (sizeof(Id) == 8) there &= __ballot(static_cast<uint32_t>(static_cast<uint64_t>(id) >> 32) == 0);
            below += __popcll(__ballot(low < lo) & there);
            const uint64_t in = __ballot(low - lo < range) & there;
            if (in == 0) return;
            if (in >> lane & 1) {
                const uint32_t to = n + __popcll(in & ((uint64_t{1} << lane) - 1));
                if (to < kList) list[wave][to] = (static_cast<uint32_t>(first - start) + lane) << 8 | (low - lo);
            }
            n += __popcll(in);
        };
        const auto work = [&](int64_t at, const Id (&id)[kLook]) {
            if (at + kLook * kWave <= end) {
#pragma unroll
                for (int k = 0; k < kLook; ++k) one(id[k], at + k * kWave, ~uint64_t{0});
            } else {
#pragma unroll
                for (int k = 0; k < kLook; ++k) {
                    const int64_t left = end - (at + k * kWave);
                    if (left > 0) one(id[k], at + k * kWave, left < kWave ? (uint64_t{1} << left) - 1 : ~uint64_t{0});
                }
            }
        };
        for (int64_t at = start; at < end; at += kLook * kWave) {
            Id id[kLook];
            fetch(at, id);
            work(at, id);
        }
    };
    if (a.ids.wide) look(int64_t{});
    else look(int32_t{});
    // f(step) over what the wavefront has found, 64 at a time
    const auto each = [&](auto f) {
        if (n <= kList) {
            for (uint32_t k = 0; k < n; k += kWave) {
                const bool there = k + lane < n;
                const uint32_t found = there ? list[wave][k + lane] : 0;
                f(step_of({found & 255, static_cast<uint32_t>(start) + (found >> 8)}, there, 0, 8));
            }
        } else {
            for (int64_t at = start; at < end; at += kLook * kWave) {
                uint32_t code[kLook];
#pragma unroll
                for (int k = 0; k < kLook; ++k) {
                    const int64_t i = at + k * kWave + lane;
                    code[k] = a.ids[i < end ? i : end - 1] - lo;
                    if (i >= end) code[k] = kRange;
                }
#pragma unroll
                for (int k = 0; k < kLook; ++k)
                    f(step_of({code[k], static_cast<uint32_t>(at + k * kWave + lane)}, code[k] < range, 0, 8));
            }
        }
    };
    __syncthreads();
    if (lane == 0) atomicAdd(&lower, below);
    each([&](const Step& s) { count_place(next[wave], s); });
    __syncthreads();
    uint32_t count = 0;
    if (threadIdx.x < kRange) {
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) count += next[w][threadIdx.x];
        if (a.present && lo + threadIdx.x < V) a.present[lo + threadIdx.x] = count > 0;
    }
    places_of_digits(next, sums, kRange, count, lower);
    if (blockIdx.x + 1 == gridDim.x && threadIdx.x == 0) {  // what is none is not listed
        uint32_t all = lower;
        for (int w = 0; w < kSortWaves; ++w) all += sums[w];
        a.found[1] = all;
    }
    each([&](const Step& s) {
        const uint32_t at = take_place(next[wave], s);
        if (s.there) a.to[at] = {lo + s.p.token, s.p.t};
    });
}

// ----------------------------------------------------------------------------------------- sums
constexpr int kAhead = 8, kSumThreads = 256;

struct SumArgs {
    const void* dY;
    void* dE;
    int64_t lddy, ldde, T, pieces;
    int n, tiles;
    uint32_t V;
    float scale;
    const Place* places;
    const uint8_t* present;
    uint32_t *found, *list;  // how many tokens have more places than a piece, and how many are listed; the pieces where such tokens start
    float* partial;          // two rows a piece: of the token that it starts within, and of the long one that starts in it
    int64_t width;           // floats of such a row
    int64_t sum_blocks, blocks;  // that add up pieces, and with those that write zeros
    int zero_rows;               // of dE, for one of these
};

// Columns `from` .. `from` + N - 1 of a row of n: the row's last N where fewer are left, of which the first `skip` are another
// lane's (all of them: the lane has none).
template <int N>
struct Columns {
    int64_t from;
    int skip, n;
    Columns() = default;
    __device__ __forceinline__ Columns(int64_t c, int width) : n(width) {
        from = c + N <= n ? c : n > N ? n - N : 0;
        skip = static_cast<int>(c - from < N ? c - from : N);
    }
    template <bool kOnce, typename T>
    __device__ __forceinline__ void load(const T* row, Raw<T, N>& x) const {
        if (n >= N) x.template load_as<kOnce>(row + from);
        else x.load_some(row, n);
    }
    template <bool kOnce, typename T>
    __device__ __forceinline__ void store(T* row, const float (&x)[N]) const {
        Raw<T, N> r;
        r.set(x);
        if (skip == 0 && n >= N) return r.template store_as<kOnce>(row + from);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i >= skip && from + i < n) row[from + i] = r.element(i);
    }
};

// Zeros in those of up to 64 rows from `first` on whose bit in `absent` is set, kSumThreads to a row.
template <typename TE, bool kOnce>
__device__ __forceinline__ void zero_rows(const SumArgs& a, int64_t first, uint64_t absent) {
    constexpr int N = 16 / sizeof(TE);
    Raw<TE, N> zero;
    zero.zero();
    for (; absent; absent &= absent - 1) {
        TE* row = static_cast<TE*>(a.dE) + (first + __ffsll(static_cast<unsigned long long>(absent)) - 1) * a.ldde;
        for (int64_t c = threadIdx.x * N; c < a.n; c += kSumThreads * N) {
            if (c + N <= a.n) zero.template store_as<kOnce>(row + c);
            else zero.store_some(row + c, static_cast<int>(a.n - c));
        }
    }
}

// A wavefront's work: the columns of a tile in a piece.
template <typename TY, typename TE, int kPiece, bool kAccumulate, bool kIn, bool kOut>
__device__ __forceinline__ void sum_piece(const SumArgs& a, int64_t item) {
    // 16 bytes of dY a lane, and of dE at a time
    constexpr int N = 16 / sizeof(TY), kEach = sizeof(TY) < sizeof(TE) ? 16 / sizeof(TE) : N, kGroups = N / kEach;
    const int lane = threadIdx.x % kWave;
    const int64_t piece = item / a.tiles;
    const int tile = static_cast<int>(item - piece * a.tiles);
    if (piece >= a.pieces) return;
    // the piece's places and as many behind it; a start is a place whose token is not the one before's
    const int64_t p0 = piece * kPiece;
    const int64_t T = a.found[1];
    const auto token_at = [&](int64_t i) { return i < 0 ? 0xFFFFFFFEu : i < T ? a.places[i].token : 0xFFFFFFFFu; };
    const int64_t mine = p0 + lane;
    const Place here = mine < T ? a.places[mine] : Place{0xFFFFFFFFu, 0};
    const uint32_t left = token_at(mine - 1), back = token_at(p0 - 1 - lane);  // (back: lane l is l + 1 places before the piece)
    const uint64_t starts = __ballot(here.token != left);
    const uint32_t head = __builtin_amdgcn_readfirstlane(here.token);
    const uint64_t none = __ballot(here.token >= a.V);
    const int tokens = none ? __ffsll(static_cast<unsigned long long>(none)) - 1 : kWave;  // places that have one
    const uint64_t within = (uint64_t{1} << kPiece) - 1;
    const int first = starts & within ? __ffsll(static_cast<unsigned long long>(starts & within)) - 1 : kPiece;
    // the places behind place i up to the next start (64 - i: none in sight)
    const auto length = [&](int i) {
        const uint64_t later = i < 63 ? starts >> (i + 1) << (i + 1) : 0;
        return (later ? __ffsll(static_cast<unsigned long long>(later)) - 1 : kWave) - i;
    };
    bool head_long = false;
    if (first > 0) {
        const uint64_t other = __ballot(back != head);
        const int since = other ? __ffsll(static_cast<unsigned long long>(other)) - 1 : kWave;  // places before the piece
        head_long = since >= kPiece || since + (starts & 1 ? 0 : length(0)) > kPiece;
    }
    int begin = head_long ? 0 : first, end = head_long && first == kPiece ? kPiece : begin, tail = kWave;
    if (first < kPiece) {
        const int last = 63 - __clzll(static_cast<long long>(starts & within));
        const int len = length(last);
        end = last + len;
        if (len > kPiece) {
            end = kPiece;
            tail = last;
        }
    }
    if (end > tokens) end = tokens;
    if (begin >= end) return;
    if (tail < end && tile == 0 && lane == 0) a.list[atomicAdd(a.found, 1u)] = static_cast<uint32_t>(piece);

    // a lane's columns: kGroups times kEach side by side
    Columns<kEach> at[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) at[g] = Columns<kEach>((static_cast<int64_t>(tile) * kGroups + g) * (kWave * kEach) + lane * kEach, a.n);
    const auto some = [&](int g) { return g == 0 || (static_cast<int64_t>(tile) * kGroups + g) * (kWave * kEach) < a.n; };
    float sum[kGroups][kEach];
    const auto clear = [&] {
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
#pragma unroll
            for (int q = 0; q < kEach; ++q) sum[g][q] = 0.f;
    };
    clear();
    const auto last_of_token = [&](int j) { return j + 1 == end || (starts >> (j + 1) & 1); };
    const auto partly = [&](int j) { return j < first || j >= tail; };
    const auto row_of = [&](int j) { return static_cast<TE*>(a.dE) + static_cast<uint32_t>(__builtin_amdgcn_readlane(here.token, j)) * a.ldde; };
    for (int i = begin; i < end; i += kAhead) {
        Raw<TY, kEach> x[kAhead][kGroups];
        Raw<TE, kEach> was[kAccumulate ? kAhead : 1][kGroups];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int j = i + k < end ? i + k : end - 1;
            const TY* row = static_cast<const TY*>(a.dY) + static_cast<uint32_t>(__builtin_amdgcn_readlane(here.t, j)) * a.lddy;
#pragma unroll
            for (int g = 0; g < kGroups; ++g)
                if (some(g)) at[g].template load<kIn>(row, x[k][g]);
        }
        // (The rows that are added to are on their way at the same time.  Their registers, bf16 added to fp32, leave room for three
        // wavefronts a SIMD, where six fit without.)
        if constexpr (kAccumulate)
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int j = i + k;
                if (j >= end || !last_of_token(j) || partly(j)) continue;
                const TE* row = row_of(j);
#pragma unroll
                for (int g = 0; g < kGroups; ++g)
                    if (some(g)) at[g].template load<false>(row, was[k][g]);
            }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int j = i + k;
            if (j >= end) break;
#pragma unroll
            for (int g = 0; g < kGroups; ++g)
                if (some(g))
#pragma unroll
                    for (int q = 0; q < kEach; ++q) sum[g][q] += x[k][g].get(q);
            if (!last_of_token(j)) continue;
            if (partly(j)) {
                float* row = a.partial + (2 * piece + (j >= tail ? 1 : 0)) * a.width;
#pragma unroll
                for (int g = 0; g < kGroups; ++g)
                    if (some(g)) at[g].template store<false>(row, sum[g]);
            } else {
                TE* row = row_of(j);
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {
                    if (!some(g)) continue;
#pragma unroll
                    for (int q = 0; q < kEach; ++q) sum[g][q] = sum[g][q] * a.scale + (kAccumulate ? was[k][g].get(q) : 0.f);
                    at[g].template store<kOut>(row, sum[g]);
                }
            }
            clear();
        }
    }
}

template <typename TY, typename TE, int kPiece, bool kAccumulate, bool kIn, bool kOut>
__global__ __launch_bounds__(kSumThreads) void sum_kernel(SumArgs a) {
    for (int64_t block = blockIdx.x; block < a.blocks; block += gridDim.x) {
        if (block >= a.sum_blocks) {
            const int64_t first = (block - a.sum_blocks) * a.zero_rows, v = first + threadIdx.x % kWave;
            zero_rows<TE, kOut>(a, first, __ballot(threadIdx.x % kWave < a.zero_rows && v < a.V && !a.present[v < a.V ? v : 0]));
        } else sum_piece<TY, TE, kPiece, kAccumulate, kIn, kOut>(a, block * (kSumThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave));
    }
}

// Up to kFew places: a wavefront to each (and tile) looks at all of them, and the one at a token's first place adds up its rows.  One
// launch, without an order: 64 or 256 places and 64 features, added, 13.1 and 14.9 -> 6.9 us, what the call takes the host; 256 places and
// 4096 features 15.9 -> 6.9; 64 places into 32000 x 2048 fp32 56.7 -> 51.9, rows of zeros (5.0 TB/s).  A frequent token is one
// wavefront's work: 256 places, a third of them one token's, 12 us (512 features) and 14 (4096), all of them 38.
constexpr int kFew = 256;

template <typename TY, typename TE, bool kAccumulate, bool kOut>
__global__ __launch_bounds__(kSumThreads) void few_kernel(SumArgs a, Tokens ids) {
    constexpr int N = 16 / sizeof(TY), kChunks = kFew / kWave;
    const int lane = threadIdx.x % kWave, T = static_cast<int>(a.T);
    uint32_t id[kChunks];
#pragma unroll
    for (int b = 0; b < kChunks; ++b) id[b] = b * kWave + lane < T ? ids[b * kWave + lane] : ids.V;
    for (int64_t block = blockIdx.x; block < a.blocks; block += gridDim.x) {
        if (block >= a.sum_blocks) {
            const int64_t first = (block - a.sum_blocks) * a.zero_rows;
            const int rows = static_cast<int>(a.V - first < a.zero_rows ? a.V - first : a.zero_rows);
            uint64_t mine = 0;
#pragma unroll
            for (int b = 0; b < kChunks; ++b) mine |= id[b] >= first && id[b] < first + rows ? uint64_t{1} << (id[b] - first) : 0;
            uint32_t low = static_cast<uint32_t>(mine), high = static_cast<uint32_t>(mine >> 32);
#pragma unroll
            for (int o = kWave / 2; o > 0; o >>= 1) {
                low |= __shfl_xor(low, o, kWave);
                high |= __shfl_xor(high, o, kWave);
            }
            const uint64_t present = static_cast<uint64_t>(__builtin_amdgcn_readfirstlane(high)) << 32 | static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(low));
            zero_rows<TE, kOut>(a, first, ~present & (rows == 64 ? ~uint64_t{0} : (uint64_t{1} << rows) - 1));
            continue;
        }
        const int64_t item = block * (kSumThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        const int place = static_cast<int>(item / a.tiles), tile = static_cast<int>(item % a.tiles);
        if (place >= T) continue;
        uint32_t v = ids.V;
        uint64_t same[kChunks];
#pragma unroll
        for (int b = 0; b < kChunks; ++b)
            if (place / kWave == b) v = __builtin_amdgcn_readlane(id[b], place % kWave);
        bool earlier = v >= ids.V;
#pragma unroll
        for (int b = 0; b < kChunks; ++b) {
            same[b] = __ballot(id[b] == v);
            const int before = place - b * kWave;  // places of the chunk that come before this one
            earlier |= (before >= kWave ? same[b] : before > 0 ? same[b] & ((uint64_t{1} << before) - 1) : 0) != 0;
        }
        if (earlier) continue;
        const Columns<N> at((static_cast<int64_t>(tile) * kWave + lane) * N, a.n);
        TE* const row = static_cast<TE*>(a.dE) + v * a.ldde;
        Raw<TE, N> was;
        if constexpr (kAccumulate) at.template load<false>(row, was);
        float sum[N];
#pragma unroll
        for (int q = 0; q < N; ++q) sum[q] = 0.f;
#pragma unroll
        for (int b = 0; b < kChunks; ++b)
            for (uint64_t left = same[b]; left;) {
                Raw<TY, N> x[kAhead];
                int count = 0;
#pragma unroll
                for (int k = 0; k < kAhead; ++k)
                    if (left) {
                        const int64_t t = b * kWave + __ffsll(static_cast<unsigned long long>(left)) - 1;
                        left &= left - 1;
                        ++count;
                        at.template load<false>(static_cast<const TY*>(a.dY) + t * a.lddy, x[k]);
                    }
#pragma unroll
                for (int k = 0; k < kAhead; ++k)
                    if (k < count)
#pragma unroll
                        for (int q = 0; q < N; ++q) sum[q] += x[k].get(q);
            }
#pragma unroll
        for (int q = 0; q < N; ++q) sum[q] = sum[q] * a.scale + (kAccumulate ? was.get(q) : 0.f);
        at.template store<false>(row, sum);
    }
}

// The partial sums of a long token, 256 columns a workgroup at a time: each wavefront adds up a share of the pieces in order, and the
// shares are added in order.  A very frequent token leaves narrow rows' sums to few workgroups: whole calls with Zipf's law alone / one
// token in 30 % of the places besides / in all of them, 65536 x 512 bf16 into fp32 55 / 69 / 99 us, 131072 x 4096 into bf16 315 / 325 / 375.
constexpr int kJoinThreads = 256, kJoinWaves = kJoinThreads / kWave;

template <typename TE, int kPiece, bool kAccumulate>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(SumArgs a) {
    __shared__ float4 part[kJoinWaves][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int64_t tiles = (static_cast<int64_t>(a.n) + 255) / 256, items = a.found[0] * tiles, T = a.found[1];
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t piece = a.list[item / tiles];
        const int64_t c = item % tiles * 256 + lane * 4;
        // the token of the piece's last place, and how many pieces behind it start within that token
        const uint32_t v = a.places[piece * kPiece + kPiece - 1].token;
        int64_t more = 0;
        for (;; more += kWave) {
            const int64_t i = (piece + 1 + more + lane) * kPiece;
            const uint64_t other = __ballot(i >= T || a.places[i].token != v);
            if (other) {
                more += __ffsll(static_cast<unsigned long long>(other)) - 1;
                break;
            }
        }
        // rows piece's second, then the first ones of those behind it
        const int64_t rows = more + 1, share = (rows + kJoinWaves - 1) / kJoinWaves;
        const int64_t from = wave * share, to = from + share < rows ? from + share : rows;
        float s[4] = {0.f, 0.f, 0.f, 0.f};
        for (int64_t i = from; i < to; i += 8) {
            float4 x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int64_t r = i + k < to ? i + k : to - 1;
                x[k] = *reinterpret_cast<const float4*>(a.partial + (2 * (piece + r) + (r == 0 ? 1 : 0)) * a.width + c);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (i + k < to) {
                    s[0] += x[k].x;
                    s[1] += x[k].y;
                    s[2] += x[k].z;
                    s[3] += x[k].w;
                }
        }
        part[wave][lane] = {s[0], s[1], s[2], s[3]};
        __syncthreads();
        if (wave == 0) {
            for (int w = 1; w < kJoinWaves; ++w) {
                const float4 p = part[w][lane];
                s[0] += p.x;
                s[1] += p.y;
                s[2] += p.z;
                s[3] += p.w;
            }
            TE* row = static_cast<TE*>(a.dE) + v * a.ldde;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (c + q < a.n) store_from_f32(row + c + q, s[q] * a.scale + (kAccumulate ? load_as_f32(row + c + q) : 0.f));
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------ workspace
constexpr int kSteps = 2;  // of a wavefront in a chunk of a sort over not too many places

struct Room {
    int64_t chunk, pieces, width;
    int bits, passes, blocks, piece;
    size_t places, counts, present, found, list, partial, bytes;  // where each starts (two lists of places)
};

Room room_of(int64_t T, int64_t V, int64_t n) {
    Room r{};
    int all = 0;
    while (V >> all) ++all;  // tokens 0 .. V - 1, and V for what is none
    r.passes = (all + kMostBits - 1) / kMostBits;
    r.bits = (all + r.passes - 1) / r.passes;
    r.chunk = kSteps * kSortThreads;
    while ((T + r.chunk - 1) / r.chunk > 256) r.chunk *= 2;
    r.blocks = T > 0 ? static_cast<int>((T + r.chunk - 1) / r.chunk) : 1;
    const int64_t tiles = (n + 511) / 512, few = 1023 / tiles * 32;
    r.width = tiles * 512;
    // Short pieces where pieces of 32 would be fewer than four wavefronts a compute unit: more of them, and more partial sums.  us with 8 / 32:
    // 2047 x 5461 28 / 36; 65536 x 512, twice that number, 82 / 67.
    r.piece = T <= few ? 8 : 32;
    r.pieces = (T + r.piece - 1) / r.piece;
    // (workspaces grow with T, so that one serves shorter batches, too)
    const int64_t least = ((T < few ? T : few) + 7) / 8, pieces = r.pieces > least ? r.pieces : least;
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t start = at;
        at += (bytes + 15) / 16 * 16;
        return start;
    };
    r.places = take(2 * static_cast<size_t>(T) * sizeof(Place));
    const int64_t blocks = (T + kSteps * kSortThreads - 1) / (kSteps * kSortThreads);
    r.counts = take((static_cast<size_t>(blocks > 256 ? 256 : blocks > 0 ? blocks : 1) << r.bits) * 4);
    r.present = take(static_cast<size_t>(V));
    r.found = take(8);
    r.list = take((static_cast<size_t>(pieces) + 1) * 4);
    r.partial = take(2 * static_cast<size_t>(pieces) * r.width * 4);
    r.bytes = at;
    return r;
}

// Workgroups for so many pieces, and for rows of zeros.
template <typename TY>
void divide(SumArgs& a, int64_t pieces, bool accumulate) {
    constexpr int N = 16 / sizeof(TY);
    a.tiles = static_cast<int>((static_cast<int64_t>(a.n) + kWave * N - 1) / (kWave * N));
    a.sum_blocks = (pieces * a.tiles + kSumThreads / kWave - 1) / (kSumThreads / kWave);
    a.zero_rows = a.n >= 2048 ? 8 : 16384 / a.n < 64 ? 16384 / a.n : 64;
    a.blocks = a.sum_blocks + (accumulate ? 0 : (static_cast<int64_t>(a.V) + a.zero_rows - 1) / a.zero_rows);
}

// Whether the streaming hint goes with dE.
template <typename TE>
bool large(const SumArgs& a) { return static_cast<double>(a.V) * a.n * sizeof(TE) > 1 << 25; }

template <typename TY, typename TE>
void launch_few(SumArgs a, const Tokens& ids, bool accumulate, hipStream_t s) {
    divide<TY>(a, a.T, accumulate);
    const unsigned blocks = walking_grid(a.blocks);
    if (accumulate) few_kernel<TY, TE, true, false><<<blocks, kSumThreads, 0, s>>>(a, ids);
    else if (large<TE>(a)) few_kernel<TY, TE, false, true><<<blocks, kSumThreads, 0, s>>>(a, ids);
    else few_kernel<TY, TE, false, false><<<blocks, kSumThreads, 0, s>>>(a, ids);
}

template <typename TY, typename TE, int kPiece, bool kAccumulate>
void launch_sums(SumArgs a, hipStream_t s) {
    divide<TY>(a, a.pieces, kAccumulate);
    const int64_t joins = (a.T / kPiece) * ((static_cast<int64_t>(a.n) + 255) / 256);
    // The streaming hint, for dE where it is large and for dY beyond half the cache.  us with neither / the first / both, bf16 into
    // 32000 rows, all with the hint on rows of zeros (8192 x 2048 into fp32 without it 73): 131072 x 4096 into bf16 335 / 326 / 314;
    // into fp32 65536 x 512 68.5 / 57.0 / 68.3, 65536 x 1024 95.3 / 93.9 / 91.7, 65536 x 2048 150 / 148 / 146, 8192 x 1024 36.0 / 37.9 /
    // 43.3, 8192 x 2048 59.2 / 63.2 / 77.7.
    const bool out = large<TE>(a), in = static_cast<double>(a.T) * a.n * sizeof(TY) > kStreamed;
    const unsigned blocks = walking_grid(a.blocks);
    if (kPiece == 32 && in && out) sum_kernel<TY, TE, kPiece, kAccumulate, kPiece == 32, true><<<blocks, kSumThreads, 0, s>>>(a);
    else if (out) sum_kernel<TY, TE, kPiece, kAccumulate, false, true><<<blocks, kSumThreads, 0, s>>>(a);
    else sum_kernel<TY, TE, kPiece, kAccumulate, false, false><<<blocks, kSumThreads, 0, s>>>(a);
    if (joins) join_kernel<TE, kPiece, kAccumulate><<<walking_grid(joins, 8 * kUnits), kJoinThreads, 0, s>>>(a);
}

}  // namespace

size_t embed_backward_workspace_bytes(int64_t T, int64_t V, int64_t n) { return room_of(T, V, n).bytes; }

grass_status launch_embed_backward(const void* dY, grass_dtype dt, int64_t lddy, const void* ids, grass_index idt, int64_t T,
                                   int64_t V, int64_t n, float scale, bool accumulate, void* dE, grass_dtype gdt,
                                   int64_t ldde, void* ws, hipStream_t s) {
    if (T == 0 && accumulate) return GRASS_OK;
    const Room r = room_of(T, V, n);
    char* base = static_cast<char*>(ws);
    Place* places = reinterpret_cast<Place*>(base + r.places);
    uint8_t* present = accumulate ? nullptr : reinterpret_cast<uint8_t*>(base + r.present);
    uint32_t* found = reinterpret_cast<uint32_t*>(base + r.found);
    SortArgs sort{tokens(ids, idt, V), nullptr, places, T, r.chunk, 0, r.bits, r.blocks, reinterpret_cast<uint32_t*>(base + r.counts),
                  present, found};
    const int64_t ranges = (V + kRange - 1) / kRange;
    // One kernel does as much as there are ranges times places.  us of whole calls with it / with the radix sort, 64 bf16 features:
    // 32000 tokens 16384 places 24.4 / 45.6, 32768 39.5 / 45.7, 65536 51.9 / 52.8; 128000 tokens 16384 places 29.4 / 36.4, 65536 66.8 / 61.2.
    if (T > kFew && T <= 32768 && ranges * T <= (1 << 23)) {
        static_assert((1 << 23) / kFew < (int64_t{1} << 32) / kSortThreads, "a grid has fewer than 2^32 threads");
        order_kernel<<<static_cast<unsigned>(ranges), kSortThreads, 0, s>>>(sort);
    } else if (T > kFew) {
        const unsigned grid = static_cast<unsigned>(r.blocks);
        for (int pass = 0; pass < r.passes; ++pass) {
            sort.shift = pass * r.bits;
            sort.from = pass == 0 ? nullptr : places + (pass - 1) % 2 * T;
            sort.to = places + pass % 2 * T;
            if (r.chunk == kSteps * kSortThreads) {
                count_kernel<kSteps><<<grid, kSortThreads, 0, s>>>(sort);
                scatter_kernel<kSteps><<<grid, kSortThreads, 0, s>>>(sort);
            } else {
                count_kernel<0><<<grid, kSortThreads, 0, s>>>(sort);
                scatter_kernel<0><<<grid, kSortThreads, 0, s>>>(sort);
            }
        }
    }
    const SumArgs a{dY, dE, lddy, ldde, T, r.pieces, static_cast<int>(n), 0, static_cast<uint32_t>(V), scale, sort.to, present, found,
                    reinterpret_cast<uint32_t*>(base + r.list), reinterpret_cast<float*>(base + r.partial), r.width, 0, 0, 0};
    const auto go = [&](auto from, auto to) {
        typedef decltype(from) TY;
        typedef decltype(to) TE;
        if (T <= kFew) return launch_few<TY, TE>(a, sort.ids, accumulate, s);
        if (r.piece == 8) accumulate ? launch_sums<TY, TE, 8, true>(a, s) : launch_sums<TY, TE, 8, false>(a, s);
        else accumulate ? launch_sums<TY, TE, 32, true>(a, s) : launch_sums<TY, TE, 32, false>(a, s);
    };
    if (dt == GRASS_F32) gdt == GRASS_F32 ? go(float{}, float{}) : go(float{}, uint16_t{});
    else gdt == GRASS_F32 ? go(uint16_t{}, float{}) : go(uint16_t{}, uint16_t{});
    return launch_status();
}

}  // namespace grass
