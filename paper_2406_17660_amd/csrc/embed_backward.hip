// grass_embed_backward: the gradient of the embedding, summed by tokens.
//
// The places of the batch are sorted by token (stably, so that a token's places stay in order), and the rows of dY are then
// read once in that order, each piece of kPiece places by a wavefront that adds the rows of a token up in registers.  Tokens of up
// to kPiece places are summed and stored by the wavefront whose piece has the first of them; longer ones, the
// frequent ones, leave a partial sum a piece, which a second kernel adds up in order.  All sums are fp32.
//
// Bound by memory: dY is read once, dE written once.
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
    uint32_t* longs;    // how many tokens have more than kPiece places: 0 here
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

// f(i, place, digit, lanes of the same digit) for 64 places at a time of the wavefront's share of the workgroup's chunk.
template <typename F>
__device__ __forceinline__ void each_place(const SortArgs& a, F f) {
    const int64_t share = a.chunk / kSortWaves, start = blockIdx.x * a.chunk + threadIdx.x / kWave * share;
    for (int64_t at = start; at < start + share && at < a.T; at += kWave) {
        const int64_t i = at + threadIdx.x % kWave;
        const bool there = i < a.T;
        const Place p = there ? place_at(a, i) : Place{0, 0};
        const uint32_t digit = p.token >> a.shift & ((1u << a.bits) - 1);
        f(p, digit, same_digit(digit, a.bits, there), there);
    }
}

__global__ __launch_bounds__(kSortThreads) void count_kernel(SortArgs a) {
    __shared__ uint32_t count[kMostBins];
    const uint32_t bins = 1u << a.bits;
    if (threadIdx.x < bins) count[threadIdx.x] = 0;
    if (!a.from) {  // what later kernels start from
        if (blockIdx.x == 0 && threadIdx.x == 0) *a.longs = 0;
        if (a.present)
            for (int64_t v = (static_cast<int64_t>(blockIdx.x) * kSortThreads + threadIdx.x) * 16; v < a.ids.V;
                 v += static_cast<int64_t>(gridDim.x) * kSortThreads * 16)
                *reinterpret_cast<uint4*>(a.present + v) = {0, 0, 0, 0};
    }
    __syncthreads();
    each_place(a, [&](Place, uint32_t digit, uint64_t same, bool there) {
        if (there && (same & ((uint64_t{1} << threadIdx.x % kWave) - 1)) == 0) atomicAdd(&count[digit], __popcll(same));
    });
    __syncthreads();
    if (threadIdx.x < bins) a.counts[blockIdx.x * bins + threadIdx.x] = count[threadIdx.x];
}

__global__ __launch_bounds__(kSortThreads) void scatter_kernel(SortArgs a) {
    __shared__ uint32_t next[kSortWaves][kMostBins], before[kSortThreads], all[kSortThreads], sums[kSortWaves];
    const uint32_t bins = 1u << a.bits, wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    // all counts of a digit, and those of the workgroups before this one, by several threads
    const uint32_t digit = threadIdx.x & (bins - 1), groups = kSortThreads / bins, group = threadIdx.x / bins;
    uint32_t b = 0, n = 0;
#pragma unroll 8
    for (uint32_t k = group; k < static_cast<uint32_t>(a.blocks); k += groups) {
        const uint32_t c = a.counts[k * bins + digit];
        n += c;
        b += k < blockIdx.x ? c : 0;
    }
    before[threadIdx.x] = b;
    all[threadIdx.x] = n;
    for (uint32_t k = threadIdx.x; k < kSortWaves * kMostBins; k += kSortThreads) (&next[0][0])[k] = 0;
    __syncthreads();
    each_place(a, [&](Place, uint32_t d, uint64_t same, bool there) {
        if (there && (same & ((uint64_t{1} << lane) - 1)) == 0) next[wave][d] += __popcll(same);
    });
    if (threadIdx.x < bins)
        for (uint32_t g = 1; g < groups; ++g) {
            b += before[threadIdx.x + g * bins];
            n += all[threadIdx.x + g * bins];
        }
    const uint32_t upto = wave_inclusive_scan(threadIdx.x < bins ? n : 0u);
    if (lane == kWave - 1) sums[wave] = upto;
    __syncthreads();
    if (threadIdx.x < bins) {
        uint32_t at = upto - n + b;
        for (uint32_t w = 0; w < wave; ++w) at += sums[w];
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = next[w][threadIdx.x];
            next[w][threadIdx.x] = at;
            at += c;
        }
    }
    __syncthreads();
    each_place(a, [&](Place p, uint32_t d, uint64_t same, bool there) {
        if (!there) return;
        const uint64_t lower = same & ((uint64_t{1} << lane) - 1);
        const uint32_t at = next[wave][d];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (lower == 0) next[wave][d] = at + __popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        a.to[at + __popcll(lower)] = p;
        if (!a.from && a.present && p.token < a.ids.V) a.present[p.token] = 1;
    });
}

// ----------------------------------------------------------------------------------------- sums
constexpr int kPiece = 32, kAhead = 8, kSumThreads = 256;

struct SumArgs {
    const void* dY;
    void* dE;
    int64_t lddy, ldde, T, pieces;
    int n, tiles;
    uint32_t V;
    float scale;
    const Place* places;
    const uint8_t* present;
    uint32_t *longs, *list;  // pieces in which a token of more than kPiece places starts
    float* partial;          // two rows a piece: of the token that it starts within, and of the long one that starts in it
    int64_t width;           // floats of such a row
    int64_t sum_blocks, blocks;  // that add up pieces, and with those that write zeros
    int zero_rows;               // of dE, for one of these
};

// The N columns of a lane: the row's last N where fewer are left, of which the first `skip` are another lane's.
template <typename T, int N>
__device__ __forceinline__ void add_to_row(T* row, int n, int64_t at, int skip, const float (&x)[N], bool accumulate) {
    if (skip >= N) return;
    float z[N];
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = x[i];
    Raw<T, N> r;
    if (skip == 0 && n >= N) {
        if (accumulate) {
            r.load(row + at);
#pragma unroll
            for (int i = 0; i < N; ++i) z[i] += r.get(i);
        }
        r.set(z);
        r.store(row + at);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i >= skip && at + i < n) store_from_f32(row + at + i, accumulate ? z[i] + load_as_f32(row + at + i) : z[i]);
}

// Zeros in the rows of tokens that do not occur, kSumThreads to a row.
template <typename TE>
__device__ __forceinline__ void zero_rows(const SumArgs& a, int64_t block) {
    const int64_t first = block * a.zero_rows, end = first + a.zero_rows < a.V ? first + a.zero_rows : a.V;
    for (int64_t v = first; v < end; ++v) {
        if (a.present[v]) continue;
        TE* row = static_cast<TE*>(a.dE) + v * a.ldde;
        Raw<TE, 8> zero;
        zero.zero();
        for (int64_t c = threadIdx.x * 8; c < a.n; c += kSumThreads * 8) {
            if (c + 8 <= a.n) zero.store(row + c);
            else zero.store_some(row + c, static_cast<int>(a.n - c));
        }
    }
}

// A wavefront's work: the columns of a tile in a piece.
template <typename TY, typename TE, bool kAccumulate>
__device__ __forceinline__ void sum_piece(const SumArgs& a, int64_t item) {
    constexpr int N = 16 / sizeof(TY);
    const int lane = threadIdx.x % kWave;
    const int64_t piece = item / a.tiles;
    const int tile = static_cast<int>(item - piece * a.tiles);
    if (piece >= a.pieces) return;
    // the piece's places and as many behind it; a start is a place whose token is not the one before's
    const int64_t p0 = piece * kPiece;
    const auto token_at = [&](int64_t i) { return i < 0 ? 0xFFFFFFFEu : i < a.T ? a.places[i].token : 0xFFFFFFFFu; };
    const int64_t mine = p0 + lane;
    const Place here = mine < a.T ? a.places[mine] : Place{0xFFFFFFFFu, 0};
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
    if (tail < end && tile == 0 && lane == 0) a.list[atomicAdd(a.longs, 1u)] = static_cast<uint32_t>(piece);

    const int64_t c = (static_cast<int64_t>(tile) * kWave + lane) * N, at = c + N <= a.n ? c : a.n > N ? a.n - N : 0;
    const int skip = static_cast<int>(c - at);
    float sum[N];
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = 0.f;
    const TY* column = static_cast<const TY*>(a.dY) + at;
    for (int i = begin; i < end; i += kAhead) {
        Raw<TY, N> x[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const uint32_t t = __builtin_amdgcn_readlane(here.t, i + k < end ? i + k : end - 1);
            if (a.n >= N) x[k].load(column + t * a.lddy);
            else x[k].load_some(column + t * a.lddy, a.n);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int j = i + k;
            if (j >= end) break;
#pragma unroll
            for (int q = 0; q < N; ++q) sum[q] += x[k].get(q);
            if (j + 1 < end && !(starts >> (j + 1) & 1)) continue;
            // the token's last place here
            if (j < first || j >= tail) {
                float* out = a.partial + (2 * piece + (j >= tail ? 1 : 0)) * a.width + at;
#pragma unroll
                for (int q = 0; q < N; ++q)
                    if (q >= skip) out[q] = sum[q];
            } else {
#pragma unroll
                for (int q = 0; q < N; ++q) sum[q] *= a.scale;
                const uint32_t v = __builtin_amdgcn_readlane(here.token, j);
                add_to_row<TE, N>(static_cast<TE*>(a.dE) + v * a.ldde, a.n, at, skip, sum, kAccumulate);
            }
#pragma unroll
            for (int q = 0; q < N; ++q) sum[q] = 0.f;
        }
    }
}

template <typename TY, typename TE, bool kAccumulate>
__global__ __launch_bounds__(kSumThreads) void sum_kernel(SumArgs a) {
    for (int64_t block = blockIdx.x; block < a.blocks; block += gridDim.x) {
        if (block >= a.sum_blocks) zero_rows<TE>(a, block - a.sum_blocks);
        else sum_piece<TY, TE, kAccumulate>(a, block * (kSumThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave));
    }
}

// The partial sums of a long token, 256 columns a workgroup at a time: each wavefront adds up a share of the pieces in order, and the
// shares are added in order.
constexpr int kJoinThreads = 512, kJoinWaves = kJoinThreads / kWave;

template <typename TE, bool kAccumulate>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(SumArgs a) {
    __shared__ float4 part[kJoinWaves][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int64_t tiles = (static_cast<int64_t>(a.n) + 255) / 256, items = *a.longs * tiles;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t piece = a.list[item / tiles];
        const int64_t c = item % tiles * 256 + lane * 4;
        // the token of the piece's last place, and how many pieces behind it start within that token
        const uint32_t v = a.places[piece * kPiece + kPiece - 1].token;
        int64_t more = 0;
        for (;; more += kWave) {
            const int64_t i = (piece + 1 + more + lane) * kPiece;
            const uint64_t other = __ballot(i >= a.T || a.places[i].token != v);
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
struct Room {
    int64_t chunk, pieces, width;
    int bits, passes, blocks, tiles;
    size_t places, counts, present, longs, list, partial, bytes;  // where each starts (two lists of places)
};

Room room_of(int64_t T, int64_t V, int64_t n) {
    Room r{};
    int all = 0;
    while (V >> all) ++all;  // tokens 0 .. V - 1, and V for what is none
    r.passes = (all + kMostBits - 1) / kMostBits;
    r.bits = (all + r.passes - 1) / r.passes;
    r.chunk = 2 * kSortThreads;
    while ((T + r.chunk - 1) / r.chunk > 256) r.chunk *= 2;
    r.blocks = T > 0 ? static_cast<int>((T + r.chunk - 1) / r.chunk) : 1;
    r.pieces = (T + kPiece - 1) / kPiece;
    r.tiles = static_cast<int>((n + kWave * 4 - 1) / (kWave * 4));  // of 4 columns a lane; half as many of 8
    r.width = (static_cast<int64_t>(r.tiles) * kWave * 4 + 511) / 512 * 512;
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t start = at;
        at += (bytes + 15) / 16 * 16;
        return start;
    };
    r.places = take(2 * static_cast<size_t>(T) * sizeof(Place));
    r.counts = take((static_cast<size_t>(r.blocks) << r.bits) * 4);
    r.present = take(static_cast<size_t>(V));
    r.longs = take(4);
    r.list = take((static_cast<size_t>(T) / kPiece + 1) * 4);
    r.partial = take(2 * static_cast<size_t>(r.pieces) * r.width * 4);
    r.bytes = at;
    return r;
}

template <typename TY, typename TE>
void launch_sums(SumArgs a, bool accumulate, hipStream_t s) {
    constexpr int N = 16 / sizeof(TY);
    a.tiles = static_cast<int>((static_cast<int64_t>(a.n) + kWave * N - 1) / (kWave * N));
    a.sum_blocks = (a.pieces * a.tiles + kSumThreads / kWave - 1) / (kSumThreads / kWave);
    a.zero_rows = a.n >= 2048 ? 8 : 16384 / a.n < 256 ? 16384 / a.n : 256;
    a.blocks = a.sum_blocks + (accumulate ? 0 : (a.V + a.zero_rows - 1) / a.zero_rows);
    const unsigned blocks = static_cast<unsigned>(a.blocks < kMostBlocks ? a.blocks : kMostBlocks);
    const int64_t joins = (a.T / kPiece) * ((static_cast<int64_t>(a.n) + 255) / 256);
    const unsigned grid = static_cast<unsigned>(joins < 4 * kUnits ? joins : 4 * kUnits);
    if (accumulate) {
        sum_kernel<TY, TE, true><<<blocks, kSumThreads, 0, s>>>(a);
        if (grid) join_kernel<TE, true><<<grid, kJoinThreads, 0, s>>>(a);
    } else {
        sum_kernel<TY, TE, false><<<blocks, kSumThreads, 0, s>>>(a);
        if (grid) join_kernel<TE, false><<<grid, kJoinThreads, 0, s>>>(a);
    }
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
    uint32_t* longs = reinterpret_cast<uint32_t*>(base + r.longs);
    SortArgs sort{tokens(ids, idt, V), nullptr, places, T, r.chunk, 0, r.bits, r.blocks, reinterpret_cast<uint32_t*>(base + r.counts),
                  present, longs};
    const unsigned grid = static_cast<unsigned>(r.blocks);
    for (int pass = 0; pass < r.passes; ++pass) {
        sort.shift = pass * r.bits;
        sort.from = pass == 0 ? nullptr : places + (pass - 1) % 2 * T;
        sort.to = places + pass % 2 * T;
        count_kernel<<<grid, kSortThreads, 0, s>>>(sort);
        scatter_kernel<<<grid, kSortThreads, 0, s>>>(sort);
    }
    const SumArgs a{dY, dE, lddy, ldde, T, r.pieces, static_cast<int>(n), 0, static_cast<uint32_t>(V), scale, sort.to, present, longs,
                    reinterpret_cast<uint32_t*>(base + r.list), reinterpret_cast<float*>(base + r.partial), r.width, 0, 0, 0};
    const auto go = [&](auto from, auto to) { launch_sums<decltype(from), decltype(to)>(a, accumulate, s); };
    if (dt == GRASS_F32) gdt == GRASS_F32 ? go(float{}, float{}) : go(float{}, uint16_t{});
    else gdt == GRASS_F32 ? go(uint16_t{}, float{}) : go(uint16_t{}, uint16_t{});
    return launch_status();
}

}  // namespace grass
