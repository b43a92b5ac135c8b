// Low-rank adapters of many requests beside a shared projection, and their gradients.
//
// Token t has the adapter a = index[t] (none where a is outside 0 .. N - 1).  With A_a (R x n), B_a (m x R) and a factor s_a:
//
//   forward    hidden_t = A_a x_t                  y_t = base_t + s_a B_a hidden_t
//   backward   d_t = s_a B_a^T dy_t                dx_t = base_t + A_a^T d_t
//              dA_a = sum over a's tokens of d_t x_t^T      dB_a = s_a sum over a's tokens of dy_t hidden_t^T
//
// Three kernels do all of it.  `shrink` contracts over the long axis (A_a x_t, B_a^T dy_t), `expand` goes back to a long axis (B_a hidden_t,
// A_a^T d_t), `outer` adds up the outer products of the tokens of one adapter.  x, dy, base and y are read and written once per use and the
// weights of the adapters that occur come from the caches after their first use, so that the activations' bytes bound the large calls,
// the latency of two launches the small ones.
//
// Tokens stay in their own order: a workgroup takes 16, 32 or 64 neighbours, lists the adapters that occur among them, and its waves share
// out the pairs of adapter and piece of the axis.  Requests are runs of tokens, so that the list mostly has one or two entries in a batch
// of prompts, and up to 16 in a decode step, where the adapters' own bytes are what has to be read anyway.  A product of a 16 x 16 tile has the
// adapter's rows on one side and the tokens on the other: a token of another adapter is a column of its own whose result is not kept, so
// that nothing of one request (a NaN, say) reaches another one.
//
// Measured, per call back to back (a large copy reaches 5.0 TB/s on the same card): one token, 2048 -> 2048, rank 16: 9.7 us, two launches that depend on one
// another; 64 requests of 48 adapters, 9216 -> 4096, rank 16: 21 us; 3136 tokens in columns, 4096 -> 4096, rank 16: 62 us, 2.4 TB/s; 8192 tokens in bf16
// rows, rank 64: 84 us, 2.5 TB/s; backward of 4096 tokens in bf16 rows, 9216 -> 4096, rank 32: 107 us, 2.5 TB/s.
//
// `shrink`: activations in 32 bits are multiplied by the 32-bit matrix instruction, in 16 bits by the 16-bit one, by weights of the same type; both add up in 32.
// hidden and d are kept in 32 bits.  What follows them, `expand` and `outer`, uses the 32-bit instruction for up to 256 tokens and for the gradients of activations in
// 32 bits; else numbers go into the 16-bit one as bf16 pieces that hold all their bits (pieces_of), and a sum that an infinity has reached is formed again by
// the 32-bit one.
#include <algorithm>
#include <type_traits>

#include "adapter_weights.hpp"

namespace cer {
namespace {

using F4 = Vec<float, 4>;
constexpr int kBlock = 256, kWaves = kBlock / 64;
template <int kTiles>
constexpr int kShrinkThreads = kTiles == 1 ? 1024 : 512;
constexpr int kOuterBlock = 256, kRowsBlock = 512;
constexpr int kMostTile = 64;  // tokens of a workgroup
// Up to so many tokens the kernels for 16 of them run, tiles of 64 would be too few for the chip.  Where the one is as fast as the other depends on the order and the
// requests too: 4096 -> 4096 features, these kernels against those, 320 tokens of 8 requests, columns, rank 16: 21.5 and 31.7 us, of one request, bf16, rank 64: 27.4
// and 19.8; 512 tokens: 26.4 and 18.0, 36.1 and 19.0.  The line is where neither loses yet, and the first of these cases is slower than it could be.
constexpr int64_t kFewTokens = 256;

// One side's weights: element (long axis k, rank r) of adapter a at w[a * stride + (kAlong ? r * ld + k : k * ld + r)].
struct Weights {
    const void* w;
    int64_t stride, ld;
    const int32_t* ranks;  // per adapter; nullptr: all `rank`
    const float* scales;   // nullptr: 1
    int32_t adapters, rank;
};

__device__ __forceinline__ int rank_of(const Weights& w, int a) {
    if (!w.ranks) return w.rank;
    const int r = w.ranks[a];
    return r < 0 ? 0 : r > w.rank ? w.rank : r;
}
__device__ __forceinline__ float scale_of(const Weights& w, int a) { return w.scales ? w.scales[a] : 1.f; }

// The adapter of a token; -1: none, and past the last token.
__device__ __forceinline__ int adapter_at(const int32_t* index, int64_t t, int64_t tokens, int32_t adapters) {
    const int a = t < tokens ? index[t] : -1;
    return a >= 0 && a < adapters ? a : -1;
}

// The adapters among a workgroup's tokens, each once, in the order of their first tokens; one wave makes the list for all.
struct alignas(16) Present {
    int adapter[kMostTile];  // of each token
    int slot[kMostTile];     // the adapters
    int slots;
    int none;  // whether a token of the batch has none
};
__device__ __forceinline__ void list_adapters(Present& p, const int32_t* index, int64_t t0, int tile, int64_t tokens, int32_t adapters) {
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x;
        const int a = lane < tile ? adapter_at(index, t0 + lane, tokens, adapters) : -1;
        if (lane < tile) p.adapter[lane] = a;
        unsigned long long left = __ballot(a >= 0);
        int n = 0;
        while (left) {
            const int of = __shfl(a, __ffsll(left) - 1);
            if (lane == 0) p.slot[n] = of;
            ++n;
            left &= ~__ballot(a == of);
        }
        const bool none = __ballot(lane < tile && t0 + lane < tokens && a < 0) != 0;
        if (lane == 0) {
            p.slots = n;
            p.none = none;
        }
    }
    __syncthreads();
}

__device__ __forceinline__ F4 product(float a, float b, F4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
__device__ __forceinline__ F4 product(Vec<__bf16, 8> a, Vec<__bf16, 8> b, F4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ F4 product(Vec<_Float16, 8> a, Vec<_Float16, 8> b, F4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// Workgroup n of `all` as neighbours want it: the eight XCDs take workgroups in turn and have an L2 each, so that an eighth of the work items, one after the
// other, goes to each: neighbouring tokens mostly have the same adapter, and its weights then come into one L2 or two and not into all of them.
__device__ __forceinline__ unsigned by_xcd(unsigned n, unsigned all) {
    const unsigned each = all / 8, more = all % 8, xcd = n % 8;
    return xcd * each + (xcd < more ? xcd : more) + n / 8;
}

// ---- shrink ---------------------------------------------------------------------------------------------------------------------
struct ShrinkArgs {
    Weights w;
    const int32_t* index;
    int64_t tokens, length;  // of the long axis
    const void* x;
    int64_t ldx;
    int64_t part;    // elements of the long axis for a workgroup, a multiple of 32 (few tokens), of 128 (rows) or (columns) of 512, two steps for each of eight waves, or 256
    uint32_t parts;  // of the long axis
    float* out;      // [parts][tokens][rank]
    bool scale;      // times s_a
};

// Few tokens (kTiles = 1), and columns of many (4): kTiles * 16 tokens, kRanks * 16 ranks from blockIdx.z on; the waves share out the adapters and pieces
// of the workgroup's part of the long axis.  Lane (i, g) = (lane % 16, lane / 16) holds of both sides' operands row i's (a rank's, a token's) eight elements of 32 of the long axis
// that belong to g: one 16-bit instruction, or eight 32-bit ones that take one of every g's.  The sides agree on which, and that is all that
// their order has to do.  Columns: x of 3136 x 4096 in 28 us, 1.8 TB/s; a tile of one request's end and the next one's start reads its x again for each
// adapter, from L2 (16 requests 62 us for both launches, one 47).  Few tokens: 64 of 9216 features, 48 adapters (14 MB) in 11 us: each wave's lines of the adapters'
// rows pass the address unit one by one.  Rows of ranks: 16 r + i, or where a rank's elements lie apart (!kAlong) kRanks i + r, neighbours in one load.
template <class TX, class TW, bool kColumns, bool kAlong, int kTiles, int kRanks>
__global__ __launch_bounds__(kShrinkThreads<kTiles>, kTiles * kRanks >= 16 ? 2 : 4) void shrink_kernel(ShrinkArgs c) {
    constexpr bool k16 = sizeof(TX) == 2;
    constexpr int E = 8, kStep = 4 * E, kTile = 16 * kTiles, kThreads = kShrinkThreads<kTiles>, kWaves = kThreads / 64;
    using Operand = std::conditional_t<k16, Vec<TX, E>, Vec<float, E>>;
    __shared__ Present present;
    __shared__ F4 sums[kWaves / 2][kTiles * kRanks][64];
    const unsigned item = by_xcd(blockIdx.x, gridDim.x), part = item % c.parts;
    const int64_t t0 = (int64_t)(item / c.parts) * kTile;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4, r0 = blockIdx.z * 16 * kRanks;
    list_adapters(present, c.index, t0, kTile, c.tokens, c.w.adapters);
    const int slots = __builtin_amdgcn_readfirstlane(present.slots);
    // the workgroup's part of the long axis; its waves take turns, so that together they read neighbouring lines, or, few tokens, a stretch each
    const int from = part * (int)c.part, to = std::min<int64_t>(from + c.part, c.length);
    constexpr int kAhead = kTiles * kRanks <= 2 ? 4 : kTiles * kRanks <= (kTiles == 1 && !k16 ? 4 : 8) ? 2 : 1;  // steps whose loads are on their way together
    constexpr int kRun = kAhead * kStep;
    const int want = slots > 8 ? 16 : slots > 4 ? 8 : slots > 2 ? 4 : slots > 1 ? 2 : 1;
    const int runs = kTiles > 1 ? (to - from + kRun - 1) / kRun : 1;  // many tokens: as many abreast as leave every wave a run
    const int abreast = std::min(want, runs > 4 ? 1 : runs > 2 ? 2 : runs > 1 ? 4 : kWaves), pieces = kWaves / abreast, piece = wave / abreast;
    const int stretch = kTiles == 1 ? ((to - from + pieces - 1) / pieces + kStep - 1) / kStep * kStep : kRun;
    const int k_first = from + piece * stretch, k_last = kTiles == 1 ? std::min(k_first + stretch, to) : to, k_next = kTiles == 1 ? kRun : pieces * kRun;
    int token[kTiles];  // in the tile
#pragma unroll
    for (int s = 0; s < kTiles; ++s) token[s] = kColumns ? kTiles * i + s : 16 * s + i;
    const int tokens_left = (int)std::min<int64_t>(c.tokens - t0, kTile), abreast_left = tokens_left - kTiles * i;
    // a lane's place: the rest of an address is the wave's
    const TX* x = static_cast<const TX*>(c.x) + (kColumns ? t0 : t0 * c.ldx);
    uint32_t x_lane[kTiles];
    if (kColumns) {
        x_lane[0] = (uint32_t)(E * g * c.ldx + (abreast_left > 0 ? kTiles * i : 0)) * sizeof(TX);
    } else {
#pragma unroll
        for (int s = 0; s < kTiles; ++s) x_lane[s] = (uint32_t)(std::min(token[s], tokens_left - 1) * c.ldx + E * g) * sizeof(TX);
    }
    float* out = c.out + part * c.tokens * c.w.rank;
    for (int first = 0; first < slots; first += abreast) {
        const int q = first + wave % abreast;
        const int a = q < slots ? __builtin_amdgcn_readfirstlane(present.slot[q]) : -1;
        const int rank = a >= 0 ? rank_of(c.w, a) : 0;
        F4 acc[kTiles][kRanks];
#pragma unroll
        for (int s = 0; s < kTiles; ++s)
#pragma unroll
            for (int r = 0; r < kRanks; ++r) acc[s][r] = 0.f;
        if (rank > r0) {
            const TW* w = static_cast<const TW*>(c.w.w) + a * c.w.stride + (kAlong ? r0 * c.w.ld : r0);
            uint32_t w_lane[kRanks];  // kAlong: of a rank past the last one: the last one's, its products are not kept
            if (kAlong) {
#pragma unroll
                for (int r = 0; r < kRanks; ++r) w_lane[r] = (uint32_t)(std::min(16 * r + i, rank - r0 - 1) * c.w.ld + E * g) * sizeof(TW);
            } else {
                w_lane[0] = (uint32_t)(E * g * c.w.ld + kRanks * i) * sizeof(TW);
            }
            const int ranks_left = rank - r0 - kRanks * i;
            const bool ranks_whole = rank - r0 >= 16 * kRanks;
            auto step = [&](int k, auto whole) {  // whole: nothing of the step is past the end
                constexpr bool kWhole = decltype(whole)::value;
                const int left = kWhole ? E : to - (k + E * g);
                Operand xs[kTiles], ws[kRanks];
                if constexpr (kColumns) {
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        Vec<float, 4> v = 0.f;
                        if (kWhole || j < left) {
                            const TX* p = at(x + (k + j) * c.ldx, x_lane[0]);
                            if constexpr (kTiles == 1) v[0] = p[0];
                            if constexpr (kTiles == 4) v = load_some<TX, 4>(p, abreast_left);
                        }
#pragma unroll
                        for (int s = 0; s < kTiles; ++s) xs[s][j] = v[s];
                    }
                } else {
#pragma unroll
                    for (int s = 0; s < kTiles; ++s) {
                        if constexpr (k16) xs[s] = load_own<TX, E>(at(x + k, x_lane[s]), left);
                        else xs[s] = load_some<TX, E>(at(x + k, x_lane[s]), left);
                    }
                }
                if constexpr (kAlong) {
#pragma unroll
                    for (int r = 0; r < kRanks; ++r) {
                        if constexpr (k16) ws[r] = load_own<TW, E>(at(w + k, w_lane[r]), left);
                        else ws[r] = load_some<TW, E>(at(w + k, w_lane[r]), left);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        Vec<TW, kRanks> v = (TW)0.f;
                        const TW* p = at(w + (k + j) * c.w.ld, w_lane[0]);
                        if (kWhole && ranks_whole) v = load<TW, kRanks>(p);
                        else if (kWhole || j < left) v = load_own<TW, kRanks>(p, ranks_left);
#pragma unroll
                        for (int r = 0; r < kRanks; ++r) {
                            if constexpr (k16) ws[r][j] = v[r];
                            else ws[r][j] = (float)v[r];
                        }
                    }
                }
#pragma unroll
                for (int s = 0; s < kTiles; ++s)
#pragma unroll
                    for (int r = 0; r < kRanks; ++r) {
                        if constexpr (k16) {
                            acc[s][r] = product(ws[r], xs[s], acc[s][r]);
                        } else {
#pragma unroll
                            for (int j = 0; j < E; ++j) acc[s][r] = product(ws[r][j], xs[s][j], acc[s][r]);
                        }
                    }
            };
            int k = k_first;
            for (; k + kRun <= k_last; k += k_next)
#pragma unroll
                for (int u = 0; u < kAhead; ++u) step(k + u * kStep, std::true_type());
            if (k < k_last) {  // the last run, by the wave whose turn it is
                const int end = std::min(k + kRun, k_last);
                if constexpr (kAhead > 1)
#pragma unroll 1
                    for (; k + kStep <= end; k += kStep) step(k, std::true_type());
                if (k < end) step(k, std::false_type());
            }
        }
        // the pieces of an adapter: the upper half's sums to the lower half's, until there is one
        for (int half = pieces / 2; half; half /= 2) {
            if (piece >= half && piece < 2 * half)
#pragma unroll
                for (int s = 0; s < kTiles; ++s)
#pragma unroll
                    for (int r = 0; r < kRanks; ++r) sums[wave - half * abreast][s * kRanks + r][lane] = acc[s][r];
            __syncthreads();
            if (piece < half)
#pragma unroll
                for (int s = 0; s < kTiles; ++s)
#pragma unroll
                    for (int r = 0; r < kRanks; ++r) acc[s][r] += sums[wave][s * kRanks + r][lane];
            __syncthreads();
        }
        if (piece == 0 && rank > r0) {
            const float scale = c.scale ? scale_of(c.w, a) : 1.f;
#pragma unroll
            for (int s = 0; s < kTiles; ++s) {
                if (present.adapter[token[s]] != a) continue;
                float* to_token = out + (t0 + token[s]) * c.w.rank + r0;
#pragma unroll
                for (int r = 0; r < kRanks; ++r)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int at_r = kAlong ? 16 * r + 4 * g + e : kRanks * (4 * g + e) + r;
                        if (r0 + at_r < c.w.rank) to_token[at_r] = r0 + at_r < rank ? acc[s][r][e] * scale : 0.f;
                    }
            }
        }
    }
    // tokens without an adapter, or without ranks here
    for (int e = threadIdx.x; e < kTile * 16 * kRanks; e += kThreads) {
        const int t = e / (16 * kRanks), r = e % (16 * kRanks);
        if (t0 + t >= c.tokens || r0 + r >= c.w.rank) continue;
        const int a = present.adapter[t];
        if (a < 0 || rank_of(c.w, a) <= r0) out[(t0 + t) * c.w.rank + r0 + r] = 0.f;
    }
}

// Rows, many tokens.  64 tokens, 16 for each of four waves, and 128 (16 bits) or 64 elements of the long axis at a time, half of them for each of two
// such sets of waves.  A lane's operand of x is a line of
// its own (a token's), which costs the address unit 64 clocks for a load of 1 KiB: that much of a compute unit's time pays for x, once,
// and not for the weights too.  Those come by neighbouring lanes into LDS, for up to two adapters of the tile together -- a tile in which one
// request ends and the next one begins costs hardly more than another one, and is not what the launch waits for.  x is requested
// kAhead steps before its use, the weights one.  8192 x 4096 bf16, rank 64: 38 us, 1.75 TB/s of x.
template <class TX, class TW, bool kAlong, int kRanks>
__global__ __launch_bounds__(kRowsBlock, kRanks == 8 ? 2 : 4) void shrink_rows_kernel(ShrinkArgs c) {
    constexpr bool k16 = sizeof(TX) == 2;
    constexpr int kChunk = k16 ? 128 : 64, kHalves = kChunk / 64, kTile = 64, kAhead = k16 && kRanks < 4 ? 3 : 2, R = 16 * kRanks;
    constexpr int kRow = kChunk + 16 / (int)sizeof(TW);               // of a rank in LDS
    constexpr int V = 16 / (int)sizeof(TW);                           // elements of a load
    constexpr int kLoads = (R * kChunk / V + kRowsBlock - 1) / kRowsBlock;  // of a thread for an adapter's chunk
    using Operand = std::conditional_t<k16, Vec<TX, 8>, Vec<float, 8>>;
    __shared__ Present present;
    alignas(16) __shared__ TW staged[2][2][R][kRow];  // [turn][slot]
    const unsigned item = by_xcd(blockIdx.x, gridDim.x), part = item % c.parts;
    const int64_t t0 = (int64_t)(item / c.parts) * kTile;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % 4, set = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), i = lane & 15, g = lane >> 4, r0 = blockIdx.z * R;
    const int from = part * (int)c.part, to = std::min<int64_t>(from + c.part, c.length);
    const int tokens_left = (int)std::min<int64_t>(c.tokens - t0, kTile);
    const TX* x = static_cast<const TX*>(c.x) + t0 * c.ldx;
    const uint32_t x_lane = (uint32_t)(std::min(16 * wave + i, tokens_left - 1) * c.ldx + 8 * g) * sizeof(TX);
    auto x_of = [&](int k, Operand (&v)[kHalves]) {
        k += set * (kChunk / 2);
        if (k + kChunk / 2 <= to) {
            const uint32_t place = here(x_lane);
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
                if constexpr (k16) v[h] = load<TX, 8>(at(x + k + 32 * h, place));
                else v[h] = load_f32<TX, 8>(at(x + k + 32 * h, place));
            }
        } else {
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
                const int left = to - (k + 32 * h + 8 * g);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v[h][e] = (TX)0.f;
                    if (e < left) v[h][e] = at(x + k + 32 * h, x_lane)[e];
                }
            }
        }
    };
    Operand xs[kAhead][kHalves];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) x_of(from + u * kChunk, xs[u]);
    list_adapters(present, c.index, t0, kTile, c.tokens, c.w.adapters);
    const int slots = __builtin_amdgcn_readfirstlane(present.slots), own = present.adapter[16 * wave + i];
    float* out = c.out + (part * c.tokens + t0) * c.w.rank;
    for (int first = 0; first < slots; first += 2) {
        int adapter[2], ranks[2];
        bool mine[2];  // whether the wave has tokens of it
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            adapter[q] = first + q < slots ? __builtin_amdgcn_readfirstlane(present.slot[first + q]) : -1;
            ranks[q] = adapter[q] >= 0 ? std::min(rank_of(c.w, adapter[q]) - r0, R) : 0;
            mine[q] = ranks[q] > 0 && __any(own == adapter[q]);
        }
        if (ranks[0] <= 0 && ranks[1] <= 0) continue;
        if (first)
#pragma unroll
            for (int u = 0; u < kAhead; ++u) x_of(from + u * kChunk, xs[u]);
        Vec<TW, V> ws[2][kLoads];
        auto w_of = [&](int k) {  // past the rank and past the end of the axis: 0
            unsigned thread = threadIdx.x;
            asm volatile("" : "+v"(thread));  // as in here()
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                if (ranks[q] <= 0) continue;
                const TW* w = static_cast<const TW*>(c.w.w) + adapter[q] * c.w.stride + (kAlong ? r0 * c.w.ld + k : k * c.w.ld + r0);
                const bool whole = k + kChunk <= to && ranks[q] == R && R * kChunk / V % kRowsBlock == 0;
#pragma unroll
                for (int l = 0; l < kLoads; ++l) {
                    const int n = l * kRowsBlock + thread;
                    const int r = kAlong ? n / (kChunk / V) : n % (R / V) * V, e = kAlong ? n % (kChunk / V) * V : n / (R / V);
                    const TW* p = at(w, (uint32_t)(kAlong ? r * c.w.ld + e : e * c.w.ld + r) * sizeof(TW));
                    if (whole) {
                        ws[q][l] = load<TW, V>(p);
                    } else {
                        int left = kAlong ? (r < ranks[q] ? to - k - e : 0) : (k + e < to && n < R * kChunk / V ? ranks[q] - r : 0);
                        asm volatile("" : "+v"(left));
                        ws[q][l] = load_own<TW, V>(p, left);
                    }
                }
            }
        };
        auto w_put = [&](int turn) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                if (ranks[q] <= 0) continue;
#pragma unroll
                for (int l = 0; l < kLoads; ++l) {
                    const int n = l * kRowsBlock + threadIdx.x;
                    if (n >= R * kChunk / V) continue;
                    if constexpr (kAlong) {
                        *reinterpret_cast<Vec<TW, V>*>(&staged[turn][q][n / (kChunk / V)][n % (kChunk / V) * V]) = ws[q][l];
                    } else {
#pragma unroll
                        for (int m = 0; m < V; ++m) staged[turn][q][n % (R / V) * V + m][n / (R / V)] = ws[q][l][m];
                    }
                }
            }
        };
        F4 acc[2][kRanks];
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int r = 0; r < kRanks; ++r) acc[q][r] = 0.f;
        w_of(from);
        w_put(0);
        int turn = 0;
        for (int k = from; k < to; k += kAhead * kChunk) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (k + u * kChunk >= to) break;
                const bool more = k + (u + 1) * kChunk < to;
                if (more) w_of(k + (u + 1) * kChunk);
                __syncthreads();  // this turn's weights are there, and nobody reads the other's any more
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    if (!mine[q]) continue;
#pragma unroll
                    for (int h = 0; h < kHalves; ++h)
#pragma unroll
                        for (int r = 0; r < kRanks; ++r) {
                            const TW* line = &staged[turn][q][16 * r + i][set * (kChunk / 2) + 32 * h + 8 * g];  // at a multiple of 16 bytes
                            Vec<TW, 8> w;
                            if constexpr (sizeof(TW) == 4) {
                                const F4 low = *reinterpret_cast<const F4*>(line), high = *reinterpret_cast<const F4*>(line + 4);
                                w = __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7);
                            } else {
                                w = *reinterpret_cast<const Vec<TW, 8>*>(line);
                            }
                            if constexpr (k16) {
                                acc[q][r] = product(w, xs[u][h], acc[q][r]);
                            } else {
#pragma unroll
                                for (int e = 0; e < 8; ++e) acc[q][r] = product((float)w[e], xs[u][h][e], acc[q][r]);
                            }
                        }
                }
                x_of(k + (u + kAhead) * kChunk, xs[u]);
                if (more) w_put(turn ^ 1);
                turn ^= 1;
            }
        }
        // the second set's sums to the first one's, where the weights were
        F4(*sums)[2 * kRanks][64] = reinterpret_cast<F4(*)[2 * kRanks][64]>(&staged[0][0][0][0]);
        static_assert(sizeof(staged) >= 4 * sizeof(*sums), "");
        __syncthreads();
        if (set)
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int r = 0; r < kRanks; ++r) sums[wave][q * kRanks + r][lane] = acc[q][r];
        __syncthreads();
        if (!set)
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int r = 0; r < kRanks; ++r) acc[q][r] += sums[wave][q * kRanks + r][lane];
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            if (set || !mine[q] || own != adapter[q]) continue;
            const float scale = c.scale ? scale_of(c.w, adapter[q]) : 1.f;
#pragma unroll
            for (int r = 0; r < kRanks; ++r) {
                F4 v = acc[q][r] * scale;
                const int at_r = 16 * r + 4 * g;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (at_r + e >= ranks[q]) v[e] = 0.f;
                store_some<float, 4>(out + (16 * wave + i) * c.w.rank + r0 + at_r, v, c.w.rank - r0 - at_r);
            }
        }
    }
    // tokens without an adapter, or without ranks here
    const bool nothing = own < 0 || rank_of(c.w, own) <= r0;
    if (!set && 16 * wave + i < tokens_left && nothing)
#pragma unroll
        for (int r = 0; r < kRanks; ++r) store_some<float, 4>(out + (16 * wave + i) * c.w.rank + r0 + 16 * r + 4 * g, F4(0.f), c.w.rank - r0 - 16 * r - 4 * g);
}

// The parts of `shrink` added up in their order, times s_a (scale) -- where more than one kernel wants the sum.
__global__ __launch_bounds__(kBlock) void shrink_sum_kernel(ShrinkArgs c, const float* part, uint32_t parts) {
    const int64_t e = (int64_t)blockIdx.x * kBlock + threadIdx.x, all = c.tokens * c.w.rank;
    if (e >= all) return;
    float sum = 0.f;
#pragma unroll 8
    for (uint32_t p = 0; p < parts; ++p) sum += part[p * all + e];
    const int a = adapter_at(c.index, e / c.w.rank, c.tokens, c.w.adapters);
    c.out[e] = a < 0 ? 0.f : c.scale ? sum * scale_of(c.w, a) : sum;
}

// ---- expand ---------------------------------------------------------------------------------------------------------------------
struct ExpandArgs {
    Weights w;
    const int32_t* index;
    int64_t tokens, length;
    const float* part;  // [parts][tokens][rank]
    uint32_t parts;
    float* hidden;      // their sum, for the caller; nullptr: not wanted
    bool scale;
    const void* base;   // nullptr: 0
    void* y;
    int64_t ldbase, ldy;
    uint32_t blocks;    // of 64 elements of the long axis for a workgroup
    uint32_t groups;    // of such blocks
};

// The 16 tokens from t0 on, 64 elements of the long axis from o0 on; the waves share out the adapters.  Element o0 + 4 i + j is row (column) i of
// the tile j of four, so that a lane's loads have four neighbours where the weights lie that way, and sixteen neighbouring lanes have neighbouring
// memory in base and y.  `room`: LDS of 16 * (the rank's next multiple of 16, + 4) floats.
template <class TX, class TW, bool kColumns, bool kAlong, int kThreads>
__device__ __forceinline__ void expand_some(const ExpandArgs& c, int64_t t0, int64_t o0, Present& present, float* room) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
    const int rank16 = (c.w.rank + 15) / 16 * 16, pitch = rank16 + 4;
    const int left = (int)std::min<int64_t>(c.length - o0, 64), tokens_left = (int)std::min<int64_t>(c.tokens - t0, 16);
    const TX* base = static_cast<const TX*>(c.base);
    TX* y = static_cast<TX*>(c.y);
    // What does not depend on the tokens' adapters is requested before they are known: base and hidden's parts.
    // rows: acc[j][e], element o0 + 4 i + j of token 4 g + e; columns: element o0 + 16 g + 4 e + j of token i
    F4 acc[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = 0.f;
    if (base) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (kColumns) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (16 * g + 4 * e + j < left && i < tokens_left) acc[j][e] = (float)base[(o0 + 16 * g + 4 * e + j) * c.ldbase + t0 + i];
            } else if (4 * g + e < tokens_left) {
                const F4 v = load_some<TX, 4>(base + (t0 + 4 * g + e) * c.ldbase + o0 + 4 * i, left - 4 * i);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j][e] = v[j];
            }
        }
    }
    // a token has kThreads / 16 threads: up to sixteen for its ranks, in fours, each as neighbours that share the parts
    constexpr int kToken = kThreads / 16;
    const int fours = rank16 <= 16 ? 4 : rank16 <= 32 ? 8 : 16, splits = kToken / fours;
    const int t_own = threadIdx.x / kToken, split = threadIdx.x % splits, r_own = threadIdx.x % kToken / splits * 4;
    auto sum_of = [&](int r) {
        F4 sum = 0.f;
        if (t_own < tokens_left && r < c.w.rank) {
            const float* p = c.part + (t0 + t_own) * c.w.rank + r;
            if (r + 4 <= c.w.rank)
#pragma unroll 4
                for (uint32_t k = split; k < c.parts; k += splits) sum += load<float, 4>(p + k * c.tokens * c.w.rank);
            else
                for (uint32_t k = split; k < c.parts; k += splits) sum += load_some<float, 4>(p + k * c.tokens * c.w.rank, c.w.rank - r);
        }
        for (int k = 1; k < splits; k *= 2)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += __shfl_xor(sum[e], k);
        return sum;
    };
    const F4 early = sum_of(r_own);
    list_adapters(present, c.index, t0, 16, c.tokens, c.w.adapters);
    {  // 0 past the rank and for tokens without an adapter
        const int a = present.adapter[t_own];
        const float scale = a < 0 ? 0.f : c.scale ? scale_of(c.w, a) : 1.f;
        for (int r = r_own; r < rank16; r += 4 * fours) {
            const F4 sum = r < 4 * fours ? early : sum_of(r);
            if (split) continue;
            if (c.hidden && o0 == 0 && t_own < tokens_left)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (r + e < c.w.rank) c.hidden[(t0 + t_own) * c.w.rank + r + e] = sum[e];
            *reinterpret_cast<F4*>(&room[t_own * pitch + r]) = sum * scale;
        }
    }
    __syncthreads();
    // tokens without an adapter: a list entry of their own, unless y has what they get already
    const int slots = __builtin_amdgcn_readfirstlane(present.slots), jobs = slots + (__builtin_amdgcn_readfirstlane(present.none) && c.base != c.y ? 1 : 0);
    for (int job = wave; job < jobs; job += kThreads / 64) {
        const int a = job < slots ? __builtin_amdgcn_readfirstlane(present.slot[job]) : -1;
        F4 sum[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] = acc[j];
        const int rank = a >= 0 ? rank_of(c.w, a) : 0;
        const TW* w = static_cast<const TW*>(c.w.w) + (a >= 0 ? a * c.w.stride : 0);
        for (int r0 = 0; r0 < rank; r0 += 16) {
            const int from = r0 + 4 * g;
            F4 ws[4];  // [j][rank from + (0 .. 3)]
            if constexpr (kAlong) {  // w[r * ld + o]
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    F4 v = 0.f;
                    if (from + q < rank) v = load_some<TW, 4>(w + (from + q) * c.w.ld + o0 + 4 * i, left - 4 * i);
#pragma unroll
                    for (int j = 0; j < 4; ++j) ws[j][q] = v[j];
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) ws[j] = 4 * i + j < left ? load_some<TW, 4>(w + (o0 + 4 * i + j) * c.w.ld + from, rank - from) : F4(0.f);
            }
            const F4 h = *reinterpret_cast<const F4*>(&room[i * pitch + from]);
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[j] = kColumns ? product(ws[j][q], h[q], sum[j]) : product(h[q], ws[j][q], sum[j]);
        }
        const bool mine = i < tokens_left && present.adapter[i] == a;  // columns
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (kColumns) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (mine && 16 * g + 4 * e + j < left) y[(o0 + 16 * g + 4 * e + j) * c.ldy + t0 + i] = (TX)sum[j][e];
            } else if (4 * g + e < tokens_left && present.adapter[4 * g + e] == a) {
                store_some<TX, 4>(y + (t0 + 4 * g + e) * c.ldy + o0 + 4 * i, F4{sum[0][e], sum[1][e], sum[2][e], sum[3][e]}, left - 4 * i);
            }
        }
    }
}

template <class TX, class TW, bool kColumns, bool kAlong, int kThreads>
__global__ __launch_bounds__(kThreads) void expand_kernel(ExpandArgs c) {
    extern __shared__ float room[];
    __shared__ Present present;
    expand_some<TX, TW, kColumns, kAlong, kThreads>(c, (int64_t)blockIdx.x * 16, (int64_t)blockIdx.y * 64, present, room);
}

// ---- expand, many tokens --------------------------------------------------------------------------------------------------------
// A number as bf16 pieces that add up to it, the high bits first: each is cut (the last one rounded), so that none of them is larger
// than the number and three hold all 24 bits of it down to 2^-133.  Infinities and NaN are their first piece alone; beside a piece that is 0 an infinity
// gives NaN, so that sums of pieces' products that are not finite are formed again from whole numbers.
template <int kPieces>
__device__ __forceinline__ void pieces_of(float x, uint16_t (&p)[kPieces]) {
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
        if (k + 1 < kPieces) {
            const uint32_t high = x == x ? __float_as_uint(x) & 0xFFFF0000u : 0x7FC00000u;
            p[k] = (uint16_t)(high >> 16);
            x -= __uint_as_float(high);
            x = x == x ? x : 0.f;
        } else {
            p[k] = __builtin_bit_cast(uint16_t, (__bf16)x);
        }
    }
}
template <class T>
constexpr int kWeightPieces = sizeof(T) == 4 ? 3 : std::is_same_v<T, __bf16> ? 1 : 2;

using Pieces8 = Vec<__bf16, 8>;

// Eight weights as operands, one for each piece.
template <class TW>
__device__ __forceinline__ void weight_operands(const Vec<TW, 8> v, Pieces8 (&out)[kWeightPieces<TW>]) {
    if constexpr (std::is_same_v<TW, __bf16>) {
        out[0] = v;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            uint16_t p[kWeightPieces<TW>];
            pieces_of<kWeightPieces<TW>>((float)v[e], p);
#pragma unroll
            for (int k = 0; k < kWeightPieces<TW>; ++k) out[k][e] = __builtin_bit_cast(__bf16, p[k]);
        }
    }
}

// Waves for a SIMD: what an adapter's weights in registers leave of them.  32-bit weights: three waves and not four, whose registers spill (8000 tokens of 30 requests in
// columns, 2048 -> 4096, rank 32: 161 -> 137 us); fp16 rows of ranks (kAlong) over 32 likewise (backward of 3000 tokens, rank 64: 118 -> 112), but not otherwise (8192
// tokens, forward: 97 -> 102).
template <class TX, class TW, bool kAlong, int kChunks>
constexpr int kWideWaves = kChunks == 4 ? 2 : (kChunks && sizeof(TW) == 4) || (kChunks == 2 && kAlong && std::is_same_v<TX, _Float16>) ? 3 : 4;

// 64 tokens.  A wave takes 64 elements of the long axis at a time, with what base has there in registers, and goes through the adapters, each
// one's weights (ranks up to kChunks * 32; 0: any, loaded again for every tile of 16 tokens) in registers.  Element o0 + 4 i + j is row (column) i of
// tile j of four; in columns, token t0 + 4 i + s that of tile s.  hidden is multiplied as three bf16 pieces by the weights' one (bf16), two
// (fp16) or three in the 16-bit instruction, at a fifth to a half of the 32-bit one's time.  The pieces are cut from the number, so that the second is below 2^-7 of it, the third below
// 2^-14, and three hold all its bits: only the product of both third ones is left out, 2^-28 of a product.
// Base and y of 8192 x 4096 bf16, rank 64: 51 us, 2.6 TB/s; of 3136 x 4096 fp32 columns, rank 16: 35 us, 3.0 TB/s; with the 32-bit instruction, which takes its 16
// rows of y from memory one line a lane, 201 and 66.
template <class TX, class TW, bool kColumns, bool kAlong, int kChunks>
__global__ __launch_bounds__(kBlock, (kWideWaves<TX, TW, kAlong, kChunks>)) void expand_wide_kernel(ExpandArgs c) {
    constexpr int kTile = 64, kH = 3, kW = kWeightPieces<TW>, kHeld = kChunks ? kChunks : 1;
    extern __shared__ float room[];
    __shared__ Present present;
    // the last workgroups take what the tiles of 64 by 64 leave: the last tokens, and the end of the long axis of the others
    const int tiles = (int)(c.tokens / 64), blocks = (int)(c.length / 64), all_blocks = (int)((c.length + 63) / 64);
    const unsigned inner = tiles * c.groups;
    if (blockIdx.x >= inner) {
        const int n = blockIdx.x - inner, behind = (int)((c.tokens - 64 * (int64_t)tiles + 15) / 16) * all_blocks;
        if (n < behind) expand_some<TX, TW, kColumns, kAlong, kBlock>(c, 64 * (int64_t)tiles + n / all_blocks * 16, n % all_blocks * (int64_t)64, present, room);
        else expand_some<TX, TW, kColumns, kAlong, kBlock>(c, (int64_t)(n - behind) * 16, (int64_t)blocks * 64, present, room);
        return;
    }
    uint16_t* planes = reinterpret_cast<uint16_t*>(room);  // [piece][token][pitch]: hidden, 0 past the rank and for tokens without an adapter
    const unsigned item = by_xcd(blockIdx.x, inner);
    const int64_t t0 = (int64_t)(item / c.groups) * kTile;
    const int group = item % c.groups;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
    const int rank32 = (c.w.rank + 31) / 32 * 32, pitch = rank32 + 8;
    const TX* base = static_cast<const TX*>(c.base);
    TX* y = static_cast<TX*>(c.y);
    const int first = group * c.blocks, last = std::min(first + (int)c.blocks, blocks);
    // a lane's place: the rest of an address is the wave's
    const uint32_t base_lane = (uint32_t)((kColumns ? 16 : 4) * g * c.ldbase + 4 * i) * sizeof(TX), y_lane = (uint32_t)((kColumns ? 16 : 4) * g * c.ldy + 4 * i) * sizeof(TX);
    const uint32_t w_lane = (uint32_t)(kAlong ? 4 * i : 4 * i * c.w.ld) * sizeof(TW);
    // A quarter of base, 64 x 64.  rows: [e], elements 4 i .. + 3 of token 16 u + 4 g + e; columns: [e], tokens 4 i .. + 3 of element
    // 16 g + 4 e + u.  Sixteen neighbouring lanes have neighbouring memory: a load of one line for each of them would
    // take the address unit sixteen times as long.
    auto get = [&](int block, int u, Vec<TX, 4> (&r)[4]) {
        const int64_t o0 = (int64_t)block * 64;
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = (TX)0.f;
        const uint32_t from = here(base_lane);
        if (base)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                r[e] = load<TX, 4>(at(kColumns ? base + (o0 + 4 * e + u) * c.ldbase + t0 : base + (t0 + 16 * u + e) * c.ldbase + o0, from));
    };
    // What does not depend on the tokens' adapters is requested before they are known: the first quarter of base, and hidden's parts, four threads
    // for a token, four ranks at a time.
    Vec<TX, 4> raw[2][4];  // this quarter's and the next one's
    if (first + wave < last) get(first + wave, 0, raw[0]);
    const int t = threadIdx.x >> 2, r_first = (threadIdx.x & 3) * 4;
    auto sum_of = [&](int r) {
        F4 sum = 0.f;
        const float* p = c.part + (t0 + t) * c.w.rank + r;
        if (r < c.w.rank)  // in fours
#pragma unroll 4
            for (uint32_t k = 0; k < c.parts; ++k) sum += load<float, 4>(p + k * c.tokens * c.w.rank);
        return sum;
    };
    F4 early[2 * kHeld];
    if constexpr (kChunks)
#pragma unroll
        for (int r = 0; r < 2 * kHeld; ++r) early[r] = sum_of(r_first + 16 * r);
    list_adapters(present, c.index, t0, kTile, c.tokens, c.w.adapters);
    const int slots = __builtin_amdgcn_readfirstlane(present.slots), jobs = slots + (__builtin_amdgcn_readfirstlane(present.none) && c.base != c.y ? 1 : 0);
    if (jobs == 0 && !c.hidden) return;
    {
        const int a = present.adapter[t];
        const float scale = a < 0 ? 0.f : c.scale ? scale_of(c.w, a) : 1.f;
        auto put = [&](int r, F4 sum) {  // `shrink` has left 0 for tokens without an adapter and past an adapter's rank
            if (c.hidden && group == 0 && r < c.w.rank) store<float, 4>(c.hidden + (t0 + t) * c.w.rank + r, sum);
            sum *= scale;
            uint16_t h[4][kH];
#pragma unroll
            for (int e = 0; e < 4; ++e) pieces_of<kH>(sum[e], h[e]);
#pragma unroll
            for (int k = 0; k < kH; ++k) {
                const Vec<uint16_t, 4> v = {h[0][k], h[1][k], h[2][k], h[3][k]};
                *reinterpret_cast<Vec<uint16_t, 4>*>(&planes[(k * kTile + t) * pitch + r]) = v;
            }
        };
        if constexpr (kChunks) {
#pragma unroll
            for (int r = 0; r < 2 * kHeld; ++r)
                if (r_first + 16 * r < rank32) put(r_first + 16 * r, early[r]);
        } else {
            for (int r = r_first; r < rank32; r += 16) put(r, sum_of(r));
        }
    }
    __syncthreads();
    for (int block = first + wave; block < last; block += kWaves) {
        const int64_t o0 = (int64_t)block * 64;
        for (int q = 0; q < jobs; ++q) {
            const int a = q < slots ? __builtin_amdgcn_readfirstlane(present.slot[q]) : -1;
            const int rank = a >= 0 ? rank_of(c.w, a) : 0;
            const TW* w = static_cast<const TW*>(c.w.w) + (a >= 0 ? a * c.w.stride : 0) + (kAlong ? o0 : o0 * c.w.ld);
            auto weights = [&](int r0, Pieces8 (&ws)[4][kW]) {
                Vec<TW, 8> u[4];
                weights_of<TW, kAlong>(w, w_lane, c.w.ld, rank, r0 + 8 * g, u);
#pragma unroll
                for (int j = 0; j < 4; ++j) weight_operands<TW>(u[j], ws[j]);
            };
            auto operand = [&](int k, int t, int r0) { return *reinterpret_cast<const Pieces8*>(&planes[(k * kTile + t) * pitch + r0 + 8 * g]); };
            Pieces8 held[kHeld][4][kW];
            if constexpr (kChunks)
                if (rank > 0)
#pragma unroll
                    for (int r = 0; r < kChunks; ++r)
                        if (kChunks < 4 || 32 * r < rank32) weights(32 * r, held[r]);
            unsigned again = 0;
#pragma unroll
            for (int u = 0; u < 4; ++u) {  // rows: tokens 16 u .. + 15, four tiles of elements; columns: elements 4 (0 .. 15) + u, four tiles of tokens
                if (u < 3) get(block, u + 1, raw[(u + 1) % 2]);
                else if (q + 1 < jobs) get(block, 0, raw[0]);
                else if (block + kWaves < last) get(block + kWaves, 0, raw[0]);
                // the adapters of the lane's tokens (rows: 16 u + 4 g + e; columns: 4 i + e)
                const Vec<int, 4> of = *reinterpret_cast<const Vec<int, 4>*>(&present.adapter[kColumns ? 4 * i : 16 * u + 4 * g]);
                if (!__any(of[0] == a || of[1] == a || of[2] == a || of[3] == a)) continue;
                F4 acc[4];  // [tile][row 4 g + e]
#pragma unroll
                for (int v = 0; v < 4; ++v)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[v][e] = (float)raw[u % 2][e][v];
                auto chunk = [&](int r0, const Pieces8 (&ws)[4][kW]) {
#pragma unroll
                    for (int k = kH - 1; k >= 0; --k) {  // the largest product last: the roundings of the sums before it are small (the order of the others: registers)
                        Pieces8 h;
                        if constexpr (!kColumns) h = operand(k, 16 * u + i, r0);
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            if constexpr (kColumns) h = operand(k, 4 * i + v, r0);
#pragma unroll
                            for (int m = 0; m < kW; ++m)
                                if (const int l = k ? m : kW - 1 - m; k + l < 4) acc[v] = kColumns ? product(ws[u][l], h, acc[v]) : product(h, ws[v][l], acc[v]);
                        }
                    }
                };
                if (rank > 0) {
                    if constexpr (kChunks) {
#pragma unroll
                        for (int r = 0; r < kChunks; ++r)
                            if (kChunks < 4 || 32 * r < rank32) chunk(32 * r, held[r]);
                    } else {
#pragma unroll 1
                        for (int r0 = 0; r0 < rank; r0 += 32) {
                            weights(r0, held[0]);
                            chunk(r0, held[0]);
                        }
                    }
                }
                // A sum that is not finite is formed again below.  0 times it is not 0: of[e] is the token of acc[.][e] (rows) or acc[e] (columns).
                bool odd = false;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float zero = 0.f;
#pragma unroll
                    for (int v = 0; v < 4; ++v) zero = fmaf(kColumns ? acc[e][v] : acc[v][e], 0.f, zero);
                    odd |= of[e] == a && zero != 0.f;
                }
                if (rank > 0 && __any(odd)) {
                    again |= 1u << u;
                    continue;
                }
                const uint32_t to = here(y_lane);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const Vec<float, 4> v = {acc[0][e], acc[1][e], acc[2][e], acc[3][e]};
                    TX* p = at(kColumns ? y + (o0 + 4 * e + u) * c.ldy + t0 : y + (t0 + 16 * u + e) * c.ldy + o0, to);
                    if constexpr (kColumns) {
                        if (of[0] == a && of[1] == a && of[2] == a && of[3] == a) {
                            store_f32<TX, 4>(p, v);
                        } else {
#pragma unroll
                            for (int m = 0; m < 4; ++m)
                                if (of[m] == a) p[m] = (TX)v[m];
                        }
                    } else if (of[e] == a) {
                        store_f32<TX, 4>(p, v);
                    }
                }
            }
            // Quarters with an infinity or NaN, tile by tile from whole numbers by the 32-bit instruction, four ranks at a time, one for each g.
            if (__builtin_expect(again != 0, 0))
#pragma unroll 1
                for (int n = 0; n < 16; ++n) {
                    const int u = n / 4, v = n % 4;
                    if (!(again >> u & 1)) continue;
                    // the tokens and elements of sum[e]
                    auto token = [&](int e) { return kColumns ? 4 * i + v : 16 * u + 4 * g + e; };
                    auto element = [&](int e) { return o0 + (kColumns ? 16 * g + 4 * e + u : 4 * i + v); };
                    auto place = [&](int e, int64_t ld) { return kColumns ? element(e) * ld + t0 + token(e) : (t0 + token(e)) * ld + element(e); };
                    F4 sum = 0.f;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (base) sum[e] = (float)base[place(e, c.ldbase)];  // it may be y: nobody has written what this adapter's tokens get
#pragma unroll 1
                    for (int r0 = 0; r0 < rank; r0 += 4) {
                        const int r = r0 + g;
                        float h = 0.f, x = 0.f;
                        if (r < rank) {
                            const int t = kColumns ? 4 * i + v : 16 * u + i, o = 4 * i + (kColumns ? u : v);
#pragma unroll
                            for (int k = kH - 1; k >= 0; --k) h += __uint_as_float((uint32_t)planes[(k * kTile + t) * pitch + r] << 16);
                            x = (float)w[kAlong ? r * c.w.ld + o : o * c.w.ld + r];
                        }
                        sum = kColumns ? product(x, h, sum) : product(h, x, sum);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (present.adapter[token(e)] == a) y[place(e, c.ldy)] = (TX)sum[e];
                }
        }
    }
}

// ---- outer ----------------------------------------------------------------------------------------------------------------------
struct OuterArgs {
    const float* g;          // [tokens][rank]
    const uint16_t* planes;  // the same as planes_kernel lays it out, times s_a; activations in 16 bits
    Weights w;       // adapters, ranks, scales
    const int32_t* index;
    int64_t tokens, length;
    const void* x;
    int64_t ldx;
    int64_t range;  // tokens for a workgroup (blockIdx.z), a multiple of 16
    uint32_t parts;   // such ranges
    uint32_t blocks;  // workgroups for an adapter and range
    float* out;       // [parts][adapters][rank][length], or rank_last: [parts][adapters][length][rank]
    bool scale, rank_last;
};
// dA and dB in one launch: they do not depend on one another, and alone neither fills the chip at a small step's sizes.
struct OuterPair {
    OuterArgs a, b;  // b.blocks == 0: only a
};
// Which of the two a workgroup belongs to, and its number there; false: nothing to do.
__device__ __forceinline__ bool outer_of(const OuterPair& pair, OuterArgs& c, unsigned& block) {
    const bool second = blockIdx.x >= pair.a.blocks;
    c = second ? pair.b : pair.a;
    block = blockIdx.x - (second ? pair.a.blocks : 0);
    return blockIdx.z < c.parts;
}

// The groups of kGroup tokens in from .. to in which the adapter occurs, in their order, for up to kOuterBlock groups from `first` on: their numbers
// into `list`; returns how many.  All threads call it.
template <int kGroup>
__device__ __forceinline__ int list_groups(const int32_t* index, int64_t first, int64_t to, int a, int* list, int* count) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t mine = first + (int64_t)threadIdx.x * kGroup;
    bool some = false;
    if (mine + kGroup <= to) {
        Vec<int32_t, 4> of[kGroup / 4];
#pragma unroll
        for (int k = 0; k < kGroup / 4; ++k) of[k] = load<int32_t, 4>(index + mine + 4 * k);
#pragma unroll
        for (int k = 0; k < kGroup; ++k) some |= of[k / 4][k % 4] == a;
    } else if (mine < to) {
        for (int64_t k = mine; k < to; ++k) some |= index[k] == a;
    }
    const unsigned long long here = __ballot(some);
    if (lane == 0) count[wave] = __popcll(here);
    __syncthreads();
    int at = __popcll(here & ((1ull << lane) - 1)), groups = 0;
    for (int k = 0; k < kOuterBlock / 64; ++k) {
        if (k < wave) at += count[k];
        groups += count[k];
    }
    if (some) list[at] = threadIdx.x;
    __syncthreads();
    return groups;
}

// The waves' sums of kSums registers each, in the first wave's: the upper half's to the lower half's, until there is one.
template <int kSums>
__device__ __forceinline__ void add_waves(F4 (&acc)[kSums], F4 (*room)[kSums][64]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int half = kOuterBlock / 128; half; half /= 2) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int r = 0; r < kSums; ++r) room[wave - half][r][lane] = acc[r];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int r = 0; r < kSums; ++r) acc[r] += room[wave][r][lane];
        __syncthreads();
    }
}

// Gradients of ranks at .. at + 3, `some` registers of them from `first` on: 0 past the adapter's rank, where 0 has been multiplied by whatever the
// tokens hold, an infinity or a NaN too.
template <int kSums>
__device__ __forceinline__ void past_rank(F4 (&acc)[kSums], int first, int some, int at, int rank) {
#pragma unroll
    for (int j = 0; j < some; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[first + j][e] = at + e < rank ? acc[first + j][e] : 0.f;
}

// Adapter blockIdx.y, 64 elements of the long axis from o0 on, kRanks * 16 ranks from r0 on; the waves share out the groups of 16 tokens in which the adapter occurs.
template <class TX, bool kColumns, int kRanks>
__device__ __forceinline__ void outer_some(const OuterArgs& c, int64_t o0, int r0, int* list, int* count, F4 (*room)[kRanks * 4][64]) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4, a = blockIdx.y;
    const int left = (int)std::min<int64_t>(c.length - o0, 64);
    const int rank = rank_of(c.w, a);
    const int64_t from = blockIdx.z * c.range, to = from + c.range < c.tokens ? from + c.range : c.tokens;
    F4 acc[kRanks * 4];  // [rank tile][j]
#pragma unroll
    for (int r = 0; r < kRanks * 4; ++r) acc[r] = 0.f;
    bool any = false;  // whether the adapter occurs
    for (int64_t first = from; first < to; first += kOuterBlock * 16) {
        const int groups = list_groups<16>(c.index, first, to, a, list, count);
        any |= groups > 0;
        if (rank > r0)
            for (int q = wave; q < groups; q += kOuterBlock / 64) {
                const int64_t t = first + list[q] * 16 + 4 * g;  // lane group g has tokens t .. t + 3
                const int some = (int)std::max<int64_t>(0, std::min<int64_t>(to - t, 4));
                // everything is requested before the tokens' adapters are known
                F4 xs[4];  // [token k][element 4 i + j]
                if constexpr (kColumns) {
                    F4 v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        v[j] = 4 * i + j < left ? load_some<TX, 4>(static_cast<const TX*>(c.x) + (o0 + 4 * i + j) * c.ldx + t, some) : F4(0.f);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int j = 0; j < 4; ++j) xs[k][j] = v[j][k];
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        xs[k] = k < some ? load_some<TX, 4>(static_cast<const TX*>(c.x) + (t + k) * c.ldx + o0 + 4 * i, left - 4 * i) : F4(0.f);
                }
                float gs[kRanks][4];
#pragma unroll
                for (int r = 0; r < kRanks; ++r)
#pragma unroll
                    for (int k = 0; k < 4; ++k) gs[r][k] = k < some && r0 + 16 * r + i < rank ? c.g[(t + k) * c.w.rank + r0 + 16 * r + i] : 0.f;
                Vec<int32_t, 4> of;
                if (some == 4) {
                    of = load<int32_t, 4>(c.index + t);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) of[k] = k < some ? c.index[t + k] : -1;
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (of[k] != a) {  // another adapter's token, whatever it holds
                        xs[k] = 0.f;
#pragma unroll
                        for (int r = 0; r < kRanks; ++r) gs[r][k] = 0.f;
                    }
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int r = 0; r < kRanks; ++r)
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[4 * r + j] = product(gs[r][k], xs[k][j], acc[4 * r + j]);
            }
        __syncthreads();  // the list is made anew
    }
    add_waves(acc, room);
    if (wave) return;
    const float scale = c.scale && any ? scale_of(c.w, a) : 1.f;  // an adapter that nobody has gets 0 whatever its factor is
    float* out = c.out + ((int64_t)blockIdx.z * c.w.adapters + a) * c.w.rank * c.length;
#pragma unroll
    for (int r = 0; r < kRanks; ++r) {
        const int at = r0 + 16 * r + 4 * g;
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[4 * r + j] *= scale;
        past_rank(acc, 4 * r, 4, at, rank);
        if (c.rank_last) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (4 * i + j < left && at < c.w.rank) store_some<float, 4>(out + (o0 + 4 * i + j) * c.w.rank + at, acc[4 * r + j], c.w.rank - at);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (at + k >= c.w.rank) continue;
                F4 v;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = acc[4 * r + j][k];
                store_some<float, 4>(out + (at + k) * c.length + o0 + 4 * i, v, left - 4 * i);
            }
        }
    }
}

// 999 tokens, 2048 -> 4608, rank 8, 4 adapters, columns: 15 us, the adapter's tokens and then their x and d one after the other.
template <class TX, bool kColumns, int kRanks>
__global__ __launch_bounds__(kOuterBlock) void outer_kernel(OuterPair pair) {
    OuterArgs c;
    unsigned block;
    if (!outer_of(pair, c, block)) return;
    __shared__ int list[kOuterBlock], count[kOuterBlock / 64];
    __shared__ F4 room[kOuterBlock / 128][kRanks * 4][64];
    const int rank_blocks = (c.w.rank + 16 * kRanks - 1) / (16 * kRanks);
    outer_some<TX, kColumns, kRanks>(c, (int64_t)(block / rank_blocks) * 64, (int)(block % rank_blocks) * 16 * kRanks, list, count, room);
}

// Activations in 16 bits, rows: the 16-bit instruction over 32 tokens.  It wants eight tokens of one element in a lane where memory has eight
// elements of one token: a lane loads eight by eight (kCols = 8; 16 bytes of 8 tokens, sixteen lanes 256 bytes side by side) and
// turns them in its registers.  The other operand, d or hidden as three bf16 pieces, lies in `planes` as lanes take it (planes_kernel); fp16
// activations are two bf16 pieces.  All products of pieces are taken, so that nothing is lost against products in 32 bits.  dA and dB of 4096 tokens, 9216 -> 4096, rank 32, 8 adapters: 39 us,
// 2.9 TB/s of x and dy; 158 in the kernel above.
template <class TX, int kRanks, int kCols>
__global__ __launch_bounds__(kOuterBlock, 3) void outer16_kernel(OuterPair pair) {
    OuterArgs c;
    unsigned block;
    if (!outer_of(pair, c, block)) return;
    constexpr int kX = kWeightPieces<TX>, kSums = kRanks * kCols;
    __shared__ int list[kOuterBlock], count[kOuterBlock / 64], again;
    __shared__ F4 room[kOuterBlock / 128][kSums][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4, a = blockIdx.y;
    const int rank_blocks = (c.w.rank + 16 * kRanks - 1) / (16 * kRanks), rank_tiles = (c.w.rank + 15) / 16;
    const int64_t o0 = (int64_t)(block / rank_blocks) * (16 * kCols);
    const int left = (int)std::min<int64_t>(c.length - o0, 16 * kCols) - kCols * i;
    const int tile0 = (int)(block % rank_blocks) * kRanks;
    const int rank = rank_of(c.w, a);
    const int64_t from = blockIdx.z * c.range, to = from + c.range < c.tokens ? from + c.range : c.tokens;
    const uint32_t x_lane = (uint32_t)(8 * g * c.ldx + kCols * i) * sizeof(TX);
    F4 acc[kSums];  // [rank tile][column]
#pragma unroll
    for (int r = 0; r < kSums; ++r) acc[r] = 0.f;
    for (int64_t first = from; first < to; first += kOuterBlock * 32) {
        const int groups = list_groups<32>(c.index, first, to, a, list, count);
        if (rank > 16 * tile0)
            for (int q = wave; q < groups; q += kOuterBlock / 64) {
                const int64_t t = first + __builtin_amdgcn_readfirstlane(list[q]) * 32;
                const TX* x = static_cast<const TX*>(c.x) + t * c.ldx + o0;
                Vec<TX, kCols> xs[8];
                Vec<int32_t, 8> of;
                const bool whole = t + 32 <= to;
                if (whole && left >= kCols) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) xs[e] = load<TX, kCols>(at(x + e * c.ldx, x_lane));
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) xs[e] = t + 8 * g + e < to ? load_own<TX, kCols>(at(x + e * c.ldx, x_lane), left) : Vec<TX, kCols>((TX)0.f);
                }
                Pieces8 gs[kRanks][3];
                const Pieces8* planes = reinterpret_cast<const Pieces8*>(c.planes) + (t / 32 * 3 * rank_tiles + tile0) * 64 + lane;
#pragma unroll
                for (int r = 0; r < kRanks; ++r)
#pragma unroll
                    for (int p = 0; p < 3; ++p) gs[r][p] = planes[(p * rank_tiles + std::min(r, rank_tiles - 1 - tile0)) * 64];
                if (whole) {
                    of = load<int32_t, 8>(c.index + t + 8 * g);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) of[e] = t + 8 * g + e < to ? c.index[t + 8 * g + e] : -1;
                }
                bool every = true;
#pragma unroll
                for (int e = 0; e < 8; ++e) every &= of[e] == a;
                if (!__all(every)) {  // other adapters' tokens, whatever they hold
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (of[e] == a) continue;
                        xs[e] = (TX)0.f;
#pragma unroll
                        for (int r = 0; r < kRanks; ++r)
#pragma unroll
                            for (int p = 0; p < 3; ++p) gs[r][p][e] = (__bf16)0.f;
                    }
                }
#pragma unroll
                for (int k = 0; k < kCols; ++k) {
                    const Vec<TX, 8> column = {xs[0][k], xs[1][k], xs[2][k], xs[3][k], xs[4][k], xs[5][k], xs[6][k], xs[7][k]};
                    Pieces8 ps[kX];
                    weight_operands<TX>(column, ps);
#pragma unroll
                    for (int r = 0; r < kRanks; ++r)
#pragma unroll
                        for (int p = 2; p >= 0; --p)  // the largest product last
#pragma unroll
                            for (int l = kX - 1; l >= 0; --l) acc[r * kCols + k] = product(gs[r][p], ps[l], acc[r * kCols + k]);
                }
            }
        __syncthreads();  // the list is made anew
    }
    add_waves(acc, room);
    // Sums that are not finite (0 times them is not 0): an infinity has met pieces that are 0.  Again, all of them, from whole numbers by the 32-bit instruction.
    if (wave == 0) {
        float zero = 0.f;
#pragma unroll
        for (int r = 0; r < kRanks; ++r) {
            past_rank(acc, r * kCols, kCols, 16 * (tile0 + r) + 4 * g, rank);
#pragma unroll
            for (int k = 0; k < kCols; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) zero = fmaf(acc[r * kCols + k][e], 0.f, zero);
        }
        const bool odd = __any(zero != 0.f);
        if (lane == 0) again = odd;
    }
    __syncthreads();
    if (__builtin_expect(again, 0)) {
        for (int64_t o = o0; o < std::min<int64_t>(o0 + 16 * kCols, c.length); o += 64)
#pragma unroll 1
            for (int tile = tile0; tile < std::min(tile0 + kRanks, rank_tiles); ++tile)
                outer_some<TX, false, 1>(c, o, 16 * tile, list, count, reinterpret_cast<F4(*)[4][64]>(&room[0][0][0]));
        return;
    }
    if (wave) return;
    float* out = c.out + ((int64_t)blockIdx.z * c.w.adapters + a) * c.w.rank * c.length;
#pragma unroll
    for (int r = 0; r < kRanks; ++r) {
        const int at = 16 * (tile0 + r) + 4 * g;
        if (c.rank_last) {
#pragma unroll
            for (int k = 0; k < kCols; ++k)
                if (k < left && at < c.w.rank) store_some<float, 4>(out + (o0 + kCols * i + k) * c.w.rank + at, acc[r * kCols + k], c.w.rank - at);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (at + e >= c.w.rank) continue;
                Vec<float, kCols> v;
#pragma unroll
                for (int k = 0; k < kCols; ++k) v[k] = acc[r * kCols + k][e];
                store_some<float, kCols>(out + (at + e) * c.length + o0 + kCols * i, v, left);
            }
        }
    }
}

// What outer16_kernel takes of d and hidden: pieces p = 0 .. 2 of [tokens][rank], for 32 tokens and 16 ranks lane by lane: element (token t, rank r)
// at ((((t / 32) 3 + p) rank tiles + r / 16) 64 + r % 16 + 16 (t % 32 / 8)) 8 + t % 8; 0 for tokens without an adapter, past an adapter's rank and
// past the last token.  A workgroup for 32 tokens: blockIdx.y = 0: d, from the parts that `shrink` has left, times s_a, which is also
// written as numbers in 32 bits (c.out); 1: hidden times s_a.
__global__ __launch_bounds__(kBlock) void planes_kernel(ShrinkArgs c, const float* part, uint32_t parts, const float* hidden, uint16_t* d_planes, uint16_t* hidden_planes) {
    const bool is_d = blockIdx.y == 0;
    uint16_t* planes = is_d ? d_planes : hidden_planes;
    const float* from = is_d ? part : hidden;
    const int rank_tiles = (c.w.rank + 15) / 16;
    const int64_t all = c.tokens * c.w.rank, t = (int64_t)blockIdx.x * 32 + threadIdx.x / 8;
    const int a = adapter_at(c.index, t, c.tokens, c.w.adapters);
    const int rank = a >= 0 ? rank_of(c.w, a) : 0;
    const float scale = a >= 0 ? scale_of(c.w, a) : 0.f;
    for (int r = (threadIdx.x % 8) * 4; r < 16 * rank_tiles; r += 32) {
        F4 sum = 0.f;
        if (r < rank) {
#pragma unroll 4
            for (uint32_t k = 0; k < (is_d ? parts : 1); ++k) sum += load_some<float, 4>(from + k * all + t * c.w.rank + r, rank - r);
        }
        sum *= scale;
        if (is_d && t < c.tokens) store_some<float, 4>(c.out + t * c.w.rank + r, sum, c.w.rank - r);
        if (!planes) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint16_t p[3];
            pieces_of<3>(sum[e], p);
#pragma unroll
            for (int k = 0; k < 3; ++k)
                planes[((((int64_t)blockIdx.x * 3 + k) * rank_tiles + r / 16) * 64 + (r + e) % 16 + 16 * (t % 32 / 8)) * 8 + t % 8] = p[k];
        }
    }
}

__global__ __launch_bounds__(kBlock) void outer_sum_kernel(const float* part, uint32_t parts, int64_t numbers, float* out) {
    const int64_t e = ((int64_t)blockIdx.x * kBlock + threadIdx.x) * 4;
    if (e >= numbers) return;
    F4 all = 0.f;
#pragma unroll 4
    for (uint32_t p = 0; p < parts; ++p) all += load_some<float, 4>(part + p * numbers + e, numbers - e);
    store_some<float, 4>(out + e, all, numbers - e);
}

// ---- launches -------------------------------------------------------------------------------------------------------------------
// How a contraction over `length` is cut: tokens of a workgroup, ranks of one, parts of the long axis.
struct ShrinkShape {
    int tiles, ranks, parts;
    int64_t part;
    ShrinkShape(int64_t tokens, int64_t rank, int64_t length, bool columns, int64_t adapters) {
        ranks = rank <= 16 ? 1 : rank <= 32 ? 2 : rank <= 64 ? 4 : 8;
        // columns, ranks over 64: 128 of them take all of a wave's registers with 16 tokens; 64 tokens and x twice took longer (4096 tokens of 4096
        // features, rank 128: 95 -> 131 us, both launches)
        tiles = tokens <= kFewTokens || (columns && ranks == 8) ? 1 : 4;
        int64_t blocks = (tokens + 16 * tiles - 1) / (16 * tiles);
        // Few tokens: workgroups for sixteen ranks each, while that leaves the long axis at least eight parts: more of them, and fewer parts for
        // `expand` to add up (one token, 4096 features, rank 64: 7.7 -> 4.9 us and 8.7 -> 7.5; 64 tokens: 7.4 -> 5.0 and 14.2 -> 10.0).
        for (; tokens <= kFewTokens && ranks > 1 && blocks <= 16; ranks /= 2) blocks *= 2;
        // few tokens: a workgroup for a compute unit, and no stretch of the long axis of less than 128 elements, or less than 32 for a wave where the
        // sixteen waves have up to so many adapters abreast
        const int64_t abreast = std::min<int64_t>({16, tokens, adapters});
        const int64_t want = tokens <= kFewTokens ? std::min<int64_t>(256 / blocks, length / std::max<int64_t>(128, 512 / abreast))
                                                  : std::min<int64_t>(512 / blocks, (length + 255) / 256);
        const int64_t cut = std::max<int64_t>(1, std::min<int64_t>(want, 64)), step = tokens <= kFewTokens ? 32 : columns && tiles == 4 ? (blocks < 32 ? 256 : 512) : 128;
        part = ((length + cut - 1) / cut + step - 1) / step * step;
        parts = (int)((length + part - 1) / part);
    }
};

template <class TX, class TW, bool kColumns, bool kAlong, int kRanks>
void shrink_tiles(const ShrinkArgs& c, const ShrinkShape& f, hipStream_t s) {
    const dim3 grid((unsigned)((c.tokens + 16 * f.tiles - 1) / (16 * f.tiles) * f.parts), 1, (unsigned)((c.w.rank + 16 * kRanks - 1) / (16 * kRanks)));
    if (f.tiles == 4) {
        if constexpr (!kColumns) shrink_rows_kernel<TX, TW, kAlong, kRanks><<<grid, kRowsBlock, 0, s>>>(c);
        else if constexpr (kRanks < 8) shrink_kernel<TX, TW, kColumns, kAlong, 4, kRanks><<<grid, kShrinkThreads<4>, 0, s>>>(c);
    } else if constexpr (kColumns || kRanks < 8) {  // ShrinkShape: few tokens have no eight
        shrink_kernel<TX, TW, kColumns, kAlong, 1, kRanks><<<grid, kShrinkThreads<1>, 0, s>>>(c);
    }
}
template <class TX, class TW, bool kColumns, bool kAlong>
int shrink_ranks(const ShrinkArgs& c, const ShrinkShape& f, hipStream_t s) {
    if (f.ranks == 1) shrink_tiles<TX, TW, kColumns, kAlong, 1>(c, f, s);
    else if (f.ranks == 2) shrink_tiles<TX, TW, kColumns, kAlong, 2>(c, f, s);
    else if (f.ranks == 4) shrink_tiles<TX, TW, kColumns, kAlong, 4>(c, f, s);
    else shrink_tiles<TX, TW, kColumns, kAlong, 8>(c, f, s);
    return (int)hipGetLastError();
}
template <bool kAlong>
int shrink(ShrinkArgs c, const ShrinkShape& f, const cer_tokens_t& x, int32_t weights, hipStream_t s) {
    c.x = x.data, c.ldx = x.ld, c.part = f.part, c.parts = (uint32_t)f.parts;
    if (x.type == CER_TYPE_BF16) return shrink_ranks<__bf16, __bf16, false, kAlong>(c, f, s);
    if (x.type == CER_TYPE_F16) return shrink_ranks<_Float16, _Float16, false, kAlong>(c, f, s);
    const bool columns = x.order == CER_ORDER_COLUMNS;
    if (weights == CER_TYPE_BF16) return columns ? shrink_ranks<float, __bf16, true, kAlong>(c, f, s) : shrink_ranks<float, __bf16, false, kAlong>(c, f, s);
    if (weights == CER_TYPE_F16) return columns ? shrink_ranks<float, _Float16, true, kAlong>(c, f, s) : shrink_ranks<float, _Float16, false, kAlong>(c, f, s);
    return columns ? shrink_ranks<float, float, true, kAlong>(c, f, s) : shrink_ranks<float, float, false, kAlong>(c, f, s);
}

template <class TX, class TW, bool kColumns, bool kAlong>
int expand_tiles(ExpandArgs c, hipStream_t s) {
    const int64_t blocks = (c.length + 63) / 64;
    const size_t few = (size_t)16 * ((c.w.rank + 15) / 16 * 16 + 4) * 4;
    // ranks in fours: a load takes four of a row, or four rows, and must not leave them
    if (c.tokens <= kFewTokens || c.length < 64 || c.w.rank % 4) {
        const int64_t across = (c.tokens + 15) / 16;
        const dim3 grid((unsigned)across, (unsigned)blocks);
        // sixteen waves for up to sixteen adapters, where that many workgroups run together; else eight
        if (across * blocks <= 512) expand_kernel<TX, TW, kColumns, kAlong, 1024><<<grid, 1024, few, s>>>(c);
        else expand_kernel<TX, TW, kColumns, kAlong, 512><<<grid, 512, few, s>>>(c);
    } else {
        // the tokens' hidden is made ready once for a workgroup: as many blocks for each as leave about four workgroups for a compute unit
        const int64_t across = c.tokens / 64, most = std::max<int64_t>(1, 1024 / across), whole = c.length / 64;
        c.blocks = (uint32_t)std::max<int64_t>(kWaves, (whole + most - 1) / most);
        c.groups = (uint32_t)((whole + c.blocks - 1) / c.blocks);
        const int64_t ends = (c.tokens % 64 + 15) / 16 * blocks + (c.length % 64 ? across * 4 : 0);
        const size_t lds = std::max(few, (size_t)3 * 64 * ((c.w.rank + 31) / 32 * 32 + 8) * 2);
        // An adapter's weights stay in registers for a block's 64 tokens where they are few; ranks over 64 in half as many waves then, which
        // pays in rows (4096 tokens of 64 features -> 4096, rank 128, 8 requests: 52 -> 40 us, with two pieces of hidden) and not in columns (rank 128, one: 65 -> 70).
        constexpr int kMost = sizeof(TX) == 2 || kWeightPieces<TW> == 1 ? 2 : 1, kRows = !kColumns && kWeightPieces<TW> == 1 ? 4 : kMost;  // times 32 ranks
        const auto kernel = c.w.rank <= 32           ? expand_wide_kernel<TX, TW, kColumns, kAlong, 1>
                            : c.w.rank <= 32 * kMost ? expand_wide_kernel<TX, TW, kColumns, kAlong, kMost>
                            : c.w.rank <= 32 * kRows ? expand_wide_kernel<TX, TW, kColumns, kAlong, kRows>
                                                     : expand_wide_kernel<TX, TW, kColumns, kAlong, 0>;
        if (lds > 60 * 1024)  // ranks over 128
            if (int e = (int)hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds)) return e;
        kernel<<<(unsigned)(across * c.groups + ends), kBlock, lds, s>>>(c);
    }
    return (int)hipGetLastError();
}
template <bool kAlong>
int expand(ExpandArgs c, const cer_tokens_t& base, const cer_tokens_t& y, int32_t weights, hipStream_t s) {
    c.base = base.data, c.ldbase = base.ld, c.y = y.data, c.ldy = y.ld;
    if (y.type == CER_TYPE_BF16) return expand_tiles<__bf16, __bf16, false, kAlong>(c, s);
    if (y.type == CER_TYPE_F16) return expand_tiles<_Float16, _Float16, false, kAlong>(c, s);
    const bool columns = y.order == CER_ORDER_COLUMNS;
    if (weights == CER_TYPE_BF16) return columns ? expand_tiles<float, __bf16, true, kAlong>(c, s) : expand_tiles<float, __bf16, false, kAlong>(c, s);
    if (weights == CER_TYPE_F16) return columns ? expand_tiles<float, _Float16, true, kAlong>(c, s) : expand_tiles<float, _Float16, false, kAlong>(c, s);
    return columns ? expand_tiles<float, float, true, kAlong>(c, s) : expand_tiles<float, float, false, kAlong>(c, s);
}

// How one side's outer products are cut: the tokens into ranges where an adapter's workgroups alone would be few (up to about 1024 workgroups, 512 tokens
// at least), the long axis into 64 elements, or 128 for activations in 16 bits and ranks up to 32.
void outer_shape(OuterArgs& c, const cer_tokens_t& x) {
    c.x = x.data, c.ldx = x.ld;
    const int64_t without = c.w.adapters * ((c.length + 127) / 128);
    c.parts = (uint32_t)std::max<int64_t>(1, std::min<int64_t>({16, c.tokens / 512, 1024 / without}));
    c.range = ((c.tokens + c.parts - 1) / c.parts + 31) / 32 * 32;
    const int ranks = c.w.rank <= 16 ? 1 : c.w.rank <= 32 ? 2 : 4;
    const int elements = x.type != CER_TYPE_F32 && ranks < 4 ? 128 : 64;
    c.blocks = (uint32_t)((c.length + elements - 1) / elements * ((c.w.rank + 16 * ranks - 1) / (16 * ranks)));
}

// dA and dB, or one of them (`both` false: a).
int outer(OuterPair p, bool both, const cer_tokens_t& x_of_a, const cer_tokens_t& x_of_b, hipStream_t s) {
    outer_shape(p.a, x_of_a);
    if (both) outer_shape(p.b, x_of_b);
    OuterArgs* const sides[2] = {&p.a, &p.b};
    float* out[2];
    int64_t numbers[2], room = 0;
    for (int k = 0; k < (both ? 2 : 1); ++k) {
        out[k] = sides[k]->out;
        numbers[k] = sides[k]->w.adapters * sides[k]->w.rank * sides[k]->length;
        if (sides[k]->parts > 1) room += sides[k]->parts * numbers[k];
    }
    Temporary t((size_t)room * 4, s);
    if (t.error) return t.error;
    float* next = t.floats();
    for (int k = 0; k < (both ? 2 : 1); ++k)
        if (sides[k]->parts > 1) {
            sides[k]->out = next;
            next += sides[k]->parts * numbers[k];
        }
    const dim3 grid(p.a.blocks + (both ? p.b.blocks : 0), (unsigned)p.a.w.adapters, both ? std::max(p.a.parts, p.b.parts) : p.a.parts);
    const int rank = p.a.w.rank;
    auto go = [&](auto kernel) { kernel<<<grid, kOuterBlock, 0, s>>>(p); };
    auto of_ranks = [&](auto one, auto two, auto four) {
        if (rank <= 16) go(one);
        else if (rank <= 32) go(two);
        else go(four);
    };
    if (x_of_a.type == CER_TYPE_BF16) of_ranks(outer16_kernel<__bf16, 1, 8>, outer16_kernel<__bf16, 2, 8>, outer16_kernel<__bf16, 4, 4>);
    else if (x_of_a.type == CER_TYPE_F16) of_ranks(outer16_kernel<_Float16, 1, 8>, outer16_kernel<_Float16, 2, 8>, outer16_kernel<_Float16, 4, 4>);
    else if (x_of_a.order == CER_ORDER_COLUMNS) of_ranks(outer_kernel<float, true, 1>, outer_kernel<float, true, 2>, outer_kernel<float, true, 4>);
    else of_ranks(outer_kernel<float, false, 1>, outer_kernel<float, false, 2>, outer_kernel<float, false, 4>);
    if (int e = (int)hipGetLastError()) return e;
    for (int k = 0; k < (both ? 2 : 1); ++k) {
        if (sides[k]->parts == 1) continue;
        outer_sum_kernel<<<(unsigned)((numbers[k] + 4 * kBlock - 1) / (4 * kBlock)), kBlock, 0, s>>>(sides[k]->out, sides[k]->parts, numbers[k], out[k]);
        if (int e = (int)hipGetLastError()) return e;
    }
    return 0;
}

int clear(float* out, int64_t numbers, hipStream_t s) {  // the sum of no parts
    outer_sum_kernel<<<(unsigned)((numbers + 4 * kBlock - 1) / (4 * kBlock)), kBlock, 0, s>>>(nullptr, 0, numbers, out);
    return (int)hipGetLastError();
}

Weights side_a(const cer_adapters_t& w) { return {w.A, w.stride_a, w.ld_a, w.ranks, w.scales, (int32_t)w.adapters, (int32_t)w.rank}; }
Weights side_b(const cer_adapters_t& w) { return {w.B, w.stride_b, w.ld_b, w.ranks, w.scales, (int32_t)w.adapters, (int32_t)w.rank}; }
}  // namespace

int64_t adapter_workspace(int64_t tokens, int64_t rank, int64_t in, int64_t) {
    return std::max(ShrinkShape(tokens, rank, in, false, 16).parts, ShrinkShape(tokens, rank, in, true, 16).parts) * tokens * rank * 4;  // the most, whatever the adapters' number
}

int launch_adapters(const AdapterCall& c, hipStream_t s) {
    const ShrinkShape f(c.tokens, c.w.rank, c.w.in, c.x.order == CER_ORDER_COLUMNS, c.w.adapters);
    const int64_t bytes = adapter_workspace(c.tokens, c.w.rank, c.w.in, c.w.out);
    Temporary t(c.workspace ? 0 : (size_t)bytes, s);
    if (t.error) return t.error;
    float* part = c.workspace ? static_cast<float*>(c.workspace) : t.floats();
    ShrinkArgs a{};
    a.w = side_a(c.w), a.index = c.index, a.tokens = c.tokens, a.length = c.w.in, a.out = part;
    if (int e = shrink<true>(a, f, c.x, c.w.type, s)) return e;
    ExpandArgs b{};
    b.w = side_b(c.w), b.index = c.index, b.tokens = c.tokens, b.length = c.w.out;
    b.part = part, b.parts = (uint32_t)f.parts, b.hidden = c.hidden, b.scale = true;
    return expand<false>(b, c.base, c.y, c.w.type, s);
}

int launch_adapters_backward(const AdapterBackwardCall& c, hipStream_t s) {
    if (c.tokens == 0) {
        if (c.dA)
            if (int e = clear(c.dA, c.w.adapters * c.w.rank * c.w.in, s)) return e;
        return c.dB ? clear(c.dB, c.w.adapters * c.w.rank * c.w.out, s) : 0;
    }
    const ShrinkShape f(c.tokens, c.w.rank, c.w.out, c.dy.order == CER_ORDER_COLUMNS, c.w.adapters);
    const int64_t one = c.tokens * c.w.rank;
    const bool d_wanted = c.dx.data || c.dA, k16 = c.dy.type != CER_TYPE_F32;
    // d, the parts of it, and the planes of d and hidden
    const int64_t parts = d_wanted && (f.parts > 1 || k16) ? f.parts : 0;
    const int64_t plane_floats = k16 ? (c.tokens + 31) / 32 * ((c.w.rank + 15) / 16) * (32 * 16 * 3 / 2) : 0;
    const int64_t place = (one + 63) / 64 * 64;
    Temporary t((size_t)((1 + parts) * place + 2 * plane_floats) * 4, s);
    if (t.error) return t.error;
    float *d = t.floats(), *part = d + place;
    uint16_t* d_planes = c.dA && k16 ? reinterpret_cast<uint16_t*>(d + (1 + parts) * place) : nullptr;
    uint16_t* hidden_planes = c.dB && k16 ? reinterpret_cast<uint16_t*>(d + (1 + parts) * place + plane_floats) : nullptr;
    ShrinkArgs a{};
    a.w = side_b(c.w), a.index = c.index, a.tokens = c.tokens, a.length = c.w.out;
    if (d_wanted) {
        a.out = parts ? part : d, a.scale = !parts;
        if (int e = shrink<false>(a, f, c.dy, c.w.type, s)) return e;
    }
    a.out = d, a.scale = true;
    if (k16) {
        const unsigned first = d_wanted ? 0 : 1, last = c.dB ? 2 : 1;
        if (first < last) {
            // where hidden alone is wanted, its half of the grid runs behind an empty one
            planes_kernel<<<dim3((unsigned)((c.tokens + 31) / 32), last), kBlock, 0, s>>>(a, part, d_wanted ? (uint32_t)f.parts : 0, c.hidden, d_planes, hidden_planes);
            if (int e = (int)hipGetLastError()) return e;
        }
    } else if (parts) {
        shrink_sum_kernel<<<(unsigned)((one + kBlock - 1) / kBlock), kBlock, 0, s>>>(a, part, (uint32_t)f.parts);
        if (int e = (int)hipGetLastError()) return e;
    }
    if (c.dA || c.dB) {
        OuterArgs of_a{}, of_b{};
        of_a.g = d, of_a.planes = d_planes, of_a.w = side_a(c.w), of_a.index = c.index, of_a.tokens = c.tokens, of_a.length = c.w.in, of_a.out = c.dA;
        of_b.g = c.hidden, of_b.planes = hidden_planes, of_b.w = side_b(c.w), of_b.index = c.index, of_b.tokens = c.tokens, of_b.length = c.w.out, of_b.out = c.dB;
        of_b.scale = of_b.rank_last = true;
        const bool both = c.dA && c.dB;
        if (int e = outer(c.dA ? OuterPair{of_a, of_b} : OuterPair{of_b, {}}, both, c.dA ? c.x : c.dy, c.dy, s)) return e;
    }
    if (c.dx.data) {
        ExpandArgs b{};
        b.w = side_a(c.w), b.index = c.index, b.tokens = c.tokens, b.length = c.w.in;
        b.part = d, b.parts = 1;
        return expand<true>(b, c.base, c.dx, c.w.type, s);
    }
    return 0;
}

}  // namespace cer
