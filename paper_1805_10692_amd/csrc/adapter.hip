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
// Activations in 32 bits are multiplied by the 32-bit matrix instruction, and so is everything behind `hidden` and d, which are kept in 32 bits;
// activations in 16 bits meet weights of the same type in `shrink` in the 16-bit instruction, which adds up in 32.
#include <algorithm>
#include <type_traits>

#include "operators.hpp"

namespace cer {
namespace {

using F4 = Vec<float, 4>;
constexpr int kBlock = 256, kWaves = kBlock / 64;
constexpr int kMostTile = 64;  // tokens of a workgroup

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
struct Present {
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

// Up to N elements in their own type, 0 past `left`.
template <class T, int N>
__device__ __forceinline__ Vec<T, N> load_own(const T* p, int64_t left) {
    if (left >= N) return load<T, N>(p);
    Vec<T, N> v;
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = j < left ? p[j] : (T)0.f;
    return v;
}

// ---- shrink ---------------------------------------------------------------------------------------------------------------------
struct ShrinkArgs {
    Weights w;
    const int32_t* index;
    int64_t tokens, length;  // of the long axis
    const void* x;
    int64_t ldx;
    int64_t part;  // elements of the long axis for a workgroup (blockIdx.y), a multiple of 32
    float* out;    // [gridDim.y][tokens][rank]
    bool scale;    // times s_a
};

// kTiles * 16 tokens, kRanks * 16 ranks from blockIdx.z on.  Lane (i, g) = (lane % 16, lane / 16) holds of both sides' operands row i's (a rank's, a
// token's) elements of the long axis that belong to g: 4 of 16 in 32 bits (four instructions of 4, each taking one of every g's), 8 of 32 in 16.
// The sides agree on which, and that is all that their order has to do.
template <class TX, class TW, bool kColumns, bool kAlong, int kTiles, int kRanks>
__global__ __launch_bounds__(kBlock) void shrink_kernel(ShrinkArgs c) {
    constexpr bool k16 = sizeof(TX) == 2;
    constexpr int E = k16 ? 8 : 4, kStep = 4 * E, kTile = 16 * kTiles, kPitch = 16 * kRanks + 4;
    using Operand = std::conditional_t<k16, Vec<TX, E>, F4>;
    __shared__ Present present;
    __shared__ float sums[kWaves][kTile][kPitch];
    const int64_t t0 = (int64_t)blockIdx.x * kTile;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4, r0 = blockIdx.z * 16 * kRanks;
    list_adapters(present, c.index, t0, kTile, c.tokens, c.w.adapters);
    const int slots = present.slots;
    const int abreast = slots >= kWaves ? kWaves : slots >= 2 ? 2 : 1, pieces = kWaves / abreast, piece = wave / abreast;
    // this wave's piece of the long axis
    const int64_t from = blockIdx.y * c.part, to = from + c.part < c.length ? from + c.part : c.length;
    const int64_t each = ((to - from + pieces - 1) / pieces + kStep - 1) / kStep * kStep;
    const int64_t k0 = from + piece * each, k1 = k0 + each < to ? k0 + each : to;
    int token[kTiles];  // in the tile
#pragma unroll
    for (int s = 0; s < kTiles; ++s) token[s] = kColumns ? kTiles * i + s : 16 * s + i;
    const TX* x[kTiles];
    if (kColumns) {
        x[0] = static_cast<const TX*>(c.x) + (t0 + kTiles * i < c.tokens ? t0 + kTiles * i : 0);
    } else {
#pragma unroll
        for (int s = 0; s < kTiles; ++s)
            x[s] = static_cast<const TX*>(c.x) + (t0 + token[s] < c.tokens ? t0 + token[s] : c.tokens - 1) * c.ldx;
    }
    const int64_t abreast_left = t0 + kTiles * i < c.tokens ? c.tokens - (t0 + kTiles * i) : 0;  // columns: tokens of the lane's vector
    for (int q = wave % abreast; q < slots; q += abreast) {
        const int a = __builtin_amdgcn_readfirstlane(present.slot[q]);
        const int rank = rank_of(c.w, a);
        if (rank <= r0) continue;
        const TW* w = static_cast<const TW*>(c.w.w) + a * c.w.stride;
        const TW* row[kRanks];  // of a rank past the last one: the last one's, its products are not kept
#pragma unroll
        for (int r = 0; r < kRanks; ++r) {
            const int at = r0 + 16 * r + i < rank ? r0 + 16 * r + i : rank - 1;
            row[r] = kAlong ? w + at * c.w.ld : w + at;
        }
        F4 acc[kTiles][kRanks];
#pragma unroll
        for (int s = 0; s < kTiles; ++s)
#pragma unroll
            for (int r = 0; r < kRanks; ++r) acc[s][r] = 0.f;
        auto step = [&](int64_t k, auto whole) {  // whole: nothing of the step is past k1
            constexpr bool kWhole = decltype(whole)::value;
            const int64_t at = k + E * g, left = kWhole ? E : k1 - at;
            Operand xs[kTiles], ws[kRanks];
            if constexpr (kColumns) {
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    Vec<float, 4> v = 0.f;
                    if (kWhole || j < left) {
                        const TX* p = x[0] + (at + j) * c.ldx;
                        if constexpr (kTiles == 1) v[0] = abreast_left > 0 ? p[0] : 0.f;
                        if constexpr (kTiles == 2) {
                            const Vec<float, 2> u = load_some<TX, 2>(p, abreast_left);
                            v[0] = u[0], v[1] = u[1];
                        }
                        if constexpr (kTiles == 4) v = load_some<TX, 4>(p, abreast_left);
                    }
#pragma unroll
                    for (int s = 0; s < kTiles; ++s) xs[s][j] = v[s];
                }
            } else {
#pragma unroll
                for (int s = 0; s < kTiles; ++s) {
                    if constexpr (k16) xs[s] = load_own<TX, E>(x[s] + at, left);
                    else xs[s] = load_some<TX, E>(x[s] + at, left);
                }
            }
#pragma unroll
            for (int r = 0; r < kRanks; ++r) {
                if constexpr (kAlong) {
                    if constexpr (k16) ws[r] = load_own<TW, E>(row[r] + at, left);
                    else ws[r] = load_some<TW, E>(row[r] + at, left);
                } else {
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        TW v = (TW)0.f;
                        if (kWhole || j < left) v = row[r][(at + j) * c.w.ld];
                        if constexpr (k16) ws[r][j] = v;
                        else ws[r][j] = (float)v;
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
                        for (int j = 0; j < 4; ++j) acc[s][r] = product(ws[r][j], xs[s][j], acc[s][r]);
                    }
                }
        };
        int64_t k = k0;
        constexpr int kAhead = kTiles * kRanks >= 8 ? 2 : 4;  // steps whose loads are on their way together
        for (; k + kAhead * kStep <= k1; k += kAhead * kStep)
#pragma unroll
            for (int u = 0; u < kAhead; ++u) step(k + u * kStep, std::true_type());
        for (; k + kStep <= k1; k += kStep) step(k, std::true_type());
        if (k < k1) step(k, std::false_type());
#pragma unroll
        for (int s = 0; s < kTiles; ++s)
            if (present.adapter[token[s]] == a)
#pragma unroll
                for (int r = 0; r < kRanks; ++r) *reinterpret_cast<F4*>(&sums[piece][token[s]][16 * r + 4 * g]) = acc[s][r];
    }
    __syncthreads();
    float* out = c.out + (int64_t)blockIdx.y * c.tokens * c.w.rank;
    for (int e = threadIdx.x; e < kTile * 16 * kRanks; e += kBlock) {
        const int t = e / (16 * kRanks), r = e % (16 * kRanks);
        if (t0 + t >= c.tokens || r0 + r >= c.w.rank) continue;
        const int a = present.adapter[t];
        float all = 0.f;
        if (a >= 0 && r0 + r < rank_of(c.w, a)) {
            for (int p = 0; p < pieces; ++p) all += sums[p][t][r];
            if (c.scale) all *= scale_of(c.w, a);
        }
        out[(t0 + t) * c.w.rank + r0 + r] = all;
    }
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
};

// kTiles * 16 tokens; a wave takes pairs of adapter and 64 elements of the long axis.  Element o0 + 4 i + j is row (column) i of the tile j of four:
// the operands' loads have four neighbours in a lane where the weights lie that way, and so do the results: lane (i, g) holds
// o0 + 16 g .. + 15 of token i (rows), or elements o0 + 4 i + j of tokens 4 g .. + 3 (columns).
template <class TX, class TW, bool kColumns, bool kAlong, int kTiles>
__global__ __launch_bounds__(kBlock) void expand_kernel(ExpandArgs c) {
    constexpr int kTile = 16 * kTiles;
    extern __shared__ float hidden[];  // [tile][pitch], 0 past the rank and for tokens without an adapter
    __shared__ Present present;
    const int64_t t0 = (int64_t)blockIdx.x * kTile;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
    const int rank16 = (c.w.rank + 15) / 16 * 16, pitch = rank16 + 4;
    list_adapters(present, c.index, t0, kTile, c.tokens, c.w.adapters);
    for (int e = threadIdx.x; e < kTile * rank16; e += kBlock) {
        const int t = e / rank16, r = e % rank16, a = present.adapter[t];
        float sum = 0.f;
        if (t0 + t < c.tokens && r < c.w.rank) {
            const float* p = c.part + (t0 + t) * c.w.rank + r;
            if (a >= 0 && r < rank_of(c.w, a))
#pragma unroll 8
                for (uint32_t k = 0; k < c.parts; ++k) sum += p[k * c.tokens * c.w.rank];
            if (c.hidden && blockIdx.y == 0) c.hidden[(t0 + t) * c.w.rank + r] = sum;
            if (a >= 0 && c.scale) sum *= scale_of(c.w, a);
        }
        hidden[t * pitch + r] = sum;
    }
    __syncthreads();
    const TX* base = static_cast<const TX*>(c.base);
    TX* y = static_cast<TX*>(c.y);
    // tokens without an adapter: a list entry of their own, unless y has what they get already
    const int slots = present.slots, jobs = slots + (present.none && c.base != c.y ? 1 : 0);
    const int64_t o_first = (int64_t)blockIdx.y * c.blocks * 64;
    for (int job = wave; job < jobs * (int)c.blocks; job += kWaves) {
        const int64_t o0 = o_first + job / jobs * 64;
        if (o0 >= c.length) break;
        const int a = job % jobs < slots ? __builtin_amdgcn_readfirstlane(present.slot[job % jobs]) : -1;
        const int64_t left = c.length - o0;
        F4 acc[kTiles][4];  // rows: [tile][j], elements 16 g + 4 (0 .. 3) + j; columns: [tile][j], tokens 4 g + (0 .. 3)
#pragma unroll
        for (int s = 0; s < kTiles; ++s) {
            if constexpr (kColumns) {
                const int64_t t = t0 + 16 * s + 4 * g;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[s][j] = base && 4 * i + j < left && t < c.tokens ? load_some<TX, 4>(base + (o0 + 4 * i + j) * c.ldbase + t, c.tokens - t) : F4(0.f);
            } else {
                const int64_t t = t0 + 16 * s + i;
                const bool mine = base && t < c.tokens && present.adapter[16 * s + i] == a;
                constexpr int V = 16 / sizeof(TX);
                Vec<float, 16> v;
#pragma unroll
                for (int q = 0; q < 16 / V; ++q) {
                    Vec<float, V> u = 0.f;
                    if (mine) u = load_some<TX, V>(base + t * c.ldbase + o0 + 16 * g + V * q, left - 16 * g - V * q);
#pragma unroll
                    for (int k = 0; k < V; ++k) v[V * q + k] = u[k];
                }
#pragma unroll
                for (int k = 0; k < 16; ++k) acc[s][k % 4][k / 4] = v[k];
            }
        }
        const int rank = a >= 0 ? rank_of(c.w, a) : 0;
        const TW* w = static_cast<const TW*>(c.w.w) + (a >= 0 ? a * c.w.stride : 0);
        for (int r0 = 0; r0 < rank; r0 += 16) {
            const int at = r0 + 4 * g;
            F4 ws[4];  // [j][element at + (0 .. 3)]
            if constexpr (kAlong) {  // w[r * ld + o]
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    F4 v = 0.f;
                    if (at + q < rank) v = load_some<TW, 4>(w + (at + q) * c.w.ld + o0 + 4 * i, left - 4 * i);
#pragma unroll
                    for (int j = 0; j < 4; ++j) ws[j][q] = v[j];
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) ws[j] = 4 * i + j < left ? load_some<TW, 4>(w + (o0 + 4 * i + j) * c.w.ld + at, rank - at) : F4(0.f);
            }
#pragma unroll
            for (int s = 0; s < kTiles; ++s) {
                const F4 h = *reinterpret_cast<const F4*>(&hidden[(16 * s + i) * pitch + at]);
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        acc[s][j] = kColumns ? product(h[q], ws[j][q], acc[s][j]) : product(ws[j][q], h[q], acc[s][j]);
            }
        }
#pragma unroll
        for (int s = 0; s < kTiles; ++s) {
            if constexpr (kColumns) {
                const int64_t t = t0 + 16 * s + 4 * g;
                bool mine[4], all = true;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    mine[k] = t + k < c.tokens && present.adapter[16 * s + 4 * g + k] == a;
                    all &= mine[k];
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (4 * i + j >= left) continue;
                    TX* p = y + (o0 + 4 * i + j) * c.ldy + t;
                    if (all) {
                        store_f32<TX, 4>(p, acc[s][j]);
                    } else {
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (mine[k]) p[k] = (TX)acc[s][j][k];
                    }
                }
            } else {
                const int64_t t = t0 + 16 * s + i;
                if (t >= c.tokens || present.adapter[16 * s + i] != a) continue;
                constexpr int V = 16 / sizeof(TX);
#pragma unroll
                for (int q = 0; q < 16 / V; ++q) {
                    Vec<float, V> u;
#pragma unroll
                    for (int k = 0; k < V; ++k) u[k] = acc[s][(V * q + k) % 4][(V * q + k) / 4];
                    store_some<TX, V>(y + t * c.ldy + o0 + 16 * g + V * q, u, left - 16 * g - V * q);
                }
            }
        }
    }
}

// ---- outer ----------------------------------------------------------------------------------------------------------------------
struct OuterArgs {
    const float* g;  // [tokens][rank]
    Weights w;       // adapters, ranks, scales
    const int32_t* index;
    int64_t tokens, length;
    const void* x;
    int64_t ldx;
    int64_t range;  // tokens for a workgroup (blockIdx.z), a multiple of 16
    float* out;     // [gridDim.z][adapters][rank][length], or kRankLast: [gridDim.z][adapters][length][rank]
    bool scale;
};

// Adapter blockIdx.y, 64 elements of the long axis, kRanks * 16 ranks; the waves share out the groups of 16 tokens in which the adapter occurs.
template <class TX, bool kColumns, bool kRankLast, int kRanks>
__global__ __launch_bounds__(kBlock) void outer_kernel(OuterArgs c) {
    constexpr int kGroups = 256;  // looked at together
    __shared__ int list[kGroups];
    __shared__ int count[kWaves];
    __shared__ F4 sums[kWaves / 2][kRanks * 4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4, a = blockIdx.y;
    const int rank_blocks = (c.w.rank + 16 * kRanks - 1) / (16 * kRanks);
    const int64_t o0 = (int64_t)(blockIdx.x / rank_blocks) * 64, left = c.length - o0;
    const int r0 = (int)(blockIdx.x % rank_blocks) * 16 * kRanks;
    const int rank = rank_of(c.w, a);
    const int64_t from = blockIdx.z * c.range, to = from + c.range < c.tokens ? from + c.range : c.tokens;
    F4 acc[kRanks][4];
#pragma unroll
    for (int r = 0; r < kRanks; ++r)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[r][j] = 0.f;
    for (int64_t first = from; first < to; first += kGroups * 16) {
        // the groups, in their order
        const int64_t mine = first + threadIdx.x * 16;
        bool some = false;
        for (int k = 0; k < 16; ++k) some |= mine + k < to && c.index[mine + k] == a;
        const unsigned long long here = __ballot(some);
        if (lane == 0) count[wave] = __popcll(here);
        __syncthreads();
        int at = __popcll(here & ((1ull << lane) - 1)), groups = 0;
        for (int k = 0; k < kWaves; ++k) {
            if (k < wave) at += count[k];
            groups += count[k];
        }
        if (some) list[at] = threadIdx.x;
        __syncthreads();
        if (rank > r0)
            for (int q = wave; q < groups; q += kWaves) {
                const int64_t t = first + list[q] * 16 + 4 * g;  // lane group g has tokens t .. t + 3
                bool own[4], every = true;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    own[k] = t + k < to && c.index[t + k] == a;
                    every &= own[k];
                }
                every = __all(every);
                F4 xs[4];  // [token k][element 4 i + j]
                if constexpr (kColumns) {
                    F4 v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        v[j] = 4 * i + j < left && t < to ? load_some<TX, 4>(static_cast<const TX*>(c.x) + (o0 + 4 * i + j) * c.ldx + t, to - t) : F4(0.f);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int j = 0; j < 4; ++j) xs[k][j] = v[j][k];
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        xs[k] = t + k < to ? load_some<TX, 4>(static_cast<const TX*>(c.x) + (t + k) * c.ldx + o0 + 4 * i, left - 4 * i) : F4(0.f);
                }
                float gs[kRanks][4];
#pragma unroll
                for (int r = 0; r < kRanks; ++r)
#pragma unroll
                    for (int k = 0; k < 4; ++k) gs[r][k] = own[k] && r0 + 16 * r + i < rank ? c.g[(t + k) * c.w.rank + r0 + 16 * r + i] : 0.f;
                if (!every)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (!own[k]) xs[k] = 0.f;
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int r = 0; r < kRanks; ++r)
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[r][j] = product(gs[r][k], xs[k][j], acc[r][j]);
            }
        __syncthreads();  // the list is made anew
    }
    // the waves' sums: the upper half to the lower one, twice
#pragma unroll
    for (int half = kWaves / 2; half; half /= 2) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int r = 0; r < kRanks; ++r)
#pragma unroll
                for (int j = 0; j < 4; ++j) sums[wave - half][4 * r + j][lane] = acc[r][j];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int r = 0; r < kRanks; ++r)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[r][j] += sums[wave][4 * r + j][lane];
        __syncthreads();
    }
    if (wave) return;
    const float scale = c.scale ? scale_of(c.w, a) : 1.f;
    float* out = c.out + ((int64_t)blockIdx.z * c.w.adapters + a) * c.w.rank * c.length;
#pragma unroll
    for (int r = 0; r < kRanks; ++r) {
        const int at = r0 + 16 * r + 4 * g;
        if constexpr (kRankLast) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (4 * i + j < left && at < c.w.rank) store_some<float, 4>(out + (o0 + 4 * i + j) * c.w.rank + at, acc[r][j] * scale, c.w.rank - at);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (at + k >= c.w.rank) continue;
                F4 v;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = acc[r][j][k] * scale;
                store_some<float, 4>(out + (at + k) * c.length + o0 + 4 * i, v, left - 4 * i);
            }
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
    ShrinkShape(int64_t tokens, int64_t rank, int64_t length) {
        ranks = rank <= 16 ? 1 : rank <= 32 ? 2 : rank <= 64 ? 4 : 8;
        tiles = tokens <= 256 ? 1 : tokens <= 1024 || ranks == 8 ? 2 : 4;
        const int64_t blocks = (tokens + 16 * tiles - 1) / (16 * tiles);
        const int64_t want = std::max<int64_t>(1, std::min<int64_t>((1024 + blocks - 1) / blocks, (length + 255) / 256));
        part = ((length + want - 1) / want + 31) / 32 * 32;
        parts = (int)((length + part - 1) / part);
    }
};

template <class TX, class TW, bool kColumns, bool kAlong, int kTiles>
int shrink_ranks(const ShrinkArgs& c, const ShrinkShape& f, hipStream_t s) {
    const dim3 grid((unsigned)((c.tokens + 16 * kTiles - 1) / (16 * kTiles)), f.parts, (unsigned)((c.w.rank + 16 * f.ranks - 1) / (16 * f.ranks)));
    if (f.ranks == 1) shrink_kernel<TX, TW, kColumns, kAlong, kTiles, 1><<<grid, kBlock, 0, s>>>(c);
    else if (f.ranks == 2) shrink_kernel<TX, TW, kColumns, kAlong, kTiles, 2><<<grid, kBlock, 0, s>>>(c);
    else if (f.ranks == 4) shrink_kernel<TX, TW, kColumns, kAlong, kTiles, 4><<<grid, kBlock, 0, s>>>(c);
    else if constexpr (kTiles <= 2) shrink_kernel<TX, TW, kColumns, kAlong, kTiles, 8><<<grid, kBlock, 0, s>>>(c);
    return (int)hipGetLastError();
}
template <class TX, class TW, bool kColumns, bool kAlong>
int shrink_tiles(const ShrinkArgs& c, const ShrinkShape& f, hipStream_t s) {
    if (f.tiles == 1) return shrink_ranks<TX, TW, kColumns, kAlong, 1>(c, f, s);
    if (f.tiles == 2) return shrink_ranks<TX, TW, kColumns, kAlong, 2>(c, f, s);
    return shrink_ranks<TX, TW, kColumns, kAlong, 4>(c, f, s);
}
template <bool kAlong>
int shrink(ShrinkArgs c, const ShrinkShape& f, const cer_tokens_t& x, int32_t weights, hipStream_t s) {
    c.x = x.data, c.ldx = x.ld, c.part = f.part;
    if (x.type == CER_TYPE_BF16) return shrink_tiles<__bf16, __bf16, false, kAlong>(c, f, s);
    if (x.type == CER_TYPE_F16) return shrink_tiles<_Float16, _Float16, false, kAlong>(c, f, s);
    const bool columns = x.order == CER_ORDER_COLUMNS;
    if (weights == CER_TYPE_BF16) return columns ? shrink_tiles<float, __bf16, true, kAlong>(c, f, s) : shrink_tiles<float, __bf16, false, kAlong>(c, f, s);
    if (weights == CER_TYPE_F16) return columns ? shrink_tiles<float, _Float16, true, kAlong>(c, f, s) : shrink_tiles<float, _Float16, false, kAlong>(c, f, s);
    return columns ? shrink_tiles<float, float, true, kAlong>(c, f, s) : shrink_tiles<float, float, false, kAlong>(c, f, s);
}

template <class TX, class TW, bool kColumns, bool kAlong>
int expand_tiles(ExpandArgs c, hipStream_t s) {
    const int tiles = c.tokens <= 256 ? 1 : c.tokens <= 1024 || c.w.rank > 128 ? 2 : 4;
    const int64_t across = (c.tokens + 16 * tiles - 1) / (16 * tiles), blocks = (c.length + 63) / 64;
    c.blocks = across * blocks >= 2048 ? 4 : 1;
    const dim3 grid((unsigned)across, (unsigned)((blocks + c.blocks - 1) / c.blocks));
    const size_t lds = (size_t)16 * tiles * ((c.w.rank + 15) / 16 * 16 + 4) * 4;
    if (tiles == 1) expand_kernel<TX, TW, kColumns, kAlong, 1><<<grid, kBlock, lds, s>>>(c);
    else if (tiles == 2) expand_kernel<TX, TW, kColumns, kAlong, 2><<<grid, kBlock, lds, s>>>(c);
    else expand_kernel<TX, TW, kColumns, kAlong, 4><<<grid, kBlock, lds, s>>>(c);
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

template <class TX, bool kColumns, bool kRankLast>
int outer_ranks(const OuterArgs& c, unsigned parts, hipStream_t s) {
    const int ranks = c.w.rank <= 16 ? 1 : c.w.rank <= 32 ? 2 : 4;
    const dim3 grid((unsigned)((c.length + 63) / 64 * ((c.w.rank + 16 * ranks - 1) / (16 * ranks))), (unsigned)c.w.adapters, parts);
    if (ranks == 1) outer_kernel<TX, kColumns, kRankLast, 1><<<grid, kBlock, 0, s>>>(c);
    else if (ranks == 2) outer_kernel<TX, kColumns, kRankLast, 2><<<grid, kBlock, 0, s>>>(c);
    else outer_kernel<TX, kColumns, kRankLast, 4><<<grid, kBlock, 0, s>>>(c);
    return (int)hipGetLastError();
}

// The tokens are cut into ranges where an adapter's workgroups alone would be few or one of them long: parts of up to 2048 tokens.
template <bool kRankLast>
int outer(OuterArgs c, const cer_tokens_t& x, hipStream_t s) {
    c.x = x.data, c.ldx = x.ld;
    const unsigned parts = (unsigned)std::max<int64_t>(1, std::min<int64_t>(8, c.tokens / 1024));
    c.range = ((c.tokens + parts - 1) / parts + 15) / 16 * 16;
    const int64_t numbers = c.w.adapters * c.w.rank * c.length;
    float* out = c.out;
    Temporary t(parts > 1 ? (size_t)parts * numbers * 4 : 0, s);
    if (t.error) return t.error;
    if (parts > 1) c.out = t.floats();
    int e;
    if (x.type == CER_TYPE_BF16) e = outer_ranks<__bf16, false, kRankLast>(c, parts, s);
    else if (x.type == CER_TYPE_F16) e = outer_ranks<_Float16, false, kRankLast>(c, parts, s);
    else if (x.order == CER_ORDER_COLUMNS) e = outer_ranks<float, true, kRankLast>(c, parts, s);
    else e = outer_ranks<float, false, kRankLast>(c, parts, s);
    if (!e && parts > 1) {
        outer_sum_kernel<<<(unsigned)((numbers + 4 * kBlock - 1) / (4 * kBlock)), kBlock, 0, s>>>(c.out, parts, numbers, out);
        e = (int)hipGetLastError();
    }
    return e;
}

int clear(float* out, int64_t numbers, hipStream_t s) {  // the sum of no parts
    outer_sum_kernel<<<(unsigned)((numbers + 4 * kBlock - 1) / (4 * kBlock)), kBlock, 0, s>>>(nullptr, 0, numbers, out);
    return (int)hipGetLastError();
}

Weights side_a(const cer_adapters_t& w) { return {w.A, w.stride_a, w.ld_a, w.ranks, w.scales, (int32_t)w.adapters, (int32_t)w.rank}; }
Weights side_b(const cer_adapters_t& w) { return {w.B, w.stride_b, w.ld_b, w.ranks, w.scales, (int32_t)w.adapters, (int32_t)w.rank}; }
}  // namespace

int64_t adapter_workspace(int64_t tokens, int64_t rank, int64_t in, int64_t) {
    return ShrinkShape(tokens, rank, in).parts * tokens * rank * 4;
}

int launch_adapters(const AdapterCall& c, hipStream_t s) {
    const ShrinkShape f(c.tokens, c.w.rank, c.w.in);
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
    const ShrinkShape f(c.tokens, c.w.rank, c.w.out);
    const int64_t one = c.tokens * c.w.rank;
    if (c.dx.data || c.dA) {
        Temporary t((size_t)(f.parts > 1 ? f.parts + 1 : 1) * one * 4, s);
        if (t.error) return t.error;
        float* d = t.floats();
        ShrinkArgs a{};
        a.w = side_b(c.w), a.index = c.index, a.tokens = c.tokens, a.length = c.w.out;
        a.out = f.parts > 1 ? d + one : d, a.scale = f.parts == 1;
        if (int e = shrink<false>(a, f, c.dy, c.w.type, s)) return e;
        if (f.parts > 1) {
            a.out = d, a.scale = true;
            shrink_sum_kernel<<<(unsigned)((one + kBlock - 1) / kBlock), kBlock, 0, s>>>(a, d + one, (uint32_t)f.parts);
            if (int e = (int)hipGetLastError()) return e;
        }
        if (c.dA) {  // before dx, which may lie where x does
            OuterArgs o{};
            o.g = d, o.w = side_a(c.w), o.index = c.index, o.tokens = c.tokens, o.length = c.w.in, o.out = c.dA;
            if (int e = outer<false>(o, c.x, s)) return e;
        }
        if (c.dx.data) {
            ExpandArgs b{};
            b.w = side_a(c.w), b.index = c.index, b.tokens = c.tokens, b.length = c.w.in;
            b.part = d, b.parts = 1;
            if (int e = expand<true>(b, c.base, c.dx, c.w.type, s)) return e;
        }
    }
    if (c.dB) {
        OuterArgs o{};
        o.g = c.hidden, o.w = side_b(c.w), o.index = c.index, o.tokens = c.tokens, o.length = c.w.out, o.out = c.dB, o.scale = true;
        if (int e = outer<true>(o, c.dy, s)) return e;
    }
    return 0;
}

}  // namespace cer
