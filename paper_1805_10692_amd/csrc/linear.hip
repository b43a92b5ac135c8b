// Dense products with an epilogue: z = X W^T + b, Y = r + act(z), and the gradients of X, W and b.
//
// Three products, one kernel:   C[i][j] = sum_k A(i, k) B(j, k)
//     Y  (tokens x out)   A = X,     B = W         both with k side by side in memory
//     dX (tokens x in)    A = dz,    B = W         B with j side by side
//     dW (out x in)       A = dz,    B = X         A with i, B with j side by side (k: tokens)
// and for activations in columns the same with the operands' places and orders exchanged, so that C's rows are always contiguous.
//
// A workgroup forms a tile of C.  128 bytes of k (64 numbers of 16 bits, 32 of fp32) of all its rows go from memory into LDS while the tiles before
// are multiplied: straight there where all of it is whole 16 bytes at addresses of that kind, an operand whose k lies a line apart as it is, to be
// turned where it is read; else through registers, by element-aligned loads, so that any place and leading dimension works, and turned on the way.  LDS holds rows of 128 bytes whose eight 16-byte chunks are permuted (`place`), so that both the turned
// stores and the operand loads of 32 rows touch every bank evenly.  The matrix instruction takes B's rows as its first operand: a lane
// then has four neighbouring j of one i.  fp32 goes through the 32-bit instruction.  Sums are fp32; each C is rounded once, after the epilogue.
// Where the tiles are too few for the chip the contraction is cut into parts, which a second launch adds up in their order (`plan_of`).
//
// What bounds it: the matrix cores and the way through LDS.  4096 x 4096 -> 4096 bf16 in one round of 256 tiles of 256 x 256: 113 us, 1214 TFLOP/s, over 300 calls on the same inputs,
// 121 over 20 (a library product of that size 111 and 117); through registers 126 where the direct way took 119, of which without loads 123, without stores to LDS either 111,
// without reading LDS 106, products and barriers alone 89 (the chip's clock falls under them).  fp32: 2048 x 4096 -> 4096 491 us, 140 TFLOP/s of 154, 553 over 20; through registers 105 - 135.
// 4096 tokens, 4096 -> 9216 bf16: forward 310 us on new inputs in each call, 288 on the same ones (2.25 rounds, and the epilogue of each by itself); backward 600, of which dX 267,
// dW 279, dz 53, db 5.
#include <algorithm>
#include <type_traits>

#include "operators.hpp"

namespace cer {
namespace {

using F16 = Vec<float, 16>;
using F4 = Vec<float, 4>;
using B8 = Vec<__bf16, 8>;
using H8 = Vec<_Float16, 8>;
using Chunk = Vec<uint32_t, 4>;

// ---- activations ----------------------------------------------------------------------------------------------------------------
constexpr float kHalfRoot = 0.70710678118654752f, kTanhFactor = 0.79788456080286536f, kTanhCube = 0.044715f;
// q = 1 / (1 + exp(-u)) and q (1 - q), neither by a difference; 0 and 1, and 0, at the ends.  The instructions' power of two and inverse are within 2^-23 of theirs, and
// rounding u / ln 2 adds |u| 2^-24: a division and a power rounded in full made a gradient of 4096 x 9216 bf16 take 66 us, these 56.
struct Logistic {
    float q, both;
    __device__ explicit Logistic(float u) {
        const float e = __builtin_amdgcn_exp2f(fabsf(u) * -1.4426950408889634f), inverse = __builtin_amdgcn_rcpf(1.f + e);
        q = u >= 0.f ? inverse : e * inverse;
        both = e * inverse * inverse;
    }
};
// (1 + erf(z / sqrt 2)) / 2
__device__ __forceinline__ float normal_share(float z) { return 0.5f * erfcf(-kHalfRoot * z); }
// (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))) / 2 is the logistic function of this.
__device__ __forceinline__ float tanh_argument(float z) { return 2.f * kTanhFactor * z * fmaf(kTanhCube * z, z, 1.f); }
// z . share; a share of 0 has its limit for an infinite z.
__device__ __forceinline__ float part_of(float z, float share) { return share == 0.f ? 0.f : z * share; }
// z / (1 + 2^-t); may be 0 from where 2^-t passes 2^126 (silu: z below -87.3, where it is over -1.1e-36)
__device__ __forceinline__ float share_of(float z, float t) { return part_of(z, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-t))); }
constexpr float kLog2E = 1.4426950408889634f;

__device__ __forceinline__ Vec<float, 4> activate(Vec<float, 4> z, int kind) {  // one branch for four
    switch (kind) {
        case CER_ACTIVATION_RELU:
#pragma unroll
            for (int q = 0; q < 4; ++q) z[q] = z[q] < 0.f ? 0.f : z[q];  // NaN stays
            break;
        case CER_ACTIVATION_GELU:
#pragma unroll
            for (int q = 0; q < 4; ++q) z[q] = part_of(z[q], normal_share(z[q]));
            break;
        case CER_ACTIVATION_GELU_TANH:
#pragma unroll
            for (int q = 0; q < 4; ++q) z[q] = share_of(z[q], z[q] * fmaf(2.f * kTanhFactor * kLog2E * kTanhCube * z[q], z[q], 2.f * kTanhFactor * kLog2E));
            break;
        case CER_ACTIVATION_SILU:
#pragma unroll
            for (int q = 0; q < 4; ++q) z[q] = share_of(z[q], z[q] * kLog2E);
            break;
        default: break;
    }
    return z;
}
__device__ __forceinline__ float slope(float z, int kind) {
    switch (kind) {
        case CER_ACTIVATION_RELU: return z > 0.f ? 1.f : z != z ? z : 0.f;
        case CER_ACTIVATION_GELU: return fmaf(part_of(z, expf(-0.5f * z * z)), 0.39894228040143268f, normal_share(z));
        case CER_ACTIVATION_GELU_TANH: {
            const Logistic v(tanh_argument(z));
            return v.both == 0.f ? v.q : fmaf(z * v.both, 2.f * kTanhFactor * fmaf(3.f * kTanhCube * z, z, 1.f), v.q);
        }
        case CER_ACTIVATION_SILU: {
            const Logistic v(z);
            return v.both == 0.f ? v.q : fmaf(z, v.both, v.q);
        }
        default: return 1.f;
    }
}

// ---- the product ----------------------------------------------------------------------------------------------------------------
struct Epilogue {
    const void* bias;  // along j, or i (bias_rows)
    int32_t bias_type;
    bool bias_rows;
    int32_t activation;
    const void* residual;
    void *pre, *out;
    int64_t ldr, ldp, ldo;
};
struct Product {
    const void *a, *b;
    int64_t lda, ldb;  // from a row to the next, or from one k to the next
    int64_t rows, columns, depth;
    Epilogue to;
    uint32_t tiles_i, tiles_j, parts;  // more than one: the contraction of every tile is cut
    int64_t depth_of_part;
    float* part;  // [tiles][parts][rows of a tile][columns of a tile]
};

// Four neighbouring j of row i, `left` of them in the matrix; `bias` along j, where it goes that way.
__device__ __forceinline__ Vec<float, 4> bias_along(const Epilogue& to, int64_t j, int64_t left) {
    return to.bias && !to.bias_rows ? load_some_of<4>(to.bias, to.bias_type, j, left) : Vec<float, 4>(0.f);
}
template <class T>
__device__ __forceinline__ void finish(const Epilogue& to, int64_t i, int64_t j, Vec<float, 4> z, Vec<float, 4> bias, int64_t left) {
    if (to.bias) z += to.bias_rows ? Vec<float, 4>(load_some_of<1>(to.bias, to.bias_type, i, 1)[0]) : bias;
    if (to.pre) store_some<T, 4>(static_cast<T*>(to.pre) + i * to.ldp + j, z, left);
    z = activate(z, to.activation);
    if (to.residual) z += load_some<T, 4>(static_cast<const T*>(to.residual) + i * to.ldr + j, left);
    store_some<T, 4>(static_cast<T*>(to.out) + i * to.ldo + j, z, left);
}

// Where chunk c of a row lies: eight neighbouring rows, and eight rows four (kFar: or eight) apart, have the same chunk in different places.
template <bool kFar>
__device__ __forceinline__ unsigned place(unsigned row, unsigned c) { return row * 8 + (c ^ (row & 7) ^ (row >> 3 & (kFar ? 7 : 3))); }

// Sixteen bytes of k of 32 rows on either side: lanes 0 - 31 have the lower chunk, 32 - 63 the next one.
template <class T>
__device__ __forceinline__ F16 multiply(Chunk a, Chunk b, F16 c) {
    if constexpr (sizeof(T) == 4) {
        const Vec<float, 4> x = __builtin_bit_cast(F4, a), y = __builtin_bit_cast(F4, b);
#pragma unroll
        for (int q = 0; q < 4; ++q) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[q], y[q], c, 0, 0, 0);
        return c;
    } else if constexpr (__is_same(T, __bf16)) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(B8, a), __builtin_bit_cast(B8, b), c, 0, 0, 0);
    } else {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(H8, a), __builtin_bit_cast(H8, b), c, 0, 0, 0);
    }
}

// One operand's way from memory to LDS: kRows rows of 128 bytes of k, a tile of them on its way in registers.  Of rows past the matrix any others are
// read in their place (their results are dropped); k past the end is 0 on both sides.
template <class T, int kRows, int kThreads, bool kTurn, bool kFar, int kLine>
struct Stage {
    static constexpr int E = 16 / sizeof(T), kDepth = 8 * E;
    static constexpr int kPieces = kTurn ? kRows / kLine * 8 : kRows * 8, kCount = kPieces / kThreads;  // turned: kLine rows by a chunk
    const T* at[kCount];
    uint32_t to[kCount][kTurn ? kLine : 1];  // chunks of LDS
    Chunk held[kTurn ? 1 : kCount];
    static constexpr int kWords = kLine * (int)sizeof(T) / 4;
    using Line = Vec<uint32_t, kWords>;
    Line lines[kTurn ? kCount : 1][kTurn ? E : 1];

    static __device__ __forceinline__ unsigned piece(int n) { return threadIdx.x % kThreads + n * kThreads; }
    static_assert(kPieces % kThreads == 0, "every thread has as much");
    static __device__ __forceinline__ unsigned row(int n) { return kTurn ? piece(n) % (kRows / kLine) * kLine : piece(n) / 8; }
    static __device__ __forceinline__ unsigned chunk(int n) { return kTurn ? piece(n) / (kRows / kLine) : piece(n) % 8; }

    // Turned, kLine rows are read at once: the matrix' last ones instead of any that pass the end, where it has as many.  Those of them that lie before the tile go to its
    // last row, which is past the end then.
    static __device__ __forceinline__ bool inside(int64_t rows) { return !kTurn || rows >= kLine; }
    __device__ __forceinline__ void start(const void* base, int64_t ld, int64_t row0, int64_t rows, int64_t k0) {
#pragma unroll
        for (int n = 0; n < kCount; ++n) {
            const int64_t k = k0 + chunk(n) * E, most = rows - row0;
            if constexpr (kTurn) {
                const int i = inside(rows) && row(n) + kLine > most ? (int)most - kLine : (int)row(n);
                at[n] = static_cast<const T*>(base) + k * ld + row0 + i;
#pragma unroll
                for (int r = 0; r < kLine; ++r) to[n][r] = place<kFar>(i + r < 0 ? kRows - 1 : i + r, chunk(n));
            } else {
                at[n] = static_cast<const T*>(base) + (row0 + (row(n) < most ? row(n) : most - 1)) * ld + k;
                to[n][0] = place<kFar>(row(n), chunk(n));
            }
        }
    }
    // The kDepth of k at hand, all of them in the matrix.
    __device__ __forceinline__ void load_whole(int64_t ld) {
#pragma unroll
        for (int n = 0; n < kCount; ++n) {
            if constexpr (kTurn) {
#pragma unroll
                for (int q = 0; q < E; ++q) lines[n][q] = __builtin_bit_cast(Line, (load<T, kLine>(at[n] + q * ld)));
            } else {
                held[n] = __builtin_bit_cast(Chunk, (load<T, E>(at[n])));
            }
        }
    }
    // The same where `remain` of k are left, and (turned) fewer than kLine rows may be.
    __device__ __forceinline__ void load_some(int64_t ld, int64_t remain, int64_t row0, int64_t rows) {
#pragma unroll
        for (int n = 0; n < kCount; ++n) {
            const int64_t k = remain - chunk(n) * E, most = inside(rows) ? kLine : rows - row0 - row(n);
            if constexpr (kTurn) {
#pragma unroll
                for (int q = 0; q < E; ++q) lines[n][q] = __builtin_bit_cast(Line, (load_own<T, kLine>(at[n] + q * ld, q < k ? most : 0)));
            } else {
                held[n] = __builtin_bit_cast(Chunk, (load_own<T, E>(at[n], k)));
            }
        }
    }
    __device__ __forceinline__ void advance(int64_t ld) {
#pragma unroll
        for (int n = 0; n < kCount; ++n) at[n] += kDepth * (kTurn ? ld : 1);
    }
    __device__ __forceinline__ void to_lds(Chunk* room) const {
#pragma unroll
        for (int n = 0; n < kCount; ++n) {
            if constexpr (kTurn) {
#pragma unroll
                for (int r = 0; r < kLine; ++r) {
                    Chunk line;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        if constexpr (sizeof(T) == 4) line[w] = lines[n][w][r];
                        else line[w] = __builtin_amdgcn_perm(lines[n][(2 * w + 1) % E][r / 2], lines[n][2 * w % E][r / 2], r % 2 ? 0x07060302u : 0x05040100u);
                    }
                    room[to[n][r]] = line;
                }
            } else {
                room[to[n][0]] = held[n];
            }
        }
    }
};

// Both operands' way.  Where both are turned a half of the workgroup takes one each: a thread has eight rows of one of them and not four of both, 16 bytes
// of a line and not 8, in half as many requests (dW of 4096 tokens, 4096 -> 9216 bf16: 370 -> 343 us).
template <class T, int kI, int kJ, int kThreads, bool kTurnA, bool kTurnB, bool kFar>
struct Operands {
    using A = Stage<T, kI, kThreads, kTurnA, kFar, kI * 8 / kThreads>;
    using B = Stage<T, kJ, kThreads, kTurnB, kFar, kJ * 8 / kThreads>;
    A a;
    B b;
    __device__ __forceinline__ bool inside(const Product& p) const { return A::inside(p.rows) && B::inside(p.columns); }
    __device__ __forceinline__ void start(const Product& p, int64_t i0, int64_t j0, int64_t k0) {
        a.start(p.a, p.lda, i0, p.rows, k0);
        b.start(p.b, p.ldb, j0, p.columns, k0);
    }
    __device__ __forceinline__ void load_whole(const Product& p) {
        a.load_whole(p.lda);
        b.load_whole(p.ldb);
    }
    __device__ __forceinline__ void load_some(const Product& p, int64_t remain, int64_t i0, int64_t j0) {
        a.load_some(p.lda, remain, i0, p.rows);
        b.load_some(p.ldb, remain, j0, p.columns);
    }
    __device__ __forceinline__ void advance(const Product& p) {
        a.advance(p.lda);
        b.advance(p.ldb);
    }
    __device__ __forceinline__ void to_lds(Chunk* room) const {
        a.to_lds(room);
        b.to_lds(room + kI * 8);
    }
    // One of the two steps in which a tile is exchanged.
    __device__ __forceinline__ void exchange(unsigned step, Chunk* room, const Product& p, bool more) {
        if (step == 0) {
            a.to_lds(room);
            if (more) a.advance(p.lda);
            a.load_whole(p.lda);
        } else {
            b.to_lds(room + kI * 8);
            if (more) b.advance(p.ldb);
            b.load_whole(p.ldb);
        }
    }
};
template <class T, int kSide, int kThreads>
struct Halves {
    using S = Stage<T, kSide, kThreads / 2, true, true, kSide * 16 / kThreads>;
    S s;
    int64_t ld;
    __device__ __forceinline__ static bool second() { return __builtin_amdgcn_readfirstlane(threadIdx.x / (kThreads / 2)); }
    __device__ __forceinline__ bool inside(const Product& p) const { return S::inside(p.rows) && S::inside(p.columns); }
    __device__ __forceinline__ void start(const Product& p, int64_t i0, int64_t j0, int64_t k0) {
        ld = second() ? p.ldb : p.lda;
        s.start(second() ? p.b : p.a, ld, second() ? j0 : i0, second() ? p.columns : p.rows, k0);
    }
    __device__ __forceinline__ void load_whole(const Product&) { s.load_whole(ld); }
    __device__ __forceinline__ void load_some(const Product& p, int64_t remain, int64_t i0, int64_t j0) {
        s.load_some(ld, remain, second() ? j0 : i0, second() ? p.columns : p.rows);
    }
    __device__ __forceinline__ void advance(const Product&) { s.advance(ld); }
    __device__ __forceinline__ void to_lds(Chunk* room) const { s.to_lds(room + (second() ? kSide * 8 : 0)); }
    __device__ __forceinline__ void exchange(unsigned step, Chunk* room, const Product&, bool more) {
        if (step != 0) return;
        s.to_lds(room + (second() ? kSide * 8 : 0));
        if (more) s.advance(ld);
        s.load_whole(ld);
    }
};

// Neighbouring workgroups run on different dies, each with a cache of its own: a die gets neighbouring tiles, eight rows of tiles at a time.
__device__ __forceinline__ unsigned on_dies(unsigned id, unsigned all) {
    const unsigned die = id % 8, each = all / 8, more = all % 8;
    return die * each + (die < more ? die : more) + id / 8;
}
__device__ __forceinline__ void tile_of(unsigned at, unsigned tiles_i, unsigned tiles_j, unsigned* ti, unsigned* tj) {
    const unsigned group = at / (8 * tiles_j), first = group * 8, high = tiles_i - first < 8 ? tiles_i - first : 8;
    at -= first * tiles_j;
    *ti = first + at % high;
    *tj = at / high;
}

// A barrier for LDS alone: __syncthreads would also wait for the loads from memory that are on their way for the tile after next.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// 16 or 4 bytes a lane from memory, `at` bytes behind `from`, into LDS from `to` on, lane after lane; `from` and `to` are the same for the whole wave.  Nothing waits for
// it but arrived_barrier.  (As a buffer's load: after the flat form the compiler lets every product wait for all operands that are being read; 512 tokens of 4096 -> 4096 28.1 -> 29.7 us.)
template <int kGrain>
__device__ __forceinline__ void to_lds_directly(const void* from, uint32_t at, uint32_t* to) {
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(from), 0, -1, 0x00020000);
    if constexpr (kGrain == 16) __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)to, 16, at, 0, 0, 0);
    else __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)to, 4, at, 0, 0, 0);
}
// All but the last kLater requests of the wave have arrived, and all waves are here.
template <int kLater>
__device__ __forceinline__ void arrived_barrier() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLater) : "memory");
}

// An operand's way straight into LDS.  kTurn: a tile is kDepth lines of its kSide numbers, as they lie in memory; sixteen lanes exchange 16-bit numbers as they read them, and
// fp32 is read number by number.  (Turned in registers, 4096 tokens, 4096 -> 9216 bf16: dX 278 us, dW 310; so 259 and 277.  1024 of 4096 -> 4096 fp32, dW 281 and 257.)
template <class T, int kSide, int kThreads, bool kTurn, bool kFar, int kGrain>
struct Direct {
    static constexpr unsigned E = 16 / sizeof(T), kLines = 128 / sizeof(T), kOf = kSide * 128 / kGrain / kThreads, kGrains = 16 / kGrain, kItems = kGrain / sizeof(T), kChunks = kTurn ? kSide / E : 8;
    // Lines: the chunks of a line are permuted so that what a wave reads at once (16 bits: 64 bytes of four lines, fp32: 128 of two) lies in different banks.
    static __device__ __forceinline__ unsigned turned(unsigned k) { return sizeof(T) == 4 ? (k & 4) << 1 : kSide == 64 ? (k & 2) << 1 : (k & 3) << 2; }
    const T* from;  // the same for the whole wave
    int64_t step;
    uint32_t at[kOf];
    __device__ __forceinline__ void start(const void* base, int64_t ld, int64_t first, int64_t most, int64_t k0) {
        most -= first;
        from = static_cast<const T*>(base) + (kTurn ? k0 * ld + first : first * ld + k0);
        step = kTurn ? kLines * ld : kLines;
#pragma unroll
        for (unsigned n = 0; n < kOf; ++n) {  // a wave fills 64 neighbouring slots at a time; the lane asks for what has its place in its slot (the permutations are their own inverse)
            const unsigned grain = threadIdx.x + n * kThreads, slot = grain / kGrains, line = slot / kChunks, c = kTurn ? slot % kChunks ^ turned(line) : place<kFar>(line, slot % 8) % 8;
            const unsigned item = c * E + grain % kGrains * kItems;
            if (kTurn) at[n] = (line * (uint32_t)ld + (uint32_t)(item < most ? item : most - kItems)) * sizeof(T);
            else at[n] = ((uint32_t)(line < most ? line : most - 1) * (uint32_t)ld + item) * sizeof(T);
        }
    }
    __device__ __forceinline__ void request(Chunk* to, bool more) {  // a tile, and on to the next
#pragma unroll
        for (unsigned n = 0; n < kOf; ++n) to_lds_directly<kGrain>(from, at[n], reinterpret_cast<uint32_t*>(to) + n * kThreads * (kGrain / 4));
        from += more ? step : 0;
    }
    // As multiply takes them: sixteen bytes of k, from `step` * 32 on, of the 32 numbers from `first` on.
    static __device__ __forceinline__ Chunk across(const Chunk* tile, unsigned first, unsigned step) {
        const unsigned lane = threadIdx.x & 63;
        if constexpr (sizeof(T) == 4) {
            const unsigned k = lane >> 5 << 2, c = first / E + (lane >> 2 & 7);
            const float* p = reinterpret_cast<const float*>(tile + k * kChunks + (c ^ turned(k))) + (lane & 3) + step * 8 * kSide;
            return __builtin_bit_cast(Chunk, F4{p[0], p[kSide], p[2 * kSide], p[3 * kSide]});
        } else {  // sixteen lanes exchange sixteen numbers of four lines
            typedef short S4 __attribute__((ext_vector_type(4)));
            const unsigned k = (lane >> 5 << 3) + (lane >> 2 & 3), c = first / E + (lane >> 3 & 2) + (lane >> 1 & 1);
            const auto* p = (const __attribute__((address_space(3))) S4*)(tile + k * kChunks + (c ^ turned(k))) + (lane & 1) + step * 4 * kSide;
            auto* q = const_cast<__attribute__((address_space(3))) S4*>(p);
            const S4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16(q), high = __builtin_amdgcn_ds_read_tr16_b64_v4i16(q + kSide);
            return __builtin_bit_cast(Chunk, __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// kStages: 0: two tiles in LDS, and the way there through registers.  Else so many tiles in LDS, all but one of them on their way straight from memory: no registers, no stores
// to LDS among the reads of it, and more than one tile under way where a compute unit has a single workgroup, which else waits for memory at each step.
template <class T, int kI, int kJ, int kWavesI, int kWavesJ, bool kTurnA, bool kTurnB, int kStages = 0, int kGrainA = 16, int kGrainB = 16>
__global__ __launch_bounds__(64 * kWavesI * kWavesJ) void product_kernel(Product p) {
    constexpr int kThreads = 64 * kWavesI * kWavesJ, kWideI = kI / kWavesI, kWideJ = kJ / kWavesJ, kTilesI = kWideI / 32, kTilesJ = kWideJ / 32;
    constexpr int kPitch = kWideJ + 4;
    constexpr int kDepth = 128 / sizeof(T);
    constexpr bool kHalves = kTurnA && kTurnB && kI == kJ;
    constexpr bool kFar = kHalves || kI == 256;  // eight rows a thread want it; elsewhere it costs registers (dX of 512 tokens 39 -> 45 us), or none that are missed (4096: 305 -> 290)
    using Way = std::conditional_t<kHalves, Halves<T, kI, kThreads>, Operands<T, kI, kJ, kThreads, kTurnA, kTurnB, kFar>>;
    __shared__ Chunk room[kStages ? kStages : 2][(kI + kJ) * 8];
    static_assert(sizeof(room) >= sizeof(float) * kWavesI * kWavesJ * 32 * kPitch, "");
    const unsigned lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wave_i = wave / kWavesJ, wave_j = wave % kWavesJ;
    const bool cut = p.parts > 1;
    const unsigned piece = blockIdx.x;
    unsigned ti, tj;
    tile_of(cut ? piece / p.parts : on_dies(piece, p.tiles_i * p.tiles_j), p.tiles_i, p.tiles_j, &ti, &tj);
    const int64_t i0 = (int64_t)ti * kI, j0 = (int64_t)tj * kJ, k0 = cut ? piece % p.parts * p.depth_of_part : 0;
    int64_t remain = cut && p.depth - k0 > p.depth_of_part ? p.depth_of_part : p.depth - k0;
    Way way;
    if (!kStages) way.start(p, i0, j0, k0);
    F16 sums[kTilesI][kTilesJ];
#pragma unroll
    for (int x = 0; x < kTilesI; ++x)
#pragma unroll
        for (int y = 0; y < kTilesJ; ++y) sums[x][y] = 0.f;
    // chunk 2 . step + (lane >> 5) of row lane & 31 of an even or odd 32 rows: the permutation is an exclusive or
    const unsigned at_lane = place<kFar>(lane & 31, lane >> 5);
    Chunk x[2][kTilesI], y[2][kTilesJ];
    const auto rows_a = [&](const Chunk* tile, unsigned step, Chunk(&u)[kTilesI]) {
#pragma unroll
        for (int k = 0; k < kTilesI; ++k) u[k] = tile[(wave_i * kWideI + k * 32) * 8 + (at_lane ^ 2 * step ^ (kFar ? (wave_i * kTilesI + k) % 2 * 4 : 0))];
    };
    const auto rows_b = [&](const Chunk* tile, unsigned step, Chunk(&v)[kTilesJ]) {
#pragma unroll
        for (int k = 0; k < kTilesJ; ++k) v[k] = tile[(kI + wave_j * kWideJ + k * 32) * 8 + (at_lane ^ 2 * step ^ (kFar ? (wave_j * kTilesJ + k) % 2 * 4 : 0))];
    };
    const auto operands = [&](const Chunk* tile, unsigned step, Chunk(&u)[kTilesI], Chunk(&v)[kTilesJ]) {
        rows_a(tile, step, u);
        rows_b(tile, step, v);
    };
    const auto products = [&](const Chunk(&u)[kTilesI], const Chunk(&v)[kTilesJ]) {
#pragma unroll
        for (int i = 0; i < kTilesI; ++i)
#pragma unroll
            for (int j = 0; j < kTilesJ; ++j) sums[i][j] = multiply<T>(v[j], u[i], sums[i][j]);
    };
    // Whole tiles.  While tile k is multiplied out of one half of LDS, tile k + 1 goes from registers into the other half and tile k + 2 is on its way from
    // memory; past the last one the last is read again, for nobody.  (Two or four tiles on their way gained nothing.)
    unsigned turn = 0;
    const int64_t whole = (kStages || way.inside(p)) && remain > 0 ? remain / kDepth : 0;
    if constexpr (kStages > 0) {
        using DirectA = Direct<T, kI, kThreads, kTurnA, kFar, kGrainA>;
        using DirectB = Direct<T, kJ, kThreads, kTurnB, kFar, kGrainB>;
        constexpr int kOf = DirectA::kOf + DirectB::kOf;
        DirectA a;
        DirectB b;
        a.start(p.a, p.lda, i0, p.rows, k0);
        b.start(p.b, p.ldb, j0, p.columns, k0);
        const unsigned first = __builtin_amdgcn_readfirstlane(threadIdx.x / 64) * 4;  // a wave's first chunk, for each byte of its grains
        const auto request = [&](Chunk* to, bool more) {
            a.request(to + first * kGrainA, more);
            b.request(to + kI * 8 + first * kGrainB, more);
        };
        const auto straight = [&](const Chunk* tile, unsigned step, Chunk(&u)[kTilesI], Chunk(&v)[kTilesJ]) {
            if constexpr (!kTurnA) rows_a(tile, step, u);
            if constexpr (!kTurnB) rows_b(tile, step, v);
            if constexpr (kTurnA)
#pragma unroll
                for (int k = 0; k < kTilesI; ++k) u[k] = DirectA::across(tile, wave_i * kWideI + k * 32, step);
            if constexpr (kTurnB)
#pragma unroll
                for (int k = 0; k < kTilesJ; ++k) v[k] = DirectB::across(tile + kI * 8, wave_j * kWideJ + k * 32, step);
        };
        if (whole) {  // past the last tile the last is read again, for nobody
            for (unsigned stage = 0; stage + 1 < kStages; ++stage) request(room[stage], stage + 1 < whole);
            arrived_barrier<kOf*(kStages - 2)>();
            straight(room[0], 0, x[0], y[0]);
            unsigned next = kStages - 1;  // the stage to fill: all waves are past the barrier behind their reads of it
            // The tile that is filled is another than those that are read: without that said, the compiler waits for it to arrive before it reads across (dX of 1024 tokens of
            // 4096 -> 4096 bf16 65 us for 48).  With two stages it is the following one, which is read behind the wait for it.
            const auto multiplied = [&](Chunk* __restrict fill, const Chunk* __restrict tile, const Chunk* __restrict following, bool more) __attribute__((always_inline)) {
#pragma unroll
                for (unsigned step = 0; step < 4; ++step) {
                    if (step < 3) {
                        straight(tile, step + 1, x[(step + 1) & 1], y[(step + 1) & 1]);
                    } else if (kStages > 2) {
                        arrived_barrier<kOf*(kStages - 2)>();
                        straight(following, 0, x[0], y[0]);
                    } else {
                        break;
                    }
                    if (step == 0) request(fill, more);
                    __builtin_amdgcn_sched_barrier(0);
                    products(x[step & 1], y[step & 1]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            for (int64_t k = 0; k < whole; ++k) {
                const unsigned following = turn + 1 == kStages ? 0 : turn + 1;
                multiplied(room[next], room[turn], kStages > 2 ? room[following] : nullptr, k + kStages < whole);
                if (kStages == 2) {
                    arrived_barrier<0>();
                    straight(room[following], 0, x[0], y[0]);
                    __builtin_amdgcn_sched_barrier(0);
                    products(x[1], y[1]);
                    __builtin_amdgcn_sched_barrier(0);
                }
                next = turn;
                turn = following;
            }
            arrived_barrier<0>();
            turn = 0;
            remain -= whole * kDepth;
        }
        way.start(p, i0, j0, k0 + whole * kDepth);
    } else if (whole) {
        way.load_whole(p);
        way.to_lds(room[0]);
        if (whole > 1) way.advance(p);
        way.load_whole(p);
        lds_barrier();
        operands(room[0], 0, x[0], y[0]);
        for (int64_t k = 0; k < whole; ++k, turn ^= 1) {
            const bool more = k + 2 < whole;
#pragma unroll
            for (unsigned step = 0; step < 4; ++step) {
                if (step < 3) {
                    operands(room[turn], step + 1, x[(step + 1) & 1], y[(step + 1) & 1]);
                } else {  // every operand of this tile is in registers: the next tile's first ones come while the last products run
                    lds_barrier();
                    operands(room[turn ^ 1], 0, x[0], y[0]);
                }
                if (step < 2) way.exchange(step, room[turn ^ 1], p, more);
                __builtin_amdgcn_sched_barrier(0);  // the compiler would move requests down to where their answers are needed
                products(x[step & 1], y[step & 1]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        lds_barrier();
        remain -= whole * kDepth;
        way.advance(p);
    }
    // What is left: a part of a tile, or all of them where a turned operand has fewer rows than are read at once.
    while (remain > 0) {
        way.load_some(p, remain, i0, j0);
        way.to_lds(room[turn]);
        lds_barrier();
#pragma unroll
        for (unsigned step = 0; step < 4; ++step) {
            operands(room[turn], step, x[0], y[0]);
            products(x[0], y[0]);
        }
        remain -= kDepth;
        way.advance(p);
        turn ^= 1;
    }
    __syncthreads();
    // 32 rows of each wave at a time through LDS, so that neighbouring lanes have neighbouring numbers of a row.  Nothing is multiplied meanwhile: what the epilogue computes for
    // a number counts (with two roundings in full and a branch for each number, 4096 tokens, 4096 -> 9216 with gelu_tanh and Z kept took 332 us; now 308).
    float* own = reinterpret_cast<float*>(room) + wave * 32 * kPitch;
    constexpr int kAbreast = kWideJ / 4;
    const int64_t j = j0 + wave_j * kWideJ + lane % kAbreast * 4;
    const Vec<float, 4> bias = cut ? Vec<float, 4>(0.f) : bias_along(p.to, j, p.columns - j);
#pragma unroll
    for (int x = 0; x < kTilesI; ++x) {
        if (x) __syncthreads();
#pragma unroll
        for (int y = 0; y < kTilesJ; ++y)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<Vec<float, 4>*>(own + (lane & 31) * kPitch + y * 32 + q * 8 + (lane >> 5) * 4) =
                    Vec<float, 4>{sums[x][y][4 * q], sums[x][y][4 * q + 1], sums[x][y][4 * q + 2], sums[x][y][4 * q + 3]};
        __syncthreads();
#pragma unroll 1
        for (int row = lane / kAbreast; row < 32; row += 64 / kAbreast) {
            const int64_t i = i0 + wave_i * kWideI + x * 32 + row;
            const Vec<float, 4> z = *reinterpret_cast<const Vec<float, 4>*>(own + row * kPitch + lane % kAbreast * 4);
            if (cut) {
                store<float, 4>(p.part + ((int64_t)piece * kI + (i - i0)) * kJ + (j - j0), z);
                continue;
            }
            if (i < p.rows && j < p.columns) finish<T>(p.to, i, j, z, bias, p.columns - j);
        }
    }
}

// The parts added up in their order, then the epilogue: four neighbouring numbers of C a thread.  Workgroup (b, t): 1024 numbers of tile t.
template <class T, int kI, int kJ>
__global__ __launch_bounds__(256) void parts_kernel(Product p) {
    unsigned ti, tj;
    tile_of(blockIdx.y, p.tiles_i, p.tiles_j, &ti, &tj);
    const unsigned at = blockIdx.x * 1024 + threadIdx.x * 4;
    const int64_t i = (int64_t)ti * kI + at / kJ, j = (int64_t)tj * kJ + at % kJ;
    if (i >= p.rows || j >= p.columns) return;
    const float* from = p.part + (int64_t)blockIdx.y * p.parts * (kI * kJ) + at;
    Vec<float, 4> z = 0.f;
#pragma unroll 8
    for (uint32_t k = 0; k < p.parts; ++k) z += load<float, 4>(from + (int64_t)k * (kI * kJ));
    finish<T>(p.to, i, j, z, bias_along(p.to, j, p.columns - j), p.columns - j);
}

// How a product is cut: tiles of a size, the contraction in parts; or its first rows or columns so that their tiles fill the chip some whole times, and the rest by itself.
struct Plan {
    int side = 0;
    int64_t parts = 1;
    int64_t first = 0;  // rows or columns of C before the rest; 0: there is none
    bool rows = false;
    double time = 0;  // microseconds, estimated
};
constexpr int64_t kComputeUnits = 256;

template <class T>
Plan plan_of(int64_t rows, int64_t columns, int64_t depth, bool may_cut) {
    constexpr int64_t kDepth = 128 / sizeof(T);
    // Per k, in nanoseconds: what `at_once` workgroups on a compute unit take at least (a step's way through LDS and its barrier, whatever it multiplies), and what each
    // adds once they share the matrix cores.  Measured with operands that go straight into LDS, where turned ones cost the same: 64 - 4096 tokens of 4096 -> 4096 and 9216 (16
    // bits), 256 - 1024 of 2048 and 4096 (fp32), and their gradients.  Through registers all of it is slower, and turned ones by more; fp32 by numbers up to 81.
    struct Size {
        int side, at_once;
        double alone, each;
    };
    constexpr Size wide[3] = {{256, 1, 21.5, 27.0}, {128, 2, 8.3, 7.8}, {64, 3, 2.8, 2.9}}, exact[2] = {{128, 2, 61.0, 62.0}, {64, 3, 18.0, 15.6}};
    const int64_t steps = (depth + kDepth - 1) / kDepth;
    const auto rounds = [&](const Size& size, int64_t workgroups, double k) {
        const int64_t most = (workgroups + kComputeUnits - 1) / kComputeUnits;
        const bool few = workgroups <= kComputeUnits / 2;
        return k * 1e-3 * std::max((double)((most + size.at_once - 1) / size.at_once) * size.alone, most * (size.at_once == 1 && few ? size.alone : size.each));
    };
    Plan best;
    const auto consider = [&](const Plan& p) {
        if (!best.side || p.time < best.time) best = p;
    };
    const auto of = [&](const Size& size) {
        const int64_t tiles_i = (rows + size.side - 1) / size.side, tiles_j = (columns + size.side - 1) / size.side, tiles = tiles_i * tiles_j, room = kComputeUnits * size.at_once;
        consider({size.side, 1, 0, false, 6.0 + rounds(size, tiles, (double)depth)});
        for (int64_t parts = 2; parts <= 16 && parts * 4 <= steps && parts * tiles <= room; ++parts)  // written and read again, at 5 TB/s
            consider({size.side, parts, 0, false,
                      8.0 + rounds(size, tiles * parts, (double)((steps + parts - 1) / parts * kDepth)) + (double)(tiles * parts) * size.side * size.side * 8 / 5e6});
        // Whole rounds by themselves and what is left with a plan of its own: a round is all that run at once, or (fp32, where each takes the matrix cores for as long as if it were
        // alone) one workgroup on each compute unit: 1000 tokens, 2050 -> 2050 118 -> 100 us, dX 109 -> 95; of 16 bits 2100 tokens, 2048 -> 2048, dX 35 -> 40.
        const int64_t round = sizeof(T) == 4 ? kComputeUnits : room;
        if (!may_cut || tiles <= round || tiles > 16 * room) return;
        for (const bool by_rows : {false, true}) {
            const int64_t across = by_rows ? tiles_j : tiles_i, lines = tiles / round * round / across;  // whole lines of tiles
            if (lines < 1 || lines >= (by_rows ? tiles_i : tiles_j)) continue;
            const int64_t first = lines * size.side;
            const Plan rest = plan_of<T>(by_rows ? rows - first : rows, by_rows ? columns : columns - first, depth, false);
            consider({size.side, 1, first, by_rows, 10.0 + rounds(size, lines * across, (double)depth) + rest.time});
        }
    };
    if constexpr (sizeof(T) == 2) {
        for (const Size& size : wide) of(size);
    } else {
        for (const Size& size : exact) of(size);
    }
    return best;
}

// Steps of the contraction to a part, and parts: none without a step.
template <class T>
void parts_of(int64_t depth, int64_t parts, int64_t* depth_of_part, uint32_t* many) {
    constexpr int64_t kDepth = 128 / sizeof(T);
    const int64_t steps = (depth + kDepth - 1) / kDepth, of_part = std::max<int64_t>(1, (steps + parts - 1) / parts);
    *many = (uint32_t)std::max<int64_t>(1, (steps + of_part - 1) / of_part);
    *depth_of_part = of_part * kDepth;
}
template <class T>
size_t parts_bytes(const Plan& plan, int64_t rows, int64_t columns, int64_t depth) {
    int64_t of_part;
    uint32_t parts;
    parts_of<T>(depth, plan.parts, &of_part, &parts);
    return parts > 1 ? (size_t)((rows + plan.side - 1) / plan.side * ((columns + plan.side - 1) / plan.side)) * parts * plan.side * plan.side * 4 : 0;
}
// The plan of a product, that of its rest where there is one, and the bytes of their parts (they follow one another).
struct Course {
    Plan head, rest;
    size_t bytes = 0;
};
template <class T>
Course course_of(int64_t rows, int64_t columns, int64_t depth) {
    Course c;
    c.head = plan_of<T>(rows, columns, depth, true);
    if (c.head.first) {
        (c.head.rows ? rows : columns) -= c.head.first;
        c.rest = plan_of<T>(rows, columns, depth, false);
    }
    c.bytes = parts_bytes<T>(c.head.first ? c.rest : c.head, rows, columns, depth);
    return c;
}

template <class T, int kI, int kJ, int kWavesI, int kWavesJ>
int launch_tiles(Product p, int64_t parts, bool turn_a, bool turn_b, hipStream_t s) {
    p.tiles_i = (uint32_t)((p.rows + kI - 1) / kI), p.tiles_j = (uint32_t)((p.columns + kJ - 1) / kJ);
    parts_of<T>(p.depth, parts, &p.depth_of_part, &p.parts);
    const unsigned tiles = p.tiles_i * p.tiles_j;
    constexpr int kThreads = 64 * kWavesI * kWavesJ;
    // Straight into LDS go whole grains of 16 bytes, and a tile's offsets have 32 bits.  Numbers of fp32 go there by themselves where an operand is turned (1000 tokens, 2050 -> 2050: dX
    // 120 -> 108 us, dW 100 -> 92); where none is, registers do as well (Y 117 -> 118, 657 tokens, 3563 -> 1475 108 -> 95), and pairs of 16 bits are slower (1000 tokens, Y 31, dX 36 -> 65, 67).
    // Rows of numbers in tiles of 128 are slower, too (a tile of 999 tokens in columns, 2048 -> 4608, W by numbers 226 us, by 16 bytes and X by numbers 167).
    const auto fits = [](const void* base, int64_t ld, int64_t across, bool turn, int64_t grain) {
        return (uintptr_t)base % grain == 0 && ld * sizeof(T) % grain == 0 && ld < (INT64_C(1) << 21) && (!turn || across * sizeof(T) % grain == 0);
    };
    const bool chunks_a = fits(p.a, p.lda, p.rows, turn_a, 16), direct = chunks_a && fits(p.b, p.ldb, p.columns, turn_b, 16);
    const bool by_numbers = fits(p.a, p.lda, p.rows, turn_a, 4) && fits(p.b, p.ldb, p.columns, turn_b, 4);
    // One more tile under way where a compute unit has one workgroup (256 tokens of 4096 -> 4096 bf16, 64 x 64: 3 tiles in LDS 20.5 us, 4 17.6, 6 17.9; 1024 tokens, 128 x 128:
    // 2 55, 3 43, 4 43.5); where it has several, their number counts for more (512 tokens: 27.1, 28.3, 33.8; 2048 tokens: 68, 84, 84).
    constexpr int kStages = kI == 64 ? 3 : 2, kMore = kI == 256 ? kStages : kStages + 1;
    const auto launch = [&](auto turned_a, auto turned_b) {
        constexpr bool a = decltype(turned_a)::value, b = decltype(turned_b)::value;
        const bool several = tiles * p.parts > kComputeUnits;
        const auto go = [&](auto stages, auto grain_a, auto grain_b) {
            product_kernel<T, kI, kJ, kWavesI, kWavesJ, a, b, decltype(stages)::value, decltype(grain_a)::value, decltype(grain_b)::value><<<tiles * p.parts, kThreads, 0, s>>>(p);
        };
        using Few = std::integral_constant<int, kStages>;
        using More = std::integral_constant<int, kMore>;
        using Chunks = std::integral_constant<int, 16>;
        using Numbers = std::integral_constant<int, 4>;
        if (direct) return several ? go(Few(), Chunks(), Chunks()) : go(More(), Chunks(), Chunks());
        if constexpr (sizeof(T) == 4 && b && !a)
            if (by_numbers && chunks_a) return several ? go(Few(), Chunks(), Numbers()) : go(More(), Chunks(), Numbers());
        if constexpr (sizeof(T) == 4 && b && (a || kI == 64))
            if (by_numbers) return several ? go(Few(), Numbers(), Numbers()) : go(More(), Numbers(), Numbers());
        go(std::integral_constant<int, 0>(), Chunks(), Chunks());
    };
    if (!turn_b) launch(std::false_type(), std::false_type());
    else if (!turn_a) launch(std::false_type(), std::true_type());
    else launch(std::true_type(), std::true_type());
    if (int e = (int)hipGetLastError()) return e;
    if (p.parts > 1) parts_kernel<T, kI, kJ><<<dim3(kI * kJ / 1024, tiles), 256, 0, s>>>(p);
    return (int)hipGetLastError();
}

template <class T>
int launch_planned(const Product& p, const Plan& plan, bool turn_a, bool turn_b, hipStream_t s) {
    if (plan.side == 64) return launch_tiles<T, 64, 64, 2, 2>(p, plan.parts, turn_a, turn_b, s);
    if (plan.side == 128) return launch_tiles<T, 128, 128, 2, 2>(p, plan.parts, turn_a, turn_b, s);
    if constexpr (sizeof(T) == 2) return launch_tiles<T, 256, 256, 2, 4>(p, plan.parts, turn_a, turn_b, s);
    return (int)hipErrorInvalidValue;
}
int size_of(int32_t type) { return type == CER_TYPE_F32 ? 4 : 2; }

template <class T>
int launch_product(const Product& p, const Course& course, bool turn_a, bool turn_b, hipStream_t s) {
    const Plan& plan = course.head;
    if (!plan.first) return launch_planned<T>(p, plan, turn_a, turn_b, s);
    Product head = p, rest = p;
    const auto past = [](auto* at, int64_t bytes) { return at ? (std::remove_pointer_t<decltype(at)>*)((uintptr_t)at + bytes) : at; };
    const int64_t item = sizeof(T);
    (plan.rows ? head.rows : head.columns) = plan.first;
    (plan.rows ? rest.rows : rest.columns) -= plan.first;
    if (plan.rows) rest.a = past(p.a, plan.first * (turn_a ? 1 : p.lda) * item);
    else rest.b = past(p.b, plan.first * (turn_b ? 1 : p.ldb) * item);
    if (p.to.bias_rows == plan.rows) rest.to.bias = past(p.to.bias, plan.first * size_of(p.to.bias_type));
    rest.to.residual = past(p.to.residual, plan.first * (plan.rows ? p.to.ldr : 1) * item);
    rest.to.pre = past(p.to.pre, plan.first * (plan.rows ? p.to.ldp : 1) * item);
    rest.to.out = past(p.to.out, plan.first * (plan.rows ? p.to.ldo : 1) * item);
    if (int e = launch_planned<T>(head, plan, turn_a, turn_b, s)) return e;
    return launch_planned<T>(rest, course.rest, turn_a, turn_b, s);
}

// ---- few tokens -----------------------------------------------------------------------------------------------------------------
// A decode step reads W once and does little else.  A workgroup takes 16 rows of W and every wave a part of the contraction: its operands come from memory in the
// matrix instruction's own layout, 16 bytes a lane (four lanes have 64 bytes of a row), eight requests of W on their way before
// the first product.  The waves' sums meet in LDS, in their order.
template <class T>
__device__ __forceinline__ F4 multiply16(Chunk a, Chunk b, F4 c) {
    if constexpr (sizeof(T) == 4) {
        const F4 x = __builtin_bit_cast(F4, a), y = __builtin_bit_cast(F4, b);
#pragma unroll
        for (int q = 0; q < 4; ++q) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[q], y[q], c, 0, 0, 0);
        return c;
    } else if constexpr (__is_same(T, __bf16)) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(B8, a), __builtin_bit_cast(B8, b), c, 0, 0, 0);
    } else {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(H8, a), __builtin_bit_cast(H8, b), c, 0, 0, 0);
    }
}
struct FewArgs {
    const void *w, *x;
    int64_t ldw, ldx;
    int64_t tokens, in, out;
    int64_t lines_of_wave;  // of 128 bytes of k
    Epilogue to;
};
template <class T, int kTiles, bool kColumns>
__global__ __launch_bounds__(1024) void few_tokens_kernel(FewArgs a) {
    constexpr int E = 16 / sizeof(T), kLine = 8 * E, kAtOnce = kTiles > 1 ? 2 : 4;
    __shared__ Vec<float, 4> room[16][kTiles][64];
    const unsigned lane = threadIdx.x & 63, wave = threadIdx.x >> 6, of = lane & 15, group = lane >> 4;
    const int64_t row0 = (int64_t)blockIdx.x * 16, row = row0 + of < a.out ? row0 + of : a.out - 1;
    int64_t k = wave * a.lines_of_wave * kLine;
    const int64_t last = k + a.lines_of_wave * kLine < a.in ? k + a.lines_of_wave * kLine : a.in;
    const T* w = static_cast<const T*>(a.w) + row * a.ldw + group * E;
    const T* x[kTiles];
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
        const int64_t t = n * 16 + of < a.tokens ? n * 16 + of : a.tokens - 1;  // others' results are dropped
        x[n] = static_cast<const T*>(a.x) + (kColumns ? t + group * E * a.ldx : t * a.ldx + group * E);
    }
    const auto chunk_of_x = [&](int n, int64_t at, int64_t left) {
        if constexpr (kColumns) {
            Vec<T, E> v;
#pragma unroll
            for (int j = 0; j < E; ++j) {
                v[j] = (T)0.f;
                if (j < left) v[j] = x[n][(at + j) * a.ldx];
            }
            return __builtin_bit_cast(Chunk, v);
        } else {
            return __builtin_bit_cast(Chunk, (load_own<T, E>(x[n] + at, left)));
        }
    };
    F4 sums[kTiles];
#pragma unroll
    for (int n = 0; n < kTiles; ++n) sums[n] = 0.f;
    for (; k + kAtOnce * kLine <= last; k += kAtOnce * kLine) {
        Chunk u[kAtOnce * 2], v[kAtOnce * 2][kTiles];
#pragma unroll
        for (int q = 0; q < kAtOnce * 2; ++q) u[q] = __builtin_bit_cast(Chunk, (load<T, E>(w + k + q * 4 * E)));
#pragma unroll
        for (int q = 0; q < kAtOnce * 2; ++q)
#pragma unroll
            for (int n = 0; n < kTiles; ++n) v[q][n] = chunk_of_x(n, k + q * 4 * E, E);
#pragma unroll
        for (int q = 0; q < kAtOnce * 2; ++q)
#pragma unroll
            for (int n = 0; n < kTiles; ++n) sums[n] = multiply16<T>(u[q], v[q][n], sums[n]);
    }
    for (; k < last; k += kLine)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int64_t left = last - k - (q * 4 + group) * E;
            const Chunk u = __builtin_bit_cast(Chunk, (load_own<T, E>(w + k + q * 4 * E, left)));
#pragma unroll
            for (int n = 0; n < kTiles; ++n) sums[n] = multiply16<T>(u, chunk_of_x(n, k + q * 4 * E, left), sums[n]);
        }
#pragma unroll
    for (int n = 0; n < kTiles; ++n) room[wave][n][lane] = sums[n];
    __syncthreads();
    // lane: token `of` of its tile, features 4 group ..
    const unsigned waves = blockDim.x >> 6;
    if (wave >= kTiles) return;
    const int64_t t = wave * 16 + of, j = row0 + group * 4;
    if (t >= a.tokens || j >= a.out) return;
    F4 z = room[0][wave][lane];
    for (unsigned k = 1; k < waves; ++k) z += room[k][wave][lane];
    if constexpr (kColumns) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (j + q < a.out) finish<T>(a.to, j + q, t, F4(z[q]), F4(0.f), 1);
    } else {
        finish<T>(a.to, t, j, z, bias_along(a.to, j, a.out - j), a.out - j);
    }
}
// Two tiles of 16 tokens only where W is short: there the other kernel's two launches take longer (32 tokens, 640 -> 640 bf16: 6.8 against 11.1 us; 9216 -> 4096 33 against 22).
// Few rows of a long W leave most compute units without a workgroup (one token, 12800 -> 640: 18 us against 10 in parts).
bool few_tokens(int64_t tokens, int64_t in, int64_t out, int64_t item) {
    const bool brief = in * item <= 48 * 128;
    return tokens <= (brief ? 32 : 16) && (brief || out >= 2048);
}
template <class T, bool kColumns>
int launch_few_tokens(FewArgs a, hipStream_t s) {
    constexpr int64_t kLine = 128 / sizeof(T);
    const int64_t lines = (a.in + kLine - 1) / kLine;
    const int64_t waves = std::min<int64_t>(16, std::max<int64_t>(a.tokens > 16 ? 2 : 1, lines));
    a.lines_of_wave = (lines + waves - 1) / waves;
    const unsigned grid = (unsigned)((a.out + 15) / 16), threads = (unsigned)waves * 64;
    if (a.tokens <= 16) few_tokens_kernel<T, 1, kColumns><<<grid, threads, 0, s>>>(a);
    else few_tokens_kernel<T, 2, kColumns><<<grid, threads, 0, s>>>(a);
    return (int)hipGetLastError();
}

// ---- the gradient of z, and of the bias -----------------------------------------------------------------------------------------
struct SlopeArgs {
    const void *dy, *pre;  // pre == nullptr: dz is dy, only its sums are wanted
    void* dz;
    int64_t lddy, ldp, lddz;
    int64_t tokens, out;
    int32_t activation;
    float* sums;  // rows: [parts][out]; columns: [out]
    int64_t tokens_of_part;
};
// A slope of 0 leaves nothing of any dy.
__device__ __forceinline__ float times_slope(float dy, float z, int kind) {
    const float v = slope(z, kind);
    return v == 0.f ? 0.f : dy * v;
}

// Rows: kLanes lanes of V features by 256 / kLanes tokens at a time of the workgroup's part.
template <class T, int kLanes>
__global__ __launch_bounds__(256) void slope_rows_kernel(SlopeArgs a) {
    constexpr int V = 16 / sizeof(T), kRows = 256 / kLanes;
    __shared__ Vec<float, V> room[kRows][kLanes];
    const unsigned lane = threadIdx.x % kLanes, row = threadIdx.x / kLanes;
    const int64_t e = ((int64_t)blockIdx.x * kLanes + lane) * V, left = a.out - e;
    const int64_t first = blockIdx.y * a.tokens_of_part, last = first + a.tokens_of_part < a.tokens ? first + a.tokens_of_part : a.tokens;
    Vec<float, V> sums = 0.f;
    if (left > 0)
#pragma unroll 2
        for (int64_t t = first + row; t < last; t += kRows) {
            Vec<float, V> dz = load_some<T, V>(static_cast<const T*>(a.dy) + t * a.lddy + e, left);
            if (a.pre) {
                const Vec<float, V> z = load_some<T, V>(static_cast<const T*>(a.pre) + t * a.ldp + e, left);
#pragma unroll
                for (int j = 0; j < V; ++j) dz[j] = times_slope(dz[j], z[j], a.activation);
                if (a.dz) store_some<T, V>(static_cast<T*>(a.dz) + t * a.lddz + e, dz, left);
            }
            sums += dz;
        }
    if (!a.sums) return;
    room[row][lane] = sums;
    __syncthreads();
    for (unsigned k = kRows / 2; k; k /= 2) {
        if (row < k) room[row][lane] += room[row + k][lane];
        __syncthreads();
    }
    if (row == 0 && left > 0) store_some<float, V>(a.sums + blockIdx.y * a.out + e, room[0][lane], left);
}
// Columns: a workgroup for a feature.
__global__ __launch_bounds__(256) void slope_columns_kernel(SlopeArgs a) {
    __shared__ float room[16];
    const int64_t o = blockIdx.x;
    const float *dy = static_cast<const float*>(a.dy) + o * a.lddy, *pre = static_cast<const float*>(a.pre) + (a.pre ? o * a.ldp : 0);
    float* out = static_cast<float*>(a.dz) + (a.dz ? o * a.lddz : 0);
    float sum = 0.f;
#pragma unroll 4
    for (int64_t t = threadIdx.x; t < a.tokens; t += 256) {
        float dz = dy[t];
        if (a.pre) {
            dz = times_slope(dz, pre[t], a.activation);
            if (a.dz) out[t] = dz;
        }
        sum += dz;
    }
    if (!a.sums) return;
    sum = block_total(sum, room);
    if (threadIdx.x == 0) a.sums[o] = sum;
}
// The parts added up in their order: 16 lanes of four features by 64 rows of parts.
__global__ __launch_bounds__(1024) void bias_totals_kernel(const float* part, uint32_t parts, int64_t n, float* out) {
    __shared__ Vec<float, 4> room[64][17];
    const unsigned lane = threadIdx.x & 15, row = threadIdx.x >> 4;
    const int64_t i = (int64_t)blockIdx.x * 64 + lane * 4;
    Vec<float, 4> all = 0.f;
    if (i < n)
        for (uint32_t p = row; p < parts; p += 64) all += load_some<float, 4>(part + p * n + i, n - i);
    room[row][lane] = all;
    __syncthreads();
    for (unsigned k = 32; k; k /= 2) {
        if (row < k) room[row][lane] += room[row + k][lane];
        __syncthreads();
    }
    if (row == 0 && i < n) store_some<float, 4>(out + i, room[0][lane], n - i);
}

template <class T>
Course linear_course(const LinearCall& c) {
    const bool columns = c.x.order == CER_ORDER_COLUMNS;
    return course_of<T>(columns ? c.out : c.tokens, columns ? c.tokens : c.out, c.in);
}
template <class T>
int64_t linear_bytes(const LinearCall& c) {
    return !c.tokens || few_tokens(c.tokens, c.in, c.out, sizeof(T)) ? 0 : (int64_t)Room::rounded(linear_course<T>(c).bytes);
}
template <class T>
int linear_of(const LinearCall& c, hipStream_t s) {
    const bool columns = c.x.order == CER_ORDER_COLUMNS;
    const Epilogue to{c.bias, c.bias_type, columns, c.activation, c.residual.data, c.pre.data, c.y.data, c.residual.ld, c.pre.ld, c.y.ld};
    if (few_tokens(c.tokens, c.in, c.out, sizeof(T))) {
        const FewArgs a{c.w, c.x.data, c.ldw, c.x.ld, c.tokens, c.in, c.out, 0, to};
        if constexpr (sizeof(T) == 4)
            if (columns) return launch_few_tokens<float, true>(a, s);
        return launch_few_tokens<T, false>(a, s);
    }
    Product p{};
    p.a = columns ? c.w : c.x.data, p.lda = columns ? c.ldw : c.x.ld;
    p.b = columns ? c.x.data : c.w, p.ldb = columns ? c.x.ld : c.ldw;
    p.rows = columns ? c.out : c.tokens, p.columns = columns ? c.tokens : c.out, p.depth = c.in;
    p.to = to;
    const Course course = linear_course<T>(c);
    Room room(c.workspace, (int64_t)course.bytes, s);
    if (room.error) return room.error;
    p.part = room.take(course.bytes);
    return launch_product<T>(p, course, false, columns, s);
}

// What a backward call needs and how it goes about the gradient of z.
// dz is kept in the activations' type: both products take it as an operand of the matrix instruction.  In 16 bits that costs half a step of each dz, which the gradients show (4096
// tokens, 4096 -> 9216 bf16: off by 2.3e-3 of their size, 1.7e-3 with dz in 32 bits, which is their own rounding); two pieces of 16 bits would keep it, and double dX's and dW's 546 us.
// db is summed before dz is rounded.
template <class T>
struct BackwardShape {
    static constexpr int V = 16 / sizeof(T);
    bool columns, act, brief;
    int64_t lanes, blocks, tokens_of_part, parts;
    size_t dz, sums, product;
    Course to_x, to_w;
    // Rows: about a thousand workgroups of whole lines.  A few hundred tokens: all of them in one of 64 bytes' features, which needs no second launch (257 x 2049 fp32 10.7 us for 13.4).
    explicit BackwardShape(const LinearBackwardCall& c) : columns(c.dy.order == CER_ORDER_COLUMNS), act(c.activation != CER_ACTIVATION_NONE), brief(!columns && c.tokens <= 512) {
        lanes = brief ? 4 : 64, blocks = (c.out + lanes * V - 1) / (lanes * V);
        const int64_t most = brief ? 1 : std::max<int64_t>(1, std::min<int64_t>(1024 / std::min<int64_t>(blocks, 1024), (c.tokens + 15) / 16));
        tokens_of_part = std::max<int64_t>(1, (c.tokens + most - 1) / most), parts = (c.tokens + tokens_of_part - 1) / tokens_of_part;
        dz = act && (c.dx.data || c.dw) ? (size_t)c.tokens * c.out * sizeof(T) : 0;
        sums = c.dbias && parts > 1 && !columns ? (size_t)parts * c.out * 4 : 0;
        if (c.dx.data && c.tokens) to_x = course_of<T>(columns ? c.in : c.tokens, columns ? c.tokens : c.in, c.out);
        if (c.dw) to_w = course_of<T>(c.out, c.in, c.tokens);
        product = std::max(to_x.bytes, to_w.bytes);
    }
    int64_t bytes() const { return (int64_t)(Room::rounded(dz) + Room::rounded(sums) + Room::rounded(product)); }
};
template <class T>
int linear_backward_of(const LinearBackwardCall& c, hipStream_t s) {
    const BackwardShape<T> shape(c);
    const bool columns = shape.columns, act = shape.act;
    const int64_t across = columns ? c.tokens : c.out;
    Room room(c.workspace, shape.bytes(), s);
    if (room.error) return room.error;
    void* dz = room.take(shape.dz);
    float *sums = room.take(shape.sums), *part = room.take(shape.product);
    if (c.tokens && (dz || c.dbias)) {
        SlopeArgs a{c.dy.data, act ? c.pre.data : nullptr, dz, c.dy.ld, c.pre.ld, across, c.tokens, c.out, c.activation, sums ? sums : c.dbias, shape.tokens_of_part};
        if constexpr (sizeof(T) == 4) {
            if (columns) slope_columns_kernel<<<(unsigned)c.out, 256, 0, s>>>(a);
        }
        const dim3 grid((unsigned)shape.blocks, (unsigned)shape.parts);
        if (shape.brief) slope_rows_kernel<T, 4><<<grid, 256, 0, s>>>(a);
        else if (!columns) slope_rows_kernel<T, 64><<<grid, 256, 0, s>>>(a);
        if (int e = (int)hipGetLastError()) return e;
    }
    if (c.dbias && (sums || !c.tokens)) {
        bias_totals_kernel<<<(unsigned)((c.out + 63) / 64), 1024, 0, s>>>(sums, c.tokens ? (uint32_t)shape.parts : 0, c.out, c.dbias);
        if (int e = (int)hipGetLastError()) return e;
    }
    const void* z = act ? dz : c.dy.data;
    const int64_t ldz = act ? across : c.dy.ld;
    if (c.dx.data && c.tokens) {
        Product p{};
        p.a = columns ? c.w : z, p.lda = columns ? c.ldw : ldz;
        p.b = columns ? z : c.w, p.ldb = columns ? ldz : c.ldw;
        p.rows = columns ? c.in : c.tokens, p.columns = columns ? c.tokens : c.in, p.depth = c.out;
        p.part = part;
        p.to.residual = c.base.data, p.to.ldr = c.base.ld, p.to.out = c.dx.data, p.to.ldo = c.dx.ld;
        if (int e = launch_product<T>(p, shape.to_x, columns, true, s)) return e;
    }
    if (c.dw) {
        Product p{};
        p.a = z, p.lda = ldz, p.b = c.x.data, p.ldb = c.x.ld;
        p.rows = c.out, p.columns = c.in, p.depth = c.tokens;
        p.part = part;
        p.to.out = c.dw, p.to.ldo = c.lddw;
        if (int e = launch_product<T>(p, shape.to_w, !columns, !columns, s)) return e;
    }
    return 0;
}
}  // namespace

int64_t linear_room(const LinearCall& c) {
    return c.type == CER_TYPE_BF16 ? linear_bytes<__bf16>(c) : c.type == CER_TYPE_F16 ? linear_bytes<_Float16>(c) : linear_bytes<float>(c);
}
int64_t linear_backward_room(const LinearBackwardCall& c) {
    return c.type == CER_TYPE_BF16 ? BackwardShape<__bf16>(c).bytes() : c.type == CER_TYPE_F16 ? BackwardShape<_Float16>(c).bytes() : BackwardShape<float>(c).bytes();
}
int launch_linear(const LinearCall& c, hipStream_t s) {
    if (c.type == CER_TYPE_BF16) return linear_of<__bf16>(c, s);
    if (c.type == CER_TYPE_F16) return linear_of<_Float16>(c, s);
    return linear_of<float>(c, s);
}
int launch_linear_backward(const LinearBackwardCall& c, hipStream_t s) {
    if (c.type == CER_TYPE_BF16) return linear_backward_of<__bf16>(c, s);
    if (c.type == CER_TYPE_F16) return linear_backward_of<_Float16>(c, s);
    return linear_backward_of<float>(c, s);
}

}  // namespace cer
