// Dense products with an epilogue: z = X W^T + b, Y = r + act(z), and the gradients of X, W and b.
//
// Three products, one kernel:   C[i][j] = sum_k A(i, k) B(j, k)
//     Y  (tokens x out)   A = X,     B = W         both with k side by side in memory
//     dX (tokens x in)    A = dz,    B = W         B with j side by side
//     dW (out x in)       A = dz,    B = X         A with i, B with j side by side (k: tokens)
// and for activations in columns the same with the operands' places and orders exchanged, so that C's rows are always contiguous.
//
// A workgroup forms a tile of C.  128 bytes of k (64 numbers of 16 bits, 32 of fp32) of all its rows go from memory through registers into LDS while
// the tile before is multiplied: by element-aligned loads, so that any leading dimension works, and an operand whose k lies a line apart is turned in
// registers on the way (8 x 4 numbers a thread).  LDS holds rows of 128 bytes whose eight 16-byte chunks are permuted (`place`), so that both the turned
// stores and the operand loads of 32 rows touch every bank evenly.  The matrix instruction takes B's rows as its first operand: a lane
// then has four neighbouring j of one i.  fp32 goes through the 32-bit instruction.  Sums are fp32; each C is rounded once, after the epilogue.
// Where the tiles are too few for the chip the contraction is cut into parts, which a second launch adds up in their order.
#include <algorithm>

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
// q = 1 / (1 + exp(-u)) and q (1 - q), neither by a difference; 0 and 1, and 0, at the ends.
struct Logistic {
    float q, both;
    __device__ explicit Logistic(float u) {
        const float e = expf(-fabsf(u)), inverse = 1.f / (1.f + e);
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

__device__ __forceinline__ float activate(float z, int kind) {
    switch (kind) {
        case CER_ACTIVATION_RELU: return z < 0.f ? 0.f : z;  // NaN stays
        case CER_ACTIVATION_GELU: return part_of(z, normal_share(z));
        case CER_ACTIVATION_GELU_TANH: return part_of(z, Logistic(tanh_argument(z)).q);
        case CER_ACTIVATION_SILU: return part_of(z, Logistic(z).q);
        default: return z;
    }
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
    float* part;          // [parts][rows][columns], or nullptr: one part, through the epilogue
    int64_t depth_of_part;
    uint32_t tiles_i, tiles_j;
};

// Four neighbouring j of row i, `left` of them in the matrix.
template <class T>
__device__ __forceinline__ void finish(const Epilogue& to, int64_t i, int64_t j, Vec<float, 4> z, int64_t left) {
    if (to.bias) z += to.bias_rows ? Vec<float, 4>(load_some_of<1>(to.bias, to.bias_type, i, 1)[0]) : load_some_of<4>(to.bias, to.bias_type, j, left);
    if (to.pre) store_some<T, 4>(static_cast<T*>(to.pre) + i * to.ldp + j, z, left);
    if (to.activation)
#pragma unroll
        for (int q = 0; q < 4; ++q) z[q] = activate(z[q], to.activation);
    if (to.residual) z += load_some<T, 4>(static_cast<const T*>(to.residual) + i * to.ldr + j, left);
    store_some<T, 4>(static_cast<T*>(to.out) + i * to.ldo + j, z, left);
}

// Where chunk c of a row lies: eight neighbouring rows, and eight rows four apart, have the same chunk in different places.
__device__ __forceinline__ unsigned place(unsigned row, unsigned c) { return row * 8 + (c ^ (row & 7) ^ (row >> 3 & 3)); }

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

// One operand's way from memory to LDS: kRows rows of 128 bytes of k.  Rows past the matrix repeat its last one or are 0 (their results are dropped);
// k past the end is 0 on both sides.
template <class T, int kRows, int kThreads, bool kTurn>
struct Stage {
    static constexpr int E = 16 / sizeof(T), kDepth = 8 * E;
    static constexpr int kPieces = kTurn ? kRows * 2 : kRows * 8, kCount = (kPieces + kThreads - 1) / kThreads;  // turned: 4 rows by a chunk
    const T* at[kCount];
    int left[kTurn ? kCount : 1];
    Chunk held[kTurn ? 1 : kCount];
    Vec<T, 4> lines[kTurn ? kCount : 1][kTurn ? E : 1];

    static __device__ __forceinline__ unsigned piece(int n) { return threadIdx.x + n * kThreads; }
    static __device__ __forceinline__ bool busy(int n) { return kPieces % kThreads == 0 || piece(n) < (unsigned)kPieces; }
    static __device__ __forceinline__ unsigned row(int n) { return kTurn ? piece(n) % (kRows / 4) * 4 : piece(n) / 8; }
    static __device__ __forceinline__ unsigned chunk(int n) { return kTurn ? piece(n) / (kRows / 4) : piece(n) % 8; }

    __device__ __forceinline__ void start(const void* base, int64_t ld, int64_t row0, int64_t rows, int64_t k0) {
#pragma unroll
        for (int n = 0; n < kCount; ++n) {
            const int64_t i = row0 + row(n), k = k0 + chunk(n) * E;
            if constexpr (kTurn) {
                at[n] = static_cast<const T*>(base) + k * ld + i;
                left[n] = (int)(rows - i < 4 ? rows - i : 4);
            } else {
                at[n] = static_cast<const T*>(base) + (i < rows ? i : rows - 1) * ld + k;
            }
        }
    }
    // The next kDepth of k; `remain`: how many there are up to the end.
    __device__ __forceinline__ void load_next(int64_t ld, int64_t remain) {
#pragma unroll
        for (int n = 0; n < kCount; ++n) {
            if (!busy(n)) continue;
            if constexpr (kTurn) {
                const int64_t k = remain - chunk(n) * E;
                if (remain >= kDepth && left[n] == 4) {
#pragma unroll
                    for (int q = 0; q < E; ++q) lines[n][q] = load<T, 4>(at[n] + q * ld);
                } else {
#pragma unroll
                    for (int q = 0; q < E; ++q) lines[n][q] = load_own<T, 4>(at[n] + q * ld, q < k ? left[n] : 0);
                }
                at[n] += kDepth * ld;
            } else {
                if (remain >= kDepth) held[n] = __builtin_bit_cast(Chunk, (load<T, E>(at[n])));
                else held[n] = __builtin_bit_cast(Chunk, (load_own<T, E>(at[n], remain - chunk(n) * E)));
                at[n] += kDepth;
            }
        }
    }
    __device__ __forceinline__ void to_lds(Chunk* room) const {
#pragma unroll
        for (int n = 0; n < kCount; ++n) {
            if (!busy(n)) continue;
            if constexpr (kTurn) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    Vec<T, E> line;
#pragma unroll
                    for (int q = 0; q < E; ++q) line[q] = lines[n][q][r];
                    room[place(row(n) + r, chunk(n))] = __builtin_bit_cast(Chunk, line);
                }
            } else {
                room[place(row(n), chunk(n))] = held[n];
            }
        }
    }
};

// Neighbouring workgroups run on different dies, each with a cache of its own: a die gets neighbouring tiles, eight rows of tiles at a time.
__device__ __forceinline__ void tile_of(unsigned id, unsigned tiles_i, unsigned tiles_j, unsigned* ti, unsigned* tj) {
    const unsigned all = tiles_i * tiles_j, die = id % 8, each = all / 8, more = all % 8;
    id = die * each + (die < more ? die : more) + id / 8;
    const unsigned group = id / (8 * tiles_j), first = group * 8, high = tiles_i - first < 8 ? tiles_i - first : 8;
    id -= first * tiles_j;
    *ti = first + id % high;
    *tj = id / high;
}

template <class T, int kI, int kJ, int kWavesI, int kWavesJ, bool kTurnA, bool kTurnB>
__global__ __launch_bounds__(64 * kWavesI * kWavesJ) void product_kernel(Product p) {
    constexpr int kThreads = 64 * kWavesI * kWavesJ, kWideI = kI / kWavesI, kWideJ = kJ / kWavesJ, kTilesI = kWideI / 32, kTilesJ = kWideJ / 32;
    constexpr int kPitch = kWideJ + 4;
    using StageA = Stage<T, kI, kThreads, kTurnA>;
    using StageB = Stage<T, kJ, kThreads, kTurnB>;
    constexpr int kDepth = StageA::kDepth;
    __shared__ Chunk room[2][(kI + kJ) * 8];
    static_assert(sizeof(room) >= sizeof(float) * kWavesI * kWavesJ * 32 * kPitch, "");
    const unsigned lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wave_i = wave / kWavesJ, wave_j = wave % kWavesJ;
    unsigned ti, tj;
    tile_of(blockIdx.x, p.tiles_i, p.tiles_j, &ti, &tj);
    const int64_t i0 = (int64_t)ti * kI, j0 = (int64_t)tj * kJ, k0 = (int64_t)blockIdx.y * p.depth_of_part;
    int64_t remain = p.depth - k0 < p.depth_of_part ? p.depth - k0 : p.depth_of_part;
    StageA a;
    StageB b;
    a.start(p.a, p.lda, i0, p.rows, k0);
    b.start(p.b, p.ldb, j0, p.columns, k0);
    F16 sums[kTilesI][kTilesJ];
#pragma unroll
    for (int x = 0; x < kTilesI; ++x)
#pragma unroll
        for (int y = 0; y < kTilesJ; ++y) sums[x][y] = 0.f;
    if (remain > 0) {
        a.load_next(p.lda, remain);
        b.load_next(p.ldb, remain);
        a.to_lds(room[0]);
        b.to_lds(room[0] + kI * 8);
        __syncthreads();
    }
    for (unsigned turn = 0; remain > 0; turn ^= 1) {
        remain -= kDepth;
        if (remain > 0) {
            a.load_next(p.lda, remain);
            b.load_next(p.ldb, remain);
        }
        const Chunk *from_a = room[turn] + wave_i * kWideI * 8, *from_b = room[turn] + (kI + wave_j * kWideJ) * 8;
#pragma unroll
        for (unsigned step = 0; step < 4; ++step) {
            Chunk x[kTilesI], y[kTilesJ];
#pragma unroll
            for (int k = 0; k < kTilesI; ++k) x[k] = from_a[place(lane & 31, 2 * step + (lane >> 5)) + k * 256];
#pragma unroll
            for (int k = 0; k < kTilesJ; ++k) y[k] = from_b[place(lane & 31, 2 * step + (lane >> 5)) + k * 256];
#pragma unroll
            for (int i = 0; i < kTilesI; ++i)
#pragma unroll
                for (int j = 0; j < kTilesJ; ++j) sums[i][j] = multiply<T>(y[j], x[i], sums[i][j]);
        }
        if (remain > 0) {
            a.to_lds(room[turn ^ 1]);
            b.to_lds(room[turn ^ 1] + kI * 8);
        }
        __syncthreads();
    }
    // 32 rows of each wave at a time through LDS, so that neighbouring lanes have neighbouring numbers of a row
    float* own = reinterpret_cast<float*>(room) + wave * 32 * kPitch;
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
        constexpr int kAbreast = kWideJ / 4;
        const int64_t j = j0 + wave_j * kWideJ + lane % kAbreast * 4;
#pragma unroll 1
        for (int row = lane / kAbreast; row < 32; row += 64 / kAbreast) {
            const int64_t i = i0 + wave_i * kWideI + x * 32 + row;
            if (i >= p.rows || j >= p.columns) continue;
            const Vec<float, 4> z = *reinterpret_cast<const Vec<float, 4>*>(own + row * kPitch + lane % kAbreast * 4);
            if (p.part) store_some<float, 4>(p.part + (blockIdx.y * p.rows + i) * p.columns + j, z, p.columns - j);
            else finish<T>(p.to, i, j, z, p.columns - j);
        }
    }
}

// The parts added up in their order, then the epilogue: four neighbouring numbers of C a thread.
template <class T>
__global__ __launch_bounds__(256) void parts_kernel(Product p, uint32_t parts) {
    const int64_t abreast = (p.columns + 3) / 4, at = (int64_t)blockIdx.x * 256 + threadIdx.x, i = at / abreast, j = at % abreast * 4;
    if (i >= p.rows) return;
    Vec<float, 4> z = 0.f;
#pragma unroll 8
    for (uint32_t k = 0; k < parts; ++k) z += load_some<float, 4>(p.part + (k * p.rows + i) * p.columns + j, p.columns - j);
    finish<T>(p.to, i, j, z, p.columns - j);
}

template <class T, int kI, int kJ, int kWavesI, int kWavesJ>
int launch_tiles(Product p, bool turn_a, bool turn_b, unsigned parts, hipStream_t s) {
    p.tiles_i = (uint32_t)((p.rows + kI - 1) / kI), p.tiles_j = (uint32_t)((p.columns + kJ - 1) / kJ);
    const dim3 grid(p.tiles_i * p.tiles_j, parts);
    constexpr int kThreads = 64 * kWavesI * kWavesJ;
    if (!turn_b) product_kernel<T, kI, kJ, kWavesI, kWavesJ, false, false><<<grid, kThreads, 0, s>>>(p);
    else if (!turn_a) product_kernel<T, kI, kJ, kWavesI, kWavesJ, false, true><<<grid, kThreads, 0, s>>>(p);
    else product_kernel<T, kI, kJ, kWavesI, kWavesJ, true, true><<<grid, kThreads, 0, s>>>(p);
    return (int)hipGetLastError();
}

template <class T>
int launch_product(Product p, bool turn_a, bool turn_b, hipStream_t s) {
    constexpr int64_t kDepth = 128 / sizeof(T);
    const auto tiles = [&](int64_t side) { return ((p.rows + side - 1) / side) * ((p.columns + side - 1) / side); };
    const int64_t side = sizeof(T) == 2 && tiles(256) >= 192 ? 256 : tiles(128) >= 192 ? 128 : 64, steps = (p.depth + kDepth - 1) / kDepth;
    int64_t parts = 1;
    if (tiles(side) < 384 && side == 64) parts = std::max<int64_t>(1, std::min<int64_t>({768 / tiles(side), steps / 4, 64}));
    const int64_t of_part = (std::max<int64_t>(steps, 1) + parts - 1) / parts;
    parts = std::max<int64_t>(1, (steps + of_part - 1) / of_part);
    p.depth_of_part = of_part * kDepth;
    Temporary t(parts > 1 ? (size_t)parts * p.rows * p.columns * 4 : 0, s);
    if (t.error) return t.error;
    p.part = t.floats();
    int e;
    if (side == 64) e = launch_tiles<T, 64, 64, 2, 2>(p, turn_a, turn_b, (unsigned)parts, s);
    else if (side == 128) e = launch_tiles<T, 128, 128, 2, 2>(p, turn_a, turn_b, (unsigned)parts, s);
    else if constexpr (sizeof(T) == 2) e = launch_tiles<T, 256, 256, 2, 4>(p, turn_a, turn_b, (unsigned)parts, s);
    else return (int)hipErrorInvalidValue;
    if (e || parts == 1) return e;
    parts_kernel<T><<<(unsigned)((p.rows * ((p.columns + 3) / 4) + 255) / 256), 256, 0, s>>>(p, (uint32_t)parts);
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

// Rows: 64 lanes of V features by 4 waves, each of every fourth token of the workgroup's part.
template <class T>
__global__ __launch_bounds__(256) void slope_rows_kernel(SlopeArgs a) {
    constexpr int V = 16 / sizeof(T);
    __shared__ Vec<float, V> room[4][64];
    const unsigned lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t e = ((int64_t)blockIdx.x * 64 + lane) * V, left = a.out - e;
    const int64_t first = blockIdx.y * a.tokens_of_part, last = first + a.tokens_of_part < a.tokens ? first + a.tokens_of_part : a.tokens;
    Vec<float, V> sums = 0.f;
    if (left > 0)
#pragma unroll 2
        for (int64_t t = first + wave; t < last; t += 4) {
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
    room[wave][lane] = sums;
    __syncthreads();
    if (wave == 0 && left > 0) store_some<float, V>(a.sums + blockIdx.y * a.out + e, room[0][lane] + room[1][lane] + (room[2][lane] + room[3][lane]), left);
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
int linear_of(const LinearCall& c, hipStream_t s) {
    const bool columns = c.x.order == CER_ORDER_COLUMNS;
    Product p{};
    p.a = columns ? c.w : c.x.data, p.lda = columns ? c.ldw : c.x.ld;
    p.b = columns ? c.x.data : c.w, p.ldb = columns ? c.x.ld : c.ldw;
    p.rows = columns ? c.out : c.tokens, p.columns = columns ? c.tokens : c.out, p.depth = c.in;
    p.to = {c.bias, c.bias_type, columns, c.activation, c.residual.data, c.pre.data, c.y.data, c.residual.ld, c.pre.ld, c.y.ld};
    return launch_product<T>(p, false, columns, s);
}

template <class T>
int linear_backward_of(const LinearBackwardCall& c, hipStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const bool columns = c.dy.order == CER_ORDER_COLUMNS, act = c.activation != CER_ACTIVATION_NONE, product = c.dx.data || c.dw;
    const int64_t across = columns ? c.tokens : c.out;
    // rows: about a thousand workgroups, each of whole tokens
    const int64_t blocks = (c.out + 64 * V - 1) / (64 * V), most = std::max<int64_t>(1, std::min<int64_t>(1024 / std::min<int64_t>(blocks, 1024), (c.tokens + 15) / 16));
    const int64_t tokens_of_part = std::max<int64_t>(1, (c.tokens + most - 1) / most), parts = (c.tokens + tokens_of_part - 1) / tokens_of_part;
    Temporary dz(act && product ? (size_t)c.tokens * c.out * sizeof(T) : 0, s), sums(c.dbias && !columns ? (size_t)parts * c.out * 4 : 0, s);
    if (dz.error || sums.error) return dz.error ? dz.error : sums.error;
    if (c.tokens && (dz.p || c.dbias)) {
        SlopeArgs a{c.dy.data, act ? c.pre.data : nullptr, dz.p, c.dy.ld, c.pre.ld, across, c.tokens, c.out, c.activation, columns ? c.dbias : sums.floats(), tokens_of_part};
        if constexpr (sizeof(T) == 4) {
            if (columns) slope_columns_kernel<<<(unsigned)c.out, 256, 0, s>>>(a);
        }
        if (!columns) slope_rows_kernel<T><<<dim3((unsigned)blocks, (unsigned)parts), 256, 0, s>>>(a);
        if (int e = (int)hipGetLastError()) return e;
    }
    if (c.dbias && (!columns || !c.tokens)) {
        bias_totals_kernel<<<(unsigned)((c.out + 63) / 64), 1024, 0, s>>>(sums.floats(), c.tokens ? (uint32_t)parts : 0, c.out, c.dbias);
        if (int e = (int)hipGetLastError()) return e;
    }
    const void* z = act ? dz.p : c.dy.data;
    const int64_t ldz = act ? across : c.dy.ld;
    if (c.dx.data && c.tokens) {
        Product p{};
        p.a = columns ? c.w : z, p.lda = columns ? c.ldw : ldz;
        p.b = columns ? z : c.w, p.ldb = columns ? ldz : c.ldw;
        p.rows = columns ? c.in : c.tokens, p.columns = columns ? c.tokens : c.in, p.depth = c.out;
        p.to.residual = c.base.data, p.to.ldr = c.base.ld, p.to.out = c.dx.data, p.to.ldo = c.dx.ld;
        if (int e = launch_product<T>(p, columns, true, s)) return e;
    }
    if (c.dw) {
        Product p{};
        p.a = z, p.lda = ldz, p.b = c.x.data, p.ldb = c.x.ld;
        p.rows = c.out, p.columns = c.in, p.depth = c.tokens;
        p.to.out = c.dw, p.to.ldo = c.lddw;
        if (int e = launch_product<T>(p, !columns, !columns, s)) return e;
    }
    return 0;
}
}  // namespace

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
