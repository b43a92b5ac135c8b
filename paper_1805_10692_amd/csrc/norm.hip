// Root-mean-square norm with the residual's addition, and its gradient.
//
// Forward, token t, feature i:   h = x + r;   rstd = 1 / sqrt(1/n sum_i h_i^2 + eps);   y_i = h_i rstd w_i.
// Backward:   g_i = dy_i w_i;   c = 1/n sum_i g_i h_i rstd;   dx_i = rstd (g_i - h_i rstd c) + dsum_i;   dw_i = sum_t dy_i h_i rstd.
// Everything is computed in 32 bits; what goes out in fewer is rounded once.  A few operations per element: the bytes bound it.
//
// Rows (a token's features one after the other): a workgroup takes a token and keeps its h in registers between the sum and the
// product, so that every input is read once and every output written once.  Columns (feature after feature, the order of
// cer_matmul's X): a token's features lie tokens * 4 bytes apart, so that a workgroup that owned whole tokens would either own
// too many of them for their number of features to fill the chip or read a few bytes of every line.  There the sums come first, a
// workgroup for 64 tokens and a part of the features, and a second launch adds the parts up and writes y, through LDS where x and y
// differ in their order.  That reads x (and r) twice, the second time mostly from the caches.
//
// Measured, per call back to back (a large copy reaches 5.0 TB/s on the same card): one token of 4096 features 4.2 us, the launch; 8192 x 4096 bf16 with
// residual and 8-bit outputs 61 us, 3.8 TB/s; backward of 4096 x 4608 bf16 38.5 us, 3.9 TB/s; 99 tokens x 9216, bf16 rows to fp32 columns 9.8 us, two launches.
// Persistent workgroups that request the next token's inputs ahead were slower (63 and 43 us).
// Backward, over 16384 features: a token's three copies do not fit the registers of 1024 threads and spill (1024 x 25088 bf16 309 us, fp32 1650; x 16384 35 and 67).
#include <algorithm>

#include "operators.hpp"

namespace cer {
namespace {

struct NormArgs {
    const void *x, *r;
    void *sum, *y;
    int64_t ldx, ldr, ldsum, ldy;
    int64_t tokens, n;
    const void* w;
    int32_t w_type;
    float eps, inverse_n;
    float *scale, *rstd;
    float* part;      // columns: [parts][tokens] sums of squares
    uint32_t parts;   // how many of them
};

// ---- rows -----------------------------------------------------------------------------------------------------------------------
// kChunks vectors of 16 bytes of x per thread.  y == nullptr: only the sum of squares (to `part`).
template <class TX, class TY, int kChunks>
__global__ __launch_bounds__(1024) void norm_rows_kernel(NormArgs a) {
    constexpr int V = 16 / sizeof(TX);
    constexpr bool k8 = sizeof(TY) == 1;
    __shared__ float room[4][16];
    unsigned turn = 0;
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x, turn ^= 2) {
        const TX* x = static_cast<const TX*>(a.x) + t * a.ldx;
        Vec<float, V> h[kChunks];
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
            h[c] = load_some<TX, V>(x + e, a.n - e);
        }
        if (a.r) {
            const TX* r = static_cast<const TX*>(a.r) + t * a.ldr;
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
                h[c] += load_some<TX, V>(r + e, a.n - e);
            }
        }
        // few registers: the weights are on their way while the squares are added up
        constexpr bool kEarly = kChunks * V <= 16;
        Vec<float, V> w[kEarly ? kChunks : 1];
        if (kEarly && a.w && a.y)
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
                w[kEarly ? c : 0] = load_some_of<V>(a.w, a.w_type, e, a.n - e);
            }
        float squares = 0.f;
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int j = 0; j < V; ++j) squares = fmaf(h[c][j], h[c][j], squares);
        if (a.sum) {
            TX* sum = static_cast<TX*>(a.sum) + t * a.ldsum;
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
                store_some<TX, V>(sum + e, h[c], a.n - e);
            }
        }
        squares = block_total(squares, room[turn]);
        if (!a.y) {
            if (threadIdx.x == 0) a.part[t] = squares;
            continue;
        }
        const float rstd = rsqrtf(fmaf(squares, a.inverse_n, a.eps));
        if (a.rstd && threadIdx.x == 0) a.rstd[t] = rstd;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
            h[c] *= rstd;
            if (a.w) h[c] *= kEarly ? w[kEarly ? c : 0] : load_some_of<V>(a.w, a.w_type, e, a.n - e);
        }
        if constexpr (k8) {
            float most = 0.f;
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
#pragma unroll
                for (int j = 0; j < V; ++j) most = larger(most, fabsf(h[c][j]));
            most = block_total<true>(most, room[turn + 1]);
            const float scale = most == 0.f ? 1.f : larger(most / kLargestF8, 0x1p-126f);  // its inverse is finite
            const float inverse = 1.f / scale;
            if (threadIdx.x == 0) a.scale[t] = scale;
            uint8_t* y = static_cast<uint8_t*>(a.y) + t * a.ldy;
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
                Vec<uint32_t, V / 4> code;
#pragma unroll
                for (int q = 0; q < V / 4; ++q) {
                    // a quotient that rounding has put past the largest code's middle is the largest code
                    float v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float u = h[c][4 * q + j] * inverse;
                        v[j] = u > kLargestF8 ? kLargestF8 : u < -kLargestF8 ? -kLargestF8 : u;
                    }
                    int word = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
                    code[q] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], word, true);
                }
                if (e + V <= a.n) {
                    typedef uint32_t Words __attribute__((ext_vector_type(V / 4), aligned(1)));
                    *reinterpret_cast<Words*>(y + e) = code;
                } else {
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        if (e + j < a.n) y[e + j] = (uint8_t)(code[j / 4] >> (8 * (j % 4)));
                }
            }
        } else {
            TY* y = static_cast<TY*>(a.y) + t * a.ldy;
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
                store_some<TY, V>(y + e, h[c], a.n - e);
            }
        }
    }
}

template <class TX, class TY, int kChunks>
int norm_rows_chunks(const NormArgs& a, hipStream_t s) {
    constexpr int V = 16 / sizeof(TX);
    const int64_t vectors = (a.n + V - 1) / V;
    const unsigned threads = (unsigned)(((vectors + kChunks - 1) / kChunks + 63) / 64 * 64);
    const unsigned grid = (unsigned)std::min<int64_t>(a.tokens, 1 << 20);
    norm_rows_kernel<TX, TY, kChunks><<<grid, threads, 0, s>>>(a);
    return (int)hipGetLastError();
}

// How many vectors of 16 bytes a thread takes: as few as the 1024 threads of a workgroup allow.
template <class TX, class TY>
int norm_rows(const NormArgs& a, hipStream_t s) {
    constexpr int V = 16 / sizeof(TX);
    const int64_t vectors = (a.n + V - 1) / V;
    if (vectors <= 1024) return norm_rows_chunks<TX, TY, 1>(a, s);
    if (vectors <= 2048) return norm_rows_chunks<TX, TY, 2>(a, s);
    if (vectors <= 4096) return norm_rows_chunks<TX, TY, 4>(a, s);
    if constexpr (V == 4)
        if (vectors > 8192) return norm_rows_chunks<TX, TY, 16>(a, s);  // up to 65536 features
    return norm_rows_chunks<TX, TY, 8>(a, s);
}

// ---- columns --------------------------------------------------------------------------------------------------------------------
// A wave holds 64 / wide features by `wide` tokens (a power of two up to 64), so that few tokens do not leave lanes idle.
struct Lanes {
    unsigned wide;
    __device__ Lanes(int64_t tokens) : wide(64) {
        while (wide > 1 && wide / 2 >= tokens) wide /= 2;
    }
    __device__ unsigned token() const { return threadIdx.x & (wide - 1); }
    __device__ unsigned feature() const { return threadIdx.x / wide; }  // of a step of blockDim.x / wide
    __device__ unsigned step() const { return blockDim.x / wide; }
};

// x, r, sum in columns.  Workgroup (b, p): 64 tokens, part p of the features.
template <int kThreads>
__global__ __launch_bounds__(kThreads) void norm_columns_sums_kernel(NormArgs a, int64_t features) {
    __shared__ float room[kThreads];
    const Lanes l(a.tokens);
    const int64_t t = (int64_t)blockIdx.x * l.wide + l.token();
    const int64_t first = blockIdx.y * features, last = first + features < a.n ? first + features : a.n;
    float squares = 0.f;
    if (t < a.tokens) {
        const float* x = static_cast<const float*>(a.x) + t;
        const float* r = static_cast<const float*>(a.r) + (a.r ? t : 0);
        float* sum = static_cast<float*>(a.sum) + (a.sum ? t : 0);
#pragma unroll 4
        for (int64_t i = first + l.feature(); i < last; i += l.step()) {
            float h = x[i * a.ldx];
            if (a.r) h += r[i * a.ldr];
            if (a.sum) sum[i * a.ldsum] = h;
            squares = fmaf(h, h, squares);
        }
    }
    room[threadIdx.x] = squares;
    __syncthreads();
    for (unsigned k = kThreads / 2; k >= l.wide; k /= 2) {
        if (threadIdx.x < k) room[threadIdx.x] += room[threadIdx.x + k];
        __syncthreads();
    }
    if (threadIdx.x < l.wide && t < a.tokens) a.part[blockIdx.y * a.tokens + t] = room[threadIdx.x];
}

// 1 / rms of `wide` tokens from the parts of their sums of squares, into LDS.  All threads call it.
__device__ __forceinline__ void norm_of_tokens(const NormArgs& a, int64_t first, unsigned wide, float* room, float* rstd, bool write) {
    const unsigned token = threadIdx.x % wide;
    const int64_t t = first + token;
    float squares = 0.f;
    if (t < a.tokens)
        for (unsigned p = threadIdx.x / wide; p < a.parts; p += blockDim.x / wide) squares += a.part[p * a.tokens + t];
    room[threadIdx.x] = squares;
    __syncthreads();
    if (threadIdx.x < wide) {
        float all = 0.f;
        for (unsigned k = threadIdx.x; k < blockDim.x; k += wide) all += room[k];
        const float v = rsqrtf(fmaf(all, a.inverse_n, a.eps));
        rstd[token] = v;
        if (write && a.rstd && t < a.tokens) a.rstd[t] = v;
    }
    __syncthreads();
}

// x and y in columns: y from `sum` where it is there (in 32 bits it is h itself), else from x and r.
template <int kThreads>
__global__ __launch_bounds__(kThreads) void norm_columns_kernel(NormArgs a, int64_t features) {
    __shared__ float room[kThreads], rstds[64];
    const Lanes l(a.tokens);
    const int64_t t = (int64_t)blockIdx.x * l.wide + l.token();
    norm_of_tokens(a, (int64_t)blockIdx.x * l.wide, l.wide, room, rstds, blockIdx.y == 0);
    if (t >= a.tokens) return;
    const int64_t first = blockIdx.y * features, last = first + features < a.n ? first + features : a.n;
    const float rstd = rstds[l.token()];
    const float* x = static_cast<const float*>(a.sum ? a.sum : a.x) + t;
    const float* r = a.sum ? nullptr : static_cast<const float*>(a.r);
    const int64_t ldx = a.sum ? a.ldsum : a.ldx;
    float* y = static_cast<float*>(a.y) + t;
#pragma unroll 4
    for (int64_t i = first + l.feature(); i < last; i += l.step()) {
        float h = x[i * ldx];
        if (r) h += r[t + i * a.ldr];
        const float w = a.w ? load_some_of<1>(a.w, a.w_type, i, 1)[0] : 1.f;
        y[i * a.ldy] = h * rstd * w;
    }
}

// x and y in different orders: a tile of 64 tokens by 64 features through LDS.  `sum` is written here and not with the sums of squares:
// it may lie where x or r does, and h is wanted in 32 bits both times.  All loads of a thread are on their way before the first store.
template <class TX, class TY, bool kFromColumns>
__global__ __launch_bounds__(256) void norm_turn_kernel(NormArgs a) {
    constexpr int V = 16 / sizeof(TX), kAbreast = 64 / V, kLoads = 64 / (256 / kAbreast);  // threads for a line of the tile; lines for a thread
    __shared__ float tile[64][69], room[256], rstds[64];  // [token][feature]; a pitch that is odd in both directions' banks of four
    const int64_t t0 = (int64_t)blockIdx.x * 64, i0 = (int64_t)blockIdx.y * 64;
    const int along = threadIdx.x % kAbreast * V, line0 = threadIdx.x / kAbreast;
    const TX *x = static_cast<const TX*>(a.x), *r = static_cast<const TX*>(a.r);
    // lines: tokens, or (from columns) features
    const int64_t first = kFromColumns ? i0 : t0, lines = (kFromColumns ? a.n : a.tokens) - first, left = (kFromColumns ? a.tokens - t0 : a.n - i0) - along;
    Vec<float, V> h[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
        const int line = line0 + k * (256 / kAbreast);
        h[k] = line < lines ? load_some<TX, V>(x + (first + line) * a.ldx + (kFromColumns ? t0 : i0) + along, left) : Vec<float, V>(0.f);
    }
    if (r)
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            const int line = line0 + k * (256 / kAbreast);
            if (line < lines) h[k] += load_some<TX, V>(r + (first + line) * a.ldr + (kFromColumns ? t0 : i0) + along, left);
        }
    norm_of_tokens(a, t0, 64, room, rstds, blockIdx.y == 0);
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
        const int line = line0 + k * (256 / kAbreast);
        if (a.sum && line < lines) store_some<TX, V>(static_cast<TX*>(a.sum) + (first + line) * a.ldsum + (kFromColumns ? t0 : i0) + along, h[k], left);
#pragma unroll
        for (int j = 0; j < V; ++j) tile[kFromColumns ? along + j : line][kFromColumns ? line : along + j] = h[k][j];
    }
    __syncthreads();
    TY* y = static_cast<TY*>(a.y);
    // y's lines: the other way round, four numbers for a thread
    const int out_along = threadIdx.x % 16 * 4;
    const int64_t out_left = (kFromColumns ? a.n - i0 : a.tokens - t0) - out_along;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int line = threadIdx.x / 16 + 16 * k;
        if (line >= (kFromColumns ? a.tokens - t0 : a.n - i0)) continue;
        Vec<float, 4> v;
        if constexpr (kFromColumns) {  // a token's features
            const Vec<float, 4> w = a.w ? load_some_of<4>(a.w, a.w_type, i0 + out_along, out_left) : Vec<float, 4>(1.f);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = tile[line][out_along + j] * rstds[line] * w[j];
            store_some<TY, 4>(y + (t0 + line) * a.ldy + i0 + out_along, v, out_left);
        } else {
            const float w = a.w ? load_some_of<1>(a.w, a.w_type, i0 + line, 1)[0] : 1.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = tile[out_along + j][line] * rstds[out_along + j] * w;
            store_some<TY, 4>(y + (i0 + line) * a.ldy + t0 + out_along, v, out_left);
        }
    }
}

// Columns on either side: tokens abreast and workgroups for them; the features are cut so that there are about two workgroups for a
// compute unit, at most 64 parts (a workgroup of the second launch adds up its tokens' parts first).
struct ColumnShape {
    unsigned wide = 64, blocks, parts;
    int64_t features;
    ColumnShape(int64_t tokens, int64_t n) {
        while (wide > 1 && wide / 2 >= tokens) wide /= 2;
        blocks = (unsigned)((tokens + wide - 1) / wide);
        const int64_t step = 256 / wide, most = (n + step * 8 - 1) / (step * 8);
        parts = (unsigned)std::max<int64_t>(1, std::min<int64_t>({64, most, 512 / (int64_t)blocks}));
        features = (n + parts - 1) / parts;
        parts = (unsigned)((n + features - 1) / features);
    }
};

template <class TX>
int norm_to(const NormCall& c, NormArgs a, hipStream_t s) {
    const bool from_columns = c.x.order == CER_ORDER_COLUMNS, to_columns = c.y.order == CER_ORDER_COLUMNS;
    if (!from_columns && !to_columns) {
        if (c.y.type == CER_TYPE_F8) return norm_rows<TX, uint8_t>(a, s);
        if (c.y.type == CER_TYPE_F32) return norm_rows<TX, float>(a, s);
        if constexpr (sizeof(TX) != 4) return norm_rows<TX, TX>(a, s);
        return (int)hipErrorInvalidValue;
    }
    const ColumnShape shape(c.tokens, c.n);
    a.parts = from_columns ? shape.parts : 1;
    Temporary t((size_t)c.tokens * a.parts * 4, s);
    if (t.error) return t.error;
    a.part = t.floats();
    int e;
    if (from_columns) {
        if constexpr (sizeof(TX) != 4) return (int)hipErrorInvalidValue;
        NormArgs sums = a;
        if (!to_columns) sums.sum = nullptr;
        norm_columns_sums_kernel<256><<<dim3(shape.blocks, shape.parts), 256, 0, s>>>(sums, shape.features);
        e = (int)hipGetLastError();
    } else {
        NormArgs sums = a;
        sums.y = sums.sum = nullptr;
        e = norm_rows<TX, float>(sums, s);
    }
    if (e) return e;
    if (from_columns && to_columns) {
        norm_columns_kernel<256><<<dim3(shape.blocks, shape.parts), 256, 0, s>>>(a, shape.features);
        return (int)hipGetLastError();
    }
    const dim3 grid((unsigned)((c.tokens + 63) / 64), (unsigned)((c.n + 63) / 64));
    if (from_columns) {
        if constexpr (sizeof(TX) == 4) norm_turn_kernel<float, float, true><<<grid, 256, 0, s>>>(a);
    } else {
        norm_turn_kernel<TX, float, false><<<grid, 256, 0, s>>>(a);
    }
    return (int)hipGetLastError();
}

// ---- backward, rows ------------------------------------------------------------------------------------------------------------
struct BackArgs {
    const void *dy, *h, *dsum;
    void* dx;
    int64_t lddy, ldh, lddsum, lddx;
    int64_t tokens, n;
    const float* rstd;
    const void* w;
    int32_t w_type;
    float inverse_n;
    float* dw;
    float* part;  // [workgroups][n] sums of dy h rstd over the workgroup's tokens
    uint32_t parts;
};

// A workgroup takes tokens blockIdx.x, + gridDim.x, ... and holds its share of dw for its own features in registers: the products' columns
// cost neither atomics, whose order would change dw, nor a second pass over dy and h (4096 x 4608 bf16: 35.4 us, 4.3 TB/s; the parts' sum 4.6 us).
template <class TD, class TH, int kChunks>
__global__ __launch_bounds__(1024) void norm_back_rows_kernel(BackArgs a) {
    constexpr int V = 16 / sizeof(TH);
    __shared__ float room[2][16];
    unsigned turn = 0;
    Vec<float, V> dw[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) dw[c] = 0.f;
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x, turn ^= 1) {
        const TD* dy = static_cast<const TD*>(a.dy) + t * a.lddy;
        const TH* h = static_cast<const TH*>(a.h) + t * a.ldh;
        const float rstd = a.rstd[t];
        Vec<float, V> g[kChunks], hat[kChunks];
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
            g[c] = load_some<TD, V>(dy + e, a.n - e);
            hat[c] = load_some<TH, V>(h + e, a.n - e);
        }
        float along = 0.f;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
            hat[c] *= rstd;
            dw[c] += g[c] * hat[c];
            if (a.w) g[c] *= load_some_of<V>(a.w, a.w_type, e, a.n - e);
#pragma unroll
            for (int j = 0; j < V; ++j) along = fmaf(g[c][j], hat[c][j], along);
        }
        along = block_total(along, room[turn]) * a.inverse_n;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
            Vec<float, V> d = (g[c] - hat[c] * along) * rstd;
            if (a.dsum) d += load_some<TH, V>(static_cast<const TH*>(a.dsum) + t * a.lddsum + e, a.n - e);
            store_some<TH, V>(static_cast<TH*>(a.dx) + t * a.lddx + e, d, a.n - e);
        }
    }
    if (a.part) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
            store_some<float, V>(a.part + blockIdx.x * a.n + e, dw[c], a.n - e);
        }
    }
}

// dw: the parts added up in their order.  A workgroup for 64 features: 16 lanes of four features by 64 rows of parts.
__global__ __launch_bounds__(1024) void norm_back_weight_kernel(const float* part, uint32_t parts, int64_t n, float* dw) {
    __shared__ Vec<float, 4> room[64][17];
    const unsigned lane = threadIdx.x & 15, row = threadIdx.x >> 4;
    const int64_t i = (int64_t)blockIdx.x * 64 + lane * 4;
    Vec<float, 4> all = 0.f;
    if (i < n) {
#pragma unroll 8
        for (uint32_t p = row; p < parts; p += 64) all += load_some<float, 4>(part + p * n + i, n - i);
    }
    room[row][lane] = all;
    __syncthreads();
    for (unsigned k = 32; k; k /= 2) {
        if (row < k) room[row][lane] += room[row + k][lane];
        __syncthreads();
    }
    if (row == 0 && i < n) store_some<float, 4>(dw + i, room[0][lane], n - i);
}

template <class TD, class TH, int kChunks>
int norm_back_rows_chunks(const BackArgs& a, hipStream_t s) {
    constexpr int V = 16 / sizeof(TH);
    const int64_t vectors = (a.n + V - 1) / V;
    const unsigned threads = (unsigned)(((vectors + kChunks - 1) / kChunks + 63) / 64 * 64);
    norm_back_rows_kernel<TD, TH, kChunks><<<a.parts, threads, 0, s>>>(a);
    return (int)hipGetLastError();
}

template <class TD, class TH>
int norm_back_rows(BackArgs a, hipStream_t s) {
    constexpr int V = 16 / sizeof(TH);
    const int64_t vectors = (a.n + V - 1) / V;
    a.parts = (unsigned)std::min<int64_t>(a.tokens, 512);
    Temporary t(a.dw ? (size_t)a.parts * a.n * 4 : 0, s);
    if (t.error) return t.error;
    a.part = t.floats();
    int e;
    if (vectors <= 1024) e = norm_back_rows_chunks<TD, TH, 1>(a, s);
    else if (vectors <= 2048) e = norm_back_rows_chunks<TD, TH, 2>(a, s);
    else if (vectors <= 4096) e = norm_back_rows_chunks<TD, TH, 4>(a, s);
    else if (vectors <= 8192) e = norm_back_rows_chunks<TD, TH, 8>(a, s);
    else e = norm_back_rows_chunks<TD, TH, V == 4 ? 16 : 8>(a, s);  // 32 bits, up to 65536 features
    if (!e && a.dw) {
        norm_back_weight_kernel<<<(unsigned)((a.n + 63) / 64), 1024, 0, s>>>(a.part, a.parts, a.n, a.dw);
        e = (int)hipGetLastError();
    }
    return e;
}

// ---- backward, columns ----------------------------------------------------------------------------------------------------------
// dy, h and the gradients of h in columns.  The products g h rstd are added up per token first, a workgroup for 64 tokens and a part
// of the features; the second launch writes dx, the third dw.
__global__ __launch_bounds__(256) void norm_back_columns_sums_kernel(BackArgs a, int64_t features) {
    __shared__ float room[256];
    const Lanes l(a.tokens);
    const int64_t t = (int64_t)blockIdx.x * l.wide + l.token();
    const int64_t first = blockIdx.y * features, last = first + features < a.n ? first + features : a.n;
    float along = 0.f;
    if (t < a.tokens) {
        const float *dy = static_cast<const float*>(a.dy) + t, *h = static_cast<const float*>(a.h) + t;
#pragma unroll 4
        for (int64_t i = first + l.feature(); i < last; i += l.step()) {
            const float w = a.w ? load_some_of<1>(a.w, a.w_type, i, 1)[0] : 1.f;
            along = fmaf(dy[i * a.lddy] * w, h[i * a.ldh], along);
        }
        along *= a.rstd[t];
    }
    room[threadIdx.x] = along;
    __syncthreads();
    for (unsigned k = 128; k >= l.wide; k /= 2) {
        if (threadIdx.x < k) room[threadIdx.x] += room[threadIdx.x + k];
        __syncthreads();
    }
    if (threadIdx.x < l.wide && t < a.tokens) a.part[blockIdx.y * a.tokens + t] = room[threadIdx.x];
}

__global__ __launch_bounds__(256) void norm_back_columns_kernel(BackArgs a, int64_t features) {
    const Lanes l(a.tokens);
    const int64_t t = (int64_t)blockIdx.x * l.wide + l.token();
    if (t >= a.tokens) return;
    const int64_t first = blockIdx.y * features, last = first + features < a.n ? first + features : a.n;
    float along = 0.f;
    for (uint32_t p = 0; p < a.parts; ++p) along += a.part[p * a.tokens + t];
    along *= a.inverse_n;
    const float rstd = a.rstd[t];
    const float *dy = static_cast<const float*>(a.dy) + t, *h = static_cast<const float*>(a.h) + t;
    const float* dsum = static_cast<const float*>(a.dsum);
    float* dx = static_cast<float*>(a.dx) + t;
#pragma unroll 4
    for (int64_t i = first + l.feature(); i < last; i += l.step()) {
        const float w = a.w ? load_some_of<1>(a.w, a.w_type, i, 1)[0] : 1.f;
        float d = rstd * (dy[i * a.lddy] * w - h[i * a.ldh] * rstd * along);
        if (dsum) d += dsum[i * a.lddsum + t];
        dx[i * a.lddx] = d;
    }
}

// dw: a wave for a feature, its lanes over the tokens.
__global__ __launch_bounds__(256) void norm_back_columns_weight_kernel(BackArgs a) {
    const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (i >= a.n) return;
    const float *dy = static_cast<const float*>(a.dy) + i * a.lddy, *h = static_cast<const float*>(a.h) + i * a.ldh;
    float all = 0.f;
#pragma unroll 4
    for (int64_t t = threadIdx.x & 63; t < a.tokens; t += 64) all = fmaf(dy[t] * h[t], a.rstd[t], all);
    all = wave_total(all);
    if ((threadIdx.x & 63) == 0) a.dw[i] = all;
}

int norm_back_columns(BackArgs a, hipStream_t s) {
    const ColumnShape shape(a.tokens, a.n);
    a.parts = shape.parts;
    Temporary t((size_t)a.tokens * a.parts * 4, s);
    if (t.error) return t.error;
    a.part = t.floats();
    const dim3 grid(shape.blocks, shape.parts);
    if (a.dw) {  // before dx, which may lie where dy or h does
        norm_back_columns_weight_kernel<<<(unsigned)((a.n + 3) / 4), 256, 0, s>>>(a);
        if (int e = (int)hipGetLastError()) return e;
    }
    norm_back_columns_sums_kernel<<<grid, 256, 0, s>>>(a, shape.features);
    if (int e = (int)hipGetLastError()) return e;
    norm_back_columns_kernel<<<grid, 256, 0, s>>>(a, shape.features);
    return (int)hipGetLastError();
}

// dy from columns into rows, a tile of 64 by 64 through LDS.
__global__ __launch_bounds__(256) void norm_back_turn_kernel(const float* from, int64_t ld, int64_t tokens, int64_t n, float* to) {
    __shared__ float tile[64][65];
    const int64_t t0 = (int64_t)blockIdx.x * 64, i0 = (int64_t)blockIdx.y * 64;
    const unsigned lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (unsigned k = 0; k < 16; ++k) {
        const int64_t t = t0 + lane, i = i0 + wave * 16 + k;
        if (t < tokens && i < n) tile[lane][wave * 16 + k] = from[i * ld + t];
    }
    __syncthreads();
#pragma unroll
    for (unsigned k = 0; k < 16; ++k) {
        const int64_t t = t0 + wave * 16 + k, i = i0 + lane;
        if (t < tokens && i < n) to[t * n + i] = tile[wave * 16 + k][lane];
    }
}

// dy in columns, h in rows (a residual stream beside a projection that wants columns): dy is turned first.
template <class TH>
int norm_back_mixed(BackArgs a, hipStream_t s) {
    Temporary t((size_t)a.tokens * a.n * 4, s);
    if (t.error) return t.error;
    norm_back_turn_kernel<<<dim3((unsigned)((a.tokens + 63) / 64), (unsigned)((a.n + 63) / 64)), 256, 0, s>>>(
        static_cast<const float*>(a.dy), a.lddy, a.tokens, a.n, t.floats());
    if (int e = (int)hipGetLastError()) return e;
    a.dy = t.p;
    a.lddy = a.n;
    return norm_back_rows<float, TH>(a, s);
}

template <class TH>
int norm_back_of(const NormBackwardCall& c, const BackArgs& a, hipStream_t s) {
    if (c.dy.order == CER_ORDER_COLUMNS) {
        if (c.h.order == CER_ORDER_ROWS) return norm_back_mixed<TH>(a, s);
        return norm_back_columns(a, s);  // 32 bits
    }
    if (c.dy.type == CER_TYPE_F32) return norm_back_rows<float, TH>(a, s);
    if constexpr (sizeof(TH) != 4) return norm_back_rows<TH, TH>(a, s);
    return (int)hipErrorInvalidValue;
}
}  // namespace

int launch_norm(const NormCall& c, hipStream_t s) {
    NormArgs a{};
    a.x = c.x.data, a.r = c.r.data, a.sum = c.sum.data, a.y = c.y.data;
    a.ldx = c.x.ld, a.ldr = c.r.ld, a.ldsum = c.sum.ld, a.ldy = c.y.ld;
    a.tokens = c.tokens, a.n = c.n;
    a.w = c.weight, a.w_type = c.weight_type;
    a.eps = c.eps, a.inverse_n = (float)(1.0 / (double)c.n);
    a.scale = c.scale, a.rstd = c.rstd;
    if (c.x.type == CER_TYPE_BF16) return norm_to<__bf16>(c, a, s);
    if (c.x.type == CER_TYPE_F16) return norm_to<_Float16>(c, a, s);
    return norm_to<float>(c, a, s);
}

int launch_norm_backward(const NormBackwardCall& c, hipStream_t s) {
    if (c.tokens == 0) {
        if (!c.dweight) return 0;
        norm_back_weight_kernel<<<(unsigned)((c.n + 63) / 64), 1024, 0, s>>>(nullptr, 0, c.n, c.dweight);
        return (int)hipGetLastError();
    }
    BackArgs a{};
    a.dy = c.dy.data, a.h = c.h.data, a.dsum = c.dsum.data, a.dx = c.dx.data;
    a.lddy = c.dy.ld, a.ldh = c.h.ld, a.lddsum = c.dsum.ld, a.lddx = c.dx.ld;
    a.tokens = c.tokens, a.n = c.n;
    a.rstd = c.rstd;
    a.w = c.weight, a.w_type = c.weight_type;
    a.inverse_n = (float)(1.0 / (double)c.n);
    a.dw = c.dweight;
    if (c.h.type == CER_TYPE_BF16) return norm_back_of<__bf16>(c, a, s);
    if (c.h.type == CER_TYPE_F16) return norm_back_of<_Float16>(c, a, s);
    return norm_back_of<float>(c, a, s);
}

}  // namespace cer
