// The output side of a block: the norm behind it, its gate, the scaled residual stream, the norm in front of the next block, and the gradient.
//
// Forward, token t, feature i:   u = f q a_i;   h = s x + g u;   y = h r b_i,   with q = 1 / sqrt(mean f^2 + eps) (1 without the norm behind the block),
// r = 1 / sqrt(mean h^2 + eps), a and b the norms' weights, g the gate (1, one number per feature, or one per token and feature).
// Backward:   d = dsum + r (k - H c), k = dy b, H = h r, c = mean(k H);   dx = s d;   dg = d u;   du = d g;
//             df = q (e - F c'), e = du a, F = f q, c' = mean(e F);   db = sum_t dy H;   da = sum_t du F;   dg of a vector = sum_t d u.
// Some 10 (25) operations per element: the bytes bound both.
//
// A workgroup takes a token and keeps it in registers through both sums, so that every input is read once and every output written once.
// Activations in columns (the order of cer_matmul's X and Y) are turned through LDS, before and behind: a token's features lie a whole line of
// tokens apart there.
#include <algorithm>

#include "operators.hpp"

namespace cer {
namespace {

// A vector of n numbers of one of three types, or nothing: 1.
struct Numbers {
    const void* p;
    int32_t type;
};
template <int V>
__device__ __forceinline__ Vec<float, V> numbers_at(const Numbers& w, int64_t e, int64_t n) {
    return w.p ? load_some_of<V>(w.p, w.type, e, n - e) : Vec<float, V>(1.f);
}

struct BlockArgs {
    const void *x, *f, *gate;
    void *h, *y;
    int64_t ldx, ldf, ldgate, ldh, ldy;
    int64_t tokens, n;
    Numbers gate_vector, post, pre;
    float scale, eps, inverse_n;
    bool norm_behind;
    float *rstd_post, *rstd_pre;
};

template <class TX, class TF, class TY, int kChunks>
__global__ __launch_bounds__(1024) void block_rows_kernel(BlockArgs a) {
    constexpr int V = 16 / sizeof(TX);
    __shared__ float room[4][16];
    unsigned turn = 0;
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x, turn ^= 2) {
        const TF* f = static_cast<const TF*>(a.f) + t * a.ldf;
        const TX* x = static_cast<const TX*>(a.x) + t * a.ldx;
        Vec<float, V> u[kChunks], h[kChunks];
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
            u[c] = load_some<TF, V>(f + e, a.n - e);
            h[c] = load_some<TX, V>(x + e, a.n - e);
        }
        if (a.norm_behind) {
            float squares = 0.f;
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
#pragma unroll
                for (int j = 0; j < V; ++j) squares = fmaf(u[c][j], u[c][j], squares);
            const float q = rsqrtf(fmaf(block_total(squares, room[turn]), a.inverse_n, a.eps));
            if (a.rstd_post && threadIdx.x == 0) a.rstd_post[t] = q;
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
                u[c] *= q;
                if (a.post.p) u[c] *= numbers_at<V>(a.post, e, a.n);
            }
        }
        float squares = 0.f;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
            if (a.gate) u[c] *= load_some<TX, V>(static_cast<const TX*>(a.gate) + t * a.ldgate + e, a.n - e);
            else if (a.gate_vector.p) u[c] *= numbers_at<V>(a.gate_vector, e, a.n);
            h[c] = h[c] * a.scale + u[c];
#pragma unroll
            for (int j = 0; j < V; ++j) squares = fmaf(h[c][j], h[c][j], squares);
            store_some<TX, V>(static_cast<TX*>(a.h) + t * a.ldh + e, h[c], a.n - e);
        }
        const float r = rsqrtf(fmaf(block_total(squares, room[turn + 1]), a.inverse_n, a.eps));
        if (a.rstd_pre && threadIdx.x == 0) a.rstd_pre[t] = r;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
            h[c] *= r;
            if (a.pre.p) h[c] *= numbers_at<V>(a.pre, e, a.n);
            store_some<TY, V>(static_cast<TY*>(a.y) + t * a.ldy + e, h[c], a.n - e);
        }
    }
}

// to[j * ldt + i] = from[i * ldf + j], i < rows, j < columns: a tile of 64 by 64 through LDS.
__global__ __launch_bounds__(256) void block_turn_kernel(const float* from, int64_t ldf, int64_t rows, int64_t columns, float* to, int64_t ldt) {
    __shared__ float tile[64][65];
    const unsigned tiles = (unsigned)((columns + 63) / 64);
    const int64_t i0 = (int64_t)(blockIdx.x / tiles) * 64, j0 = (int64_t)(blockIdx.x % tiles) * 64;
    const unsigned lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (unsigned k = 0; k < 16; ++k) {
        const int64_t i = i0 + wave * 16 + k, j = j0 + lane;
        if (i < rows && j < columns) tile[lane][wave * 16 + k] = from[i * ldf + j];
    }
    __syncthreads();
#pragma unroll
    for (unsigned k = 0; k < 16; ++k) {
        const int64_t j = j0 + wave * 16 + k, i = i0 + lane;
        if (i < rows && j < columns) to[j * ldt + i] = tile[wave * 16 + k][lane];
    }
}
int turn(const float* from, int64_t ldf, int64_t rows, int64_t columns, float* to, int64_t ldt, hipStream_t s) {
    block_turn_kernel<<<(unsigned)((rows + 63) / 64 * ((columns + 63) / 64)), 256, 0, s>>>(from, ldf, rows, columns, to, ldt);
    return (int)hipGetLastError();
}

// As few vectors of 16 bytes of the residual stream a thread as the 1024 threads of a workgroup allow, up to 32768 features.
struct Threads {
    int chunks;
    unsigned threads;
    Threads(int64_t n, int vector) {
        const int64_t vectors = (n + vector - 1) / vector;
        chunks = 1;
        while (vectors > (int64_t)1024 * chunks) chunks *= 2;
        threads = (unsigned)(((vectors + chunks - 1) / chunks + 63) / 64 * 64);
    }
};

template <class TX, class TF, class TY>
int block_rows(const BlockArgs& a, hipStream_t s) {
    const Threads w(a.n, 16 / sizeof(TX));
    const unsigned grid = (unsigned)std::min<int64_t>(a.tokens, 1 << 20);
    if (w.chunks == 1) block_rows_kernel<TX, TF, TY, 1><<<grid, w.threads, 0, s>>>(a);
    else if (w.chunks == 2) block_rows_kernel<TX, TF, TY, 2><<<grid, w.threads, 0, s>>>(a);
    else if (w.chunks == 4) block_rows_kernel<TX, TF, TY, 4><<<grid, w.threads, 0, s>>>(a);
    else if constexpr (sizeof(TX) == 4) block_rows_kernel<TX, TF, TY, 8><<<grid, w.threads, 0, s>>>(a);
    return (int)hipGetLastError();
}

template <class TX>
int block_of(const BlockCall& c, BlockArgs a, hipStream_t s) {
    const bool f_columns = c.f.order == CER_ORDER_COLUMNS, y_columns = c.y.order == CER_ORDER_COLUMNS;
    const size_t room = (size_t)c.tokens * c.n * 4;
    Temporary f(f_columns ? room : 0, s), y(y_columns ? room : 0, s);
    if (f.error || y.error) return f.error ? f.error : y.error;
    if (f_columns) {
        a.f = f.p, a.ldf = c.n;
        if (int e = turn(static_cast<const float*>(c.f.data), c.f.ld, c.n, c.tokens, f.floats(), c.n, s)) return e;
    }
    if (y_columns) a.y = y.p, a.ldy = c.n;
    int e;
    if constexpr (sizeof(TX) == 4) {
        e = block_rows<float, float, float>(a, s);
    } else {
        const bool wide_f = c.f.type == CER_TYPE_F32, wide_y = c.y.type == CER_TYPE_F32;
        e = wide_f ? wide_y ? block_rows<TX, float, float>(a, s) : block_rows<TX, float, TX>(a, s)
                   : wide_y ? block_rows<TX, TX, float>(a, s) : block_rows<TX, TX, TX>(a, s);
    }
    if (e || !y_columns) return e;
    return turn(y.floats(), c.n, c.tokens, c.n, static_cast<float*>(c.y.data), c.y.ld, s);
}

// ---- backward -------------------------------------------------------------------------------------------------------------------
struct BlockBackArgs {
    const void *dy, *h, *f, *gate, *dsum;
    void *dx, *df, *dgate;
    int64_t lddy, ldh, ldf, ldgate, lddsum, lddx, lddf, lddgate;
    int64_t tokens, n;
    const float *rstd_post, *rstd_pre;
    Numbers gate_vector, post, pre;
    float scale, inverse_n;
    float* part[3];  // [workgroups][n] sums over the workgroup's tokens: of dpre, dpost, dgate
    float* along;    // [tokens] c, where the sums have a launch of their own
    uint32_t parts;
};

// One token's share of the three sums, from what both kernels have in registers.
enum { kPre = 0, kPost = 1, kGate = 2 };

// kSums: a workgroup takes tokens blockIdx.x, + gridDim.x, ... and holds its share of the sums over tokens for its own features in registers: no
// atomics, whose order would change them, and no second pass over the inputs.
template <class TX, class TF, class TD, int kChunks, bool kSums>
__global__ __launch_bounds__(1024) void block_back_rows_kernel(BlockBackArgs a) {
    constexpr int V = 16 / sizeof(TX);
    __shared__ float room[4][16];
    unsigned turn = 0;
    Vec<float, V> sums[3][kSums ? kChunks : 1];
#pragma unroll
    for (int k = 0; k < 3; ++k)
#pragma unroll
        for (int c = 0; c < (kSums ? kChunks : 1); ++c) sums[k][c] = 0.f;
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x, turn ^= 2) {
        const float r = a.rstd_pre[t], q = a.rstd_post ? a.rstd_post[t] : 1.f;
        Vec<float, V> d[kChunks], hat[kChunks], f[kChunks];
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
            d[c] = load_some<TD, V>(static_cast<const TD*>(a.dy) + t * a.lddy + e, a.n - e);
            hat[c] = load_some<TX, V>(static_cast<const TX*>(a.h) + t * a.ldh + e, a.n - e);
            f[c] = load_some<TF, V>(static_cast<const TF*>(a.f) + t * a.ldf + e, a.n - e);
        }
        float along = 0.f;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
            hat[c] *= r;
            f[c] *= q;
            if constexpr (kSums) sums[kPre][c] += d[c] * hat[c];
            if (a.pre.p) d[c] *= numbers_at<V>(a.pre, e, a.n);
#pragma unroll
            for (int j = 0; j < V; ++j) along = fmaf(d[c][j], hat[c][j], along);
        }
        along = block_total(along, room[turn]) * a.inverse_n;
        if (!kSums && a.along && threadIdx.x == 0) a.along[t] = along;
        float across = 0.f;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
            d[c] = (d[c] - hat[c] * along) * r;
            if (a.dsum) d[c] += load_some<TX, V>(static_cast<const TX*>(a.dsum) + t * a.lddsum + e, a.n - e);
            store_some<TX, V>(static_cast<TX*>(a.dx) + t * a.lddx + e, d[c] * a.scale, a.n - e);
            const Vec<float, V> w = numbers_at<V>(a.post, e, a.n);
            if (a.gate) {
                const Vec<float, V> g = load_some<TX, V>(static_cast<const TX*>(a.gate) + t * a.ldgate + e, a.n - e);
                if (a.dgate) store_some<TX, V>(static_cast<TX*>(a.dgate) + t * a.lddgate + e, d[c] * f[c] * w, a.n - e);
                d[c] *= g;
            } else if (a.gate_vector.p) {
                if constexpr (kSums) sums[kGate][c] += d[c] * f[c] * w;
                d[c] *= numbers_at<V>(a.gate_vector, e, a.n);
            }
            if constexpr (kSums) sums[kPost][c] += d[c] * f[c];
            d[c] *= w;
#pragma unroll
            for (int j = 0; j < V; ++j) across = fmaf(d[c][j], f[c][j], across);
        }
        if (a.rstd_post) across = block_total(across, room[turn + 1]) * a.inverse_n;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
            if (a.rstd_post) d[c] = (d[c] - f[c] * across) * q;
            store_some<TF, V>(static_cast<TF*>(a.df) + t * a.lddf + e, d[c], a.n - e);
        }
    }
    if constexpr (kSums) {
#pragma unroll
        for (int k = 0; k < 3; ++k)
            if (a.part[k])
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
                    store_some<float, V>(a.part[k] + blockIdx.x * a.n + e, sums[k][c], a.n - e);
                }
    }
}

// Over 8192 features three sums, beside three copies of a token, do not fit the registers of 1024 threads: they are formed here from the inputs again and
// c of each token.  A workgroup: 64 lanes of V features by 4 waves, each of every fourth token of the workgroup's part.
template <class TX, class TF, class TD>
__global__ __launch_bounds__(256) void block_back_sums_kernel(BlockBackArgs a, int64_t tokens_of_part) {
    constexpr int V = 16 / sizeof(TX);
    __shared__ Vec<float, V> room[4][64];
    const unsigned lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t e = ((int64_t)blockIdx.x * 64 + lane) * V;
    const int64_t first = blockIdx.y * tokens_of_part, last = first + tokens_of_part < a.tokens ? first + tokens_of_part : a.tokens;
    Vec<float, V> sums[3] = {Vec<float, V>(0.f), Vec<float, V>(0.f), Vec<float, V>(0.f)};
    if (e < a.n) {
        const Vec<float, V> pre = numbers_at<V>(a.pre, e, a.n), post = numbers_at<V>(a.post, e, a.n), gate = numbers_at<V>(a.gate_vector, e, a.n);
        for (int64_t t = first + wave; t < last; t += 4) {
            const float r = a.rstd_pre[t], q = a.rstd_post ? a.rstd_post[t] : 1.f;
            const Vec<float, V> dy = load_some<TD, V>(static_cast<const TD*>(a.dy) + t * a.lddy + e, a.n - e);
            const Vec<float, V> hat = load_some<TX, V>(static_cast<const TX*>(a.h) + t * a.ldh + e, a.n - e) * r;
            const Vec<float, V> f = load_some<TF, V>(static_cast<const TF*>(a.f) + t * a.ldf + e, a.n - e) * q;
            sums[kPre] += dy * hat;
            Vec<float, V> d = (dy * pre - hat * a.along[t]) * r;
            if (a.dsum) d += load_some<TX, V>(static_cast<const TX*>(a.dsum) + t * a.lddsum + e, a.n - e);
            sums[kGate] += d * f * post;
            d *= a.gate ? load_some<TX, V>(static_cast<const TX*>(a.gate) + t * a.ldgate + e, a.n - e) : gate;
            sums[kPost] += d * f;
        }
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        if (!a.part[k]) continue;
        room[wave][lane] = sums[k];
        __syncthreads();
        if (wave == 0 && e < a.n) store_some<float, V>(a.part[k] + blockIdx.y * a.n + e, room[0][lane] + room[1][lane] + (room[2][lane] + room[3][lane]), a.n - e);
        __syncthreads();
    }
}

struct ThreeSums {
    const float* part[3];
    float* out[3];
};
// The parts added up in their order.  Workgroup (b, k): 64 features of sum k, 16 lanes of four features by 64 rows of parts.
__global__ __launch_bounds__(1024) void block_back_totals_kernel(ThreeSums w, uint32_t parts, int64_t n) {
    __shared__ Vec<float, 4> room[64][17];
    const float* part = w.part[blockIdx.y];
    float* out = w.out[blockIdx.y];
    if (!out) return;
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
    if (row == 0 && i < n) store_some<float, 4>(out + i, room[0][lane], n - i);
}

template <class TX, class TF, class TD, int kChunks, bool kSums>
int block_back_launch(const BlockBackArgs& a, unsigned threads, hipStream_t s) {
    const unsigned grid = kSums ? a.parts : (unsigned)std::min<int64_t>(a.tokens, 1 << 20);
    block_back_rows_kernel<TX, TF, TD, kChunks, kSums><<<grid, threads, 0, s>>>(a);
    return (int)hipGetLastError();
}

template <class TX, class TF, class TD>
int block_back_rows(BlockBackArgs a, const ThreeSums& outs, hipStream_t s) {
    constexpr int V = 16 / sizeof(TX);
    const Threads w(a.n, V);
    const int wanted = (outs.out[0] != nullptr) + (outs.out[1] != nullptr) + (outs.out[2] != nullptr);
    const bool inside = a.n <= 8192;  // eight features a thread
    const int64_t tokens_of_part = (a.tokens + 63) / 64;
    a.parts = (unsigned)(inside ? std::min<int64_t>(a.tokens, 512) : (a.tokens + tokens_of_part - 1) / tokens_of_part);
    Temporary parts((size_t)wanted * a.parts * a.n * 4, s), along(wanted && !inside ? (size_t)a.tokens * 4 : 0, s);
    if (parts.error || along.error) return parts.error ? parts.error : along.error;
    ThreeSums sums = outs;
    for (int k = 0, at = 0; k < 3; ++k) {
        a.part[k] = outs.out[k] ? parts.floats() + (size_t)at++ * a.parts * a.n : nullptr;
        sums.part[k] = a.part[k];
    }
    a.along = along.floats();
    int e;
    if (inside) {
        if (w.chunks == 1) e = block_back_launch<TX, TF, TD, 1, true>(a, w.threads, s);
        else if constexpr (V == 4) e = block_back_launch<TX, TF, TD, 2, true>(a, w.threads, s);
        else return (int)hipErrorInvalidValue;
    } else {
        if (w.chunks == 2) e = block_back_launch<TX, TF, TD, 2, false>(a, w.threads, s);
        else if (w.chunks == 4) e = block_back_launch<TX, TF, TD, 4, false>(a, w.threads, s);
        else if constexpr (V == 4) e = block_back_launch<TX, TF, TD, 8, false>(a, w.threads, s);
        else return (int)hipErrorInvalidValue;
        if (!e && wanted) {
            block_back_sums_kernel<TX, TF, TD><<<dim3((unsigned)((a.n + 64 * V - 1) / (64 * V)), a.parts), 256, 0, s>>>(a, tokens_of_part);
            e = (int)hipGetLastError();
        }
    }
    if (e || !wanted) return e;
    block_back_totals_kernel<<<dim3((unsigned)((a.n + 63) / 64), 3), 1024, 0, s>>>(sums, a.parts, a.n);
    return (int)hipGetLastError();
}

template <class TX>
int block_back_of(const BlockBackwardCall& c, BlockBackArgs a, const ThreeSums& outs, hipStream_t s) {
    const bool dy_columns = c.dy.order == CER_ORDER_COLUMNS, f_columns = c.f.order == CER_ORDER_COLUMNS;
    const size_t room = (size_t)c.tokens * c.n * 4;
    Temporary dy(dy_columns ? room : 0, s), f(f_columns ? room : 0, s), df(f_columns ? room : 0, s);
    if (dy.error || f.error || df.error) return dy.error ? dy.error : f.error ? f.error : df.error;
    if (dy_columns) {
        a.dy = dy.p, a.lddy = c.n;
        if (int e = turn(static_cast<const float*>(c.dy.data), c.dy.ld, c.n, c.tokens, dy.floats(), c.n, s)) return e;
    }
    if (f_columns) {
        a.f = f.p, a.df = df.p, a.ldf = a.lddf = c.n;
        if (int e = turn(static_cast<const float*>(c.f.data), c.f.ld, c.n, c.tokens, f.floats(), c.n, s)) return e;
    }
    int e;
    if constexpr (sizeof(TX) == 4) {
        e = block_back_rows<float, float, float>(a, outs, s);
    } else {
        const bool wide_f = c.f.type == CER_TYPE_F32, wide_dy = c.dy.type == CER_TYPE_F32;
        e = wide_f ? wide_dy ? block_back_rows<TX, float, float>(a, outs, s) : block_back_rows<TX, float, TX>(a, outs, s)
                   : wide_dy ? block_back_rows<TX, TX, float>(a, outs, s) : block_back_rows<TX, TX, TX>(a, outs, s);
    }
    if (e || !f_columns) return e;
    return turn(df.floats(), c.n, c.tokens, c.n, static_cast<float*>(c.df.data), c.df.ld, s);
}
}  // namespace

int launch_block_norm(const BlockCall& c, hipStream_t s) {
    BlockArgs a{};
    a.x = c.x.data, a.f = c.f.data, a.gate = c.gate.data, a.h = c.h.data, a.y = c.y.data;
    a.ldx = c.x.ld, a.ldf = c.f.ld, a.ldgate = c.gate.ld, a.ldh = c.h.ld, a.ldy = c.y.ld;
    a.tokens = c.tokens, a.n = c.n;
    a.gate_vector = {c.gate_vector, c.gate_vector_type}, a.post = {c.post_weight, c.post_weight_type}, a.pre = {c.pre_weight, c.pre_weight_type};
    a.scale = c.scale, a.eps = c.eps, a.inverse_n = (float)(1.0 / (double)c.n);
    a.norm_behind = c.post;
    a.rstd_post = c.rstd_post, a.rstd_pre = c.rstd_pre;
    if (c.x.type == CER_TYPE_BF16) return block_of<__bf16>(c, a, s);
    if (c.x.type == CER_TYPE_F16) return block_of<_Float16>(c, a, s);
    return block_of<float>(c, a, s);
}

int launch_block_norm_backward(const BlockBackwardCall& c, hipStream_t s) {
    const ThreeSums outs{{nullptr, nullptr, nullptr}, {c.dpre_weight, c.dpost_weight, c.dgate_vector}};
    if (c.tokens == 0) {
        if (!c.dpre_weight && !c.dpost_weight && !c.dgate_vector) return 0;
        block_back_totals_kernel<<<dim3((unsigned)((c.n + 63) / 64), 3), 1024, 0, s>>>(outs, 0, c.n);
        return (int)hipGetLastError();
    }
    BlockBackArgs a{};
    a.dy = c.dy.data, a.h = c.h.data, a.f = c.f.data, a.gate = c.gate.data, a.dsum = c.dsum.data, a.dx = c.dx.data, a.df = c.df.data, a.dgate = c.dgate.data;
    a.lddy = c.dy.ld, a.ldh = c.h.ld, a.ldf = c.f.ld, a.ldgate = c.gate.ld, a.lddsum = c.dsum.ld, a.lddx = c.dx.ld, a.lddf = c.df.ld, a.lddgate = c.dgate.ld;
    a.tokens = c.tokens, a.n = c.n;
    a.rstd_post = c.rstd_post, a.rstd_pre = c.rstd_pre;
    a.gate_vector = {c.gate_vector, c.gate_vector_type}, a.post = {c.post_weight, c.post_weight_type}, a.pre = {c.pre_weight, c.pre_weight_type};
    a.scale = c.scale, a.inverse_n = (float)(1.0 / (double)c.n);
    if (c.h.type == CER_TYPE_BF16) return block_back_of<__bf16>(c, a, outs, s);
    if (c.h.type == CER_TYPE_F16) return block_back_of<_Float16>(c, a, outs, s);
    return block_back_of<float>(c, a, outs, s);
}

}  // namespace cer
