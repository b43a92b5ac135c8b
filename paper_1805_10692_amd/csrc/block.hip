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
// tokens apart there (999 x 2304 fp32 forward 8.6 us, 17 with F in columns, 22 with F and Y).
#include <algorithm>
#include <atomic>
#include <type_traits>

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
        // few registers: what follows a sum is on its way while the sum is formed
        constexpr bool kEarly = kChunks * V <= 8;
        Vec<float, V> w[kEarly ? kChunks : 1];
        const auto behind = [&](int c) {  // what u is multiplied with
            const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
            Vec<float, V> v = a.norm_behind ? numbers_at<V>(a.post, e, a.n) : Vec<float, V>(1.f);
            if (a.gate) v *= load_some<TX, V>(static_cast<const TX*>(a.gate) + t * a.ldgate + e, a.n - e);
            else if (a.gate_vector.p) v *= numbers_at<V>(a.gate_vector, e, a.n);
            return v;
        };
        if (kEarly)
#pragma unroll
            for (int c = 0; c < kChunks; ++c) w[kEarly ? c : 0] = behind(c);
        if (a.norm_behind) {
            float squares = 0.f;
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
#pragma unroll
                for (int j = 0; j < V; ++j) squares = fmaf(u[c][j], u[c][j], squares);
            const float q = rsqrtf(fmaf(block_total(squares, room[turn]), a.inverse_n, a.eps));
            if (a.rstd_post && threadIdx.x == 0) a.rstd_post[t] = q;
#pragma unroll
            for (int c = 0; c < kChunks; ++c) u[c] *= q;
        }
        float squares = 0.f;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
            h[c] = h[c] * a.scale + u[c] * (kEarly ? w[kEarly ? c : 0] : behind(c));
#pragma unroll
            for (int j = 0; j < V; ++j) squares = fmaf(h[c][j], h[c][j], squares);
            store_some<TX, V>(static_cast<TX*>(a.h) + t * a.ldh + e, h[c], a.n - e);
            if (kEarly) w[kEarly ? c : 0] = numbers_at<V>(a.pre, e, a.n);
        }
        const float r = rsqrtf(fmaf(block_total(squares, room[turn + 1]), a.inverse_n, a.eps));
        if (a.rstd_pre && threadIdx.x == 0) a.rstd_pre[t] = r;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * V;
            h[c] *= r;
            h[c] *= kEarly ? w[kEarly ? c : 0] : numbers_at<V>(a.pre, e, a.n);
            store_some<TY, V>(static_cast<TY*>(a.y) + t * a.ldy + e, h[c], a.n - e);
        }
    }
}

// to[j * ldt + i] = from[i * ldf + j], i < rows, j < columns, of one matrix or two: a tile of 64 by 64 through LDS, 16 bytes a lane on both sides.
struct Turn {
    const float* from;
    float* to;
    int64_t ldf, ldt;
};
struct Turns {
    Turn each[2];
    int64_t rows, columns;
};
__global__ __launch_bounds__(256) void block_turn_kernel(Turns w) {
    __shared__ float tile[64][68];  // [j][i]
    const Turn m = w.each[blockIdx.y];
    const unsigned tiles = (unsigned)((w.columns + 63) / 64);
    const int64_t i0 = (int64_t)(blockIdx.x / tiles) * 64, j0 = (int64_t)(blockIdx.x % tiles) * 64;
    const unsigned along = threadIdx.x % 16 * 4, line = threadIdx.x / 16;
    Vec<float, 4> v[4];
#pragma unroll
    for (unsigned k = 0; k < 4; ++k) {
        const int64_t i = i0 + line + 16 * k, j = j0 + along;
        v[k] = i < w.rows ? load_some<float, 4>(m.from + i * m.ldf + j, w.columns - j) : Vec<float, 4>(0.f);
    }
#pragma unroll
    for (unsigned k = 0; k < 4; ++k)
#pragma unroll
        for (unsigned q = 0; q < 4; ++q) tile[along + q][line + 16 * k] = v[k][q];
    __syncthreads();
#pragma unroll
    for (unsigned k = 0; k < 4; ++k) {
        const int64_t j = j0 + line + 16 * k, i = i0 + along;
        if (j < w.columns) store_some<float, 4>(m.to + j * m.ldt + i, *reinterpret_cast<const Vec<float, 4>*>(&tile[line + 16 * k][along]), w.rows - i);
    }
}
int turn(const Turns& w, unsigned many, hipStream_t s) {
    block_turn_kernel<<<dim3((unsigned)((w.rows + 63) / 64 * ((w.columns + 63) / 64)), many), 256, 0, s>>>(w);
    return (int)hipGetLastError();
}

// How many workgroups of a kernel the chip holds at once.  A grid of that size takes tokens in turn and reads the next one while others write: 8192 x 4096 bf16 forward
// 62 us, 67 with a workgroup for each token, 72 - 80 with a grid of two thirds or four thirds of it.
template <auto kernel>
unsigned resident(unsigned threads) {
    static std::atomic<unsigned> known[17];  // by waves
    unsigned v = known[threads / 64].load(std::memory_order_relaxed);
    if (!v) {
        int blocks = 0;
        if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&blocks, kernel, (int)threads, 0) != hipSuccess || blocks < 1) {
            (void)hipGetLastError();
            blocks = 1;
        }
        v = 256u * (unsigned)blocks;
        known[threads / 64].store(v, std::memory_order_relaxed);
    }
    return v;
}

// As few vectors of 16 bytes of the residual stream a thread as the 1024 threads of a workgroup allow, up to 32768 features.  Over 16384 a token does not fit their 128 registers: 112 - 132
// bytes a thread lie in scratch memory forward in 16 bits, 304 in fp32 (1024 tokens: 16384 bf16 39 us, 25088 71, of 27 and 41 for the bytes; 25088 fp32 136 of 82).
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
    const auto launch = [&](auto chunks) {
        constexpr int kChunks = decltype(chunks)::value;
        const unsigned grid = (unsigned)std::min<int64_t>(a.tokens, resident<block_rows_kernel<TX, TF, TY, kChunks>>(w.threads));
        block_rows_kernel<TX, TF, TY, kChunks><<<grid, w.threads, 0, s>>>(a);
    };
    if (w.chunks == 1) launch(std::integral_constant<int, 1>());
    else if (w.chunks == 2) launch(std::integral_constant<int, 2>());
    else if (w.chunks == 4) launch(std::integral_constant<int, 4>());
    else if constexpr (sizeof(TX) == 4) launch(std::integral_constant<int, 8>());
    return (int)hipGetLastError();
}

template <class TX>
int block_of(const BlockCall& c, BlockArgs a, hipStream_t s) {
    const bool f_columns = c.f.order == CER_ORDER_COLUMNS, y_columns = c.y.order == CER_ORDER_COLUMNS;
    const size_t bytes = (size_t)c.tokens * c.n * 4;
    Room room(c.workspace, block_room(c), s);
    if (room.error) return room.error;
    float *f = room.take(f_columns ? bytes : 0), *y = room.take(y_columns ? bytes : 0);
    if (f_columns) {
        a.f = f, a.ldf = c.n;
        if (int e = turn({{{static_cast<const float*>(c.f.data), f, c.f.ld, c.n}, {}}, c.n, c.tokens}, 1, s)) return e;
    }
    if (y_columns) a.y = y, a.ldy = c.n;
    int e;
    if constexpr (sizeof(TX) == 4) {
        e = block_rows<float, float, float>(a, s);
    } else {
        const bool wide_f = c.f.type == CER_TYPE_F32, wide_y = c.y.type == CER_TYPE_F32;
        e = wide_f ? wide_y ? block_rows<TX, float, float>(a, s) : block_rows<TX, float, TX>(a, s)
                   : wide_y ? block_rows<TX, TX, float>(a, s) : block_rows<TX, TX, TX>(a, s);
    }
    if (e || !y_columns) return e;
    return turn({{{y, static_cast<float*>(c.y.data), c.n, c.y.ld}, {}}, c.tokens, c.n}, 1, s);
}

// ---- backward -------------------------------------------------------------------------------------------------------------------
// With K = dy b, B = dsum + r K and W = g a:   d = B - r H c,  so that  n c' = sum d W F = sum B W F - r c sum H W F.  All three sums of a token come from its inputs alone: one
// pass and one barrier.  Each is off by its own rounding only: |c| is at most mean |K H|, by whose rounding d is off in any order of the steps.
// Of the sums over tokens, those of da and of a gate vector are one, sum d F, times g and times a; with a gate for every token da's is sum d g F.
struct BlockBackArgs {
    const void *dy, *h, *f, *gate, *dsum;
    void *dx, *df, *dgate;
    int64_t lddy, ldh, ldf, ldgate, lddsum, lddx, lddf, lddgate;
    int64_t tokens, n;
    const float *rstd_post, *rstd_pre;
    Numbers gate_vector, post, pre;
    float scale, inverse_n;
    float* part[2];  // [parts][n] sums over a part's tokens: dy H, d F (g)
    float* means;    // [tokens][2] c and c', where they have a launch of their own
};

// V features of a token as they are in memory.
template <class TX, class TF, class TD>
struct BackInputs {
    static constexpr int V = 16 / sizeof(TX);
    using F = Vec<float, V>;
    Vec<TD, V> dy_;
    Vec<TX, V> h_, dsum_, gate_;
    Vec<TF, V> f_;
    __device__ __forceinline__ void request(const BlockBackArgs& a, int64_t t, int64_t e) {
        const int64_t left = a.n - e;
        dy_ = load_own<TD, V>(static_cast<const TD*>(a.dy) + t * a.lddy + e, left);
        h_ = load_own<TX, V>(static_cast<const TX*>(a.h) + t * a.ldh + e, left);
        f_ = load_own<TF, V>(static_cast<const TF*>(a.f) + t * a.ldf + e, left);
        if (a.dsum) dsum_ = load_own<TX, V>(static_cast<const TX*>(a.dsum) + t * a.lddsum + e, left);
        if (a.gate) gate_ = load_own<TX, V>(static_cast<const TX*>(a.gate) + t * a.ldgate + e, left);
    }
};
// The same in 32 bits, and what is formed of it: B, H, F, W.
template <class TX, class TF, class TD>
struct BackToken {
    static constexpr int V = 16 / sizeof(TX);
    using F = Vec<float, V>;
    F base, hat, f, w, gate;
    float sums[3];
    // `with_pre`: b; `with_gate`: g a of vectors; both 1 where there are none.  Returns dy H.
    __device__ __forceinline__ F take(const BackInputs<TX, TF, TD>& in, const BlockBackArgs& a, float r, float q, F with_pre, F with_gate) {
        const F dy = __builtin_convertvector(in.dy_, F), k = dy * with_pre;
        hat = __builtin_convertvector(in.h_, F) * r;
        f = __builtin_convertvector(in.f_, F) * q;
        base = k * r;
        if (a.dsum) base += __builtin_convertvector(in.dsum_, F);
        w = with_gate;
        if (a.gate) {
            gate = __builtin_convertvector(in.gate_, F);
            w *= gate;
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
            sums[0] = fmaf(k[j], hat[j], sums[0]);
            sums[1] = fmaf(base[j] * w[j], f[j], sums[1]);
            sums[2] = fmaf(hat[j] * w[j], f[j], sums[2]);
        }
        return dy * hat;
    }
    // Writes what belongs to the token; returns d F (g).
    __device__ __forceinline__ F give(const BlockBackArgs& a, int64_t t, int64_t e, float r, float q, float c, float across, F with_gate, bool write) {
        const int64_t left = a.n - e;
        const F d = base - hat * (r * c);
        F df = d * w;
        if (a.rstd_post) df = (df - f * across) * q;
        F sum = d * f;
        if (write) {
            store_some<TX, V>(static_cast<TX*>(a.dx) + t * a.lddx + e, d * a.scale, left);
            store_some<TF, V>(static_cast<TF*>(a.df) + t * a.lddf + e, df, left);
            if (a.gate && a.dgate) store_some<TX, V>(static_cast<TX*>(a.dgate) + t * a.lddgate + e, sum * with_gate, left);
        }
        if (a.gate) sum *= gate;
        return sum;
    }
};
// c and c' from the three sums over a token's features.
__device__ __forceinline__ void means_of(const BlockBackArgs& a, float s0, float s1, float s2, float r, float* c, float* across) {
    *c = s0 * a.inverse_n;
    *across = (s1 - r * *c * s2) * a.inverse_n;
}

// Three totals over the waves of a token; `room`: 48 floats that nothing else uses until the next barrier but one.
__device__ __forceinline__ void three_totals(float* v, float* room) {
#pragma unroll
    for (int k = 0; k < 3; ++k) v[k] = wave_total(v[k]);
    const unsigned waves = blockDim.x >> 6;
    if (waves == 1) return;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int k = 0; k < 3; ++k) room[k * 16 + (threadIdx.x >> 6)] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        v[k] = room[k * 16];
        for (unsigned w = 1; w < waves; ++w) v[k] += room[k * 16 + w];
    }
}

// Up to 6144 features of 16 bits, 8192 of fp32.  Workgroups take tokens in turn, blockDim.y of them abreast (narrow ones), and hold their share of the sums over tokens for their own features in
// registers: no atomics, whose order would change them, and no second pass.  The next token's inputs are requested before this one's are used; the weights lie in LDS,
// each thread's where only it reads them.
// (1024 threads with eight features each have no registers for the next token's inputs.)  4096 x 4608 bf16: 65 us, 5 of them the totals; with two sums and barriers a
// token, and one a token at a time, 92.  Nine waves of 151 registers leave room for one token on its way beside the one at hand: 8192 x 640 33 us, of 13 for the bytes.
constexpr int kMostThreads = 1024;
template <class TX, class TF, class TD, int kChunks, int kThreads>
__global__ __launch_bounds__(kThreads) void block_back_rows_kernel(BlockBackArgs a) {
    constexpr int V = 16 / sizeof(TX);
    constexpr bool kNext = kThreads < kMostThreads || kChunks == 1;
    using F = Vec<float, V>;
    extern __shared__ __align__(16) float lds[];
    __shared__ float room[2][kThreads / 64][48];
    F *with_pre = reinterpret_cast<F*>(lds), *with_gate = with_pre + kChunks * blockDim.x;
    const auto feature = [&](int c) { return ((int64_t)c * blockDim.x + threadIdx.x) * V; };
    const unsigned group = __builtin_amdgcn_readfirstlane(threadIdx.y), groups = blockDim.y;  // the same for a whole wave: addresses of a token are scalar
    const auto token = [&](int64_t first) { return first + group < a.tokens ? first + group : a.tokens - 1; };  // a group without one repeats the last
    BackInputs<TX, TF, TD> in[kChunks];
    float next_r, next_q;
    const auto request = [&](int64_t t) {
        next_r = a.rstd_pre[t], next_q = a.rstd_post ? a.rstd_post[t] : 1.f;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) in[c].request(a, t, feature(c));
    };
    if (kNext) request(token((int64_t)blockIdx.x * groups));
    if (group == 0)
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            with_pre[c * blockDim.x + threadIdx.x] = numbers_at<V>(a.pre, feature(c), a.n);
            with_gate[c * blockDim.x + threadIdx.x] = numbers_at<V>(a.post, feature(c), a.n) * numbers_at<V>(a.gate_vector, feature(c), a.n);
        }
    if (groups > 1) __syncthreads();
    F sums[2][kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) sums[0][c] = sums[1][c] = 0.f;
    unsigned turn = 0;
    for (int64_t first = (int64_t)blockIdx.x * groups; first < a.tokens; first += (int64_t)gridDim.x * groups, turn ^= 1) {
        const int64_t t = token(first);
        const bool real = first + group < a.tokens;
        if (!kNext) request(t);
        const float r = next_r, q = next_q;
        BackToken<TX, TF, TD> of[kChunks];
        float totals[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
#pragma unroll
            for (int k = 0; k < 3; ++k) of[c].sums[k] = 0.f;
            const F v = of[c].take(in[c], a, r, q, with_pre[c * blockDim.x + threadIdx.x], with_gate[c * blockDim.x + threadIdx.x]);
            if (real) sums[0][c] += v;
#pragma unroll
            for (int k = 0; k < 3; ++k) totals[k] += of[c].sums[k];
        }
        if (kNext) {
            request(token(first + (int64_t)gridDim.x * groups));
            __builtin_amdgcn_sched_barrier(0);
        }
        three_totals(totals, room[turn][group]);
        float c0, across;
        means_of(a, totals[0], totals[1], totals[2], r, &c0, &across);
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const F v = of[c].give(a, t, feature(c), r, q, c0, across, with_gate[c * blockDim.x + threadIdx.x], real);
            if (real) sums[1][c] += v;
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            if (!a.part[k]) continue;
            if (groups > 1) {
                F* joined = reinterpret_cast<F*>(lds);
                __syncthreads();
                joined[group * blockDim.x + threadIdx.x] = sums[k][c];
                __syncthreads();
                for (unsigned g = 1; g < groups && group == 0; ++g) sums[k][c] += joined[g * blockDim.x + threadIdx.x];
            }
            if (group == 0) store_some<float, V>(a.part[k] + blockIdx.x * a.n + feature(c), sums[k][c], a.n - feature(c));
        }
}

// Over that a token and the sums over tokens do not fit the registers of 1024 threads together.  Two launches then, both of which read the inputs: a workgroup for
// the means of a token, and a workgroup for 64 lanes' features of many tokens, which needs no sum over features any more (1024 x 25088 bf16 102 us, fp32 212; in one launch with
// spilled registers, and the sums in another, 231 and 437).
template <class TX, class TF, class TD>
__global__ __launch_bounds__(512) void block_back_means_kernel(BlockBackArgs a) {
    constexpr int V = 16 / sizeof(TX);
    __shared__ float room[2][48];
    unsigned turn = 0;
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x, turn ^= 1) {
        const float r = a.rstd_pre[t], q = a.rstd_post ? a.rstd_post[t] : 1.f;
        BackToken<TX, TF, TD> of;
#pragma unroll
        for (int k = 0; k < 3; ++k) of.sums[k] = 0.f;
#pragma unroll 2
        for (int64_t e = (int64_t)threadIdx.x * V; e < a.n; e += (int64_t)blockDim.x * V) {
            BackInputs<TX, TF, TD> in;
            in.request(a, t, e);
            of.take(in, a, r, q, numbers_at<V>(a.pre, e, a.n), numbers_at<V>(a.post, e, a.n) * numbers_at<V>(a.gate_vector, e, a.n));
        }
        three_totals(of.sums, room[turn]);
        float c, across;
        means_of(a, of.sums[0], of.sums[1], of.sums[2], r, &c, &across);
        if (threadIdx.x == 0) a.means[2 * t] = c, a.means[2 * t + 1] = across;
    }
}
template <class TX, class TF, class TD>
__global__ __launch_bounds__(256) void block_back_strips_kernel(BlockBackArgs a, int64_t tokens_of_part) {
    constexpr int V = 16 / sizeof(TX);
    using F = Vec<float, V>;
    __shared__ F room[4][64];
    const unsigned lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t e = ((int64_t)blockIdx.x * 64 + lane) * V;
    const int64_t first = blockIdx.y * tokens_of_part, last = first + tokens_of_part < a.tokens ? first + tokens_of_part : a.tokens;
    F sums[2] = {F(0.f), F(0.f)};
    if (e < a.n) {
        const F with_pre = numbers_at<V>(a.pre, e, a.n), with_gate = numbers_at<V>(a.post, e, a.n) * numbers_at<V>(a.gate_vector, e, a.n);
#pragma unroll 2
        for (int64_t t = first + wave; t < last; t += 4) {
            BackInputs<TX, TF, TD> in;
            in.request(a, t, e);
            const float r = a.rstd_pre[t], q = a.rstd_post ? a.rstd_post[t] : 1.f;
            BackToken<TX, TF, TD> of;
            sums[0] += of.take(in, a, r, q, with_pre, with_gate);
            sums[1] += of.give(a, t, e, r, q, a.means[2 * t], a.means[2 * t + 1], with_gate, true);
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if (!a.part[k]) continue;
        room[wave][lane] = sums[k];
        __syncthreads();
        if (wave == 0 && e < a.n) store_some<float, V>(a.part[k] + blockIdx.y * a.n + e, room[0][lane] + room[1][lane] + (room[2][lane] + room[3][lane]), a.n - e);
        __syncthreads();
    }
}

struct Totals {
    const float* part[2];
    float *pre, *post, *gate;  // wanted where not null
    Numbers with_gate, with_post;
};
// The parts added up in their order.  Workgroup (b, k): 64 features of sum k, 16 lanes of four features by 64 rows of parts.
__global__ __launch_bounds__(1024) void block_back_totals_kernel(Totals w, uint32_t parts, int64_t n) {
    __shared__ Vec<float, 4> room[64][17];
    const bool second = blockIdx.y == 1;
    if (second ? !w.post && !w.gate : !w.pre) return;
    const float* part = w.part[second];
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
    if (row != 0 || i >= n) return;
    all = room[0][lane];
    if (!second) {
        store_some<float, 4>(w.pre + i, all, n - i);
        return;
    }
    // without tokens nothing is multiplied: an infinite weight is no reason for a NaN
    if (w.post) store_some<float, 4>(w.post + i, parts ? all * numbers_at<4>(w.with_gate, i, n) : all, n - i);
    if (w.gate) store_some<float, 4>(w.gate + i, parts ? all * numbers_at<4>(w.with_post, i, n) : all, n - i);
}

constexpr unsigned kFewThreads = 768;  // up to here a thread has 168 registers
// How a backward call goes about its tokens, and its temporaries.
struct BackShape {
    Threads w;
    bool inside, sums[2];
    unsigned groups, parts;
    int64_t tokens_of_part;
    size_t turned, room, means;
    BackShape(const BlockBackwardCall& c) : w(c.n, c.h.type == CER_TYPE_F32 ? 4 : 8) {
        // 1024 threads with eight features each spill: 2048 x 8192 bf16 80 us here, 72 in strips; with four or eight of fp32 they do not
        // (2000 x 4608 57 us, 81 in strips; 4096 x 6144 127 and 212; 2000 x 7680 88 and 110).
        inside = c.n <= (c.h.type == CER_TYPE_F32 ? 8192 : 6144);
        sums[0] = c.dpre_weight != nullptr, sums[1] = c.dpost_weight || c.dgate_vector;
        groups = inside && w.chunks == 1 && w.threads <= kFewThreads ? (unsigned)std::max<int64_t>(1, std::min<int64_t>(kFewThreads / w.threads, (c.tokens + 255) / 256)) : 1;
        tokens_of_part = std::max<int64_t>(1, (c.tokens + 63) / 64);
        parts = (unsigned)(inside ? std::min<int64_t>((c.tokens + groups - 1) / groups, 256) : (c.tokens + tokens_of_part - 1) / tokens_of_part);
        turned = (size_t)c.tokens * c.n * 4;
        room = (size_t)(sums[0] + sums[1]) * parts * c.n * 4;
        means = inside ? 0 : (size_t)c.tokens * 8;
    }
    static bool columns(const cer_tokens_t& m) { return m.data && m.order == CER_ORDER_COLUMNS; }
    int64_t bytes(const BlockBackwardCall& c) const {
        return (int64_t)(Room::rounded(turned) * ((columns(c.dy) ? 1 : 0) + (columns(c.f) ? 2 : 0)) + Room::rounded(room) + Room::rounded(means));
    }
};
template <class TX, class TF, class TD>
int block_back_rows(BlockBackArgs a, Totals totals, const BackShape& shape, Room& temporaries, hipStream_t s) {
    constexpr int V = 16 / sizeof(TX);
    const Threads& w = shape.w;
    const unsigned groups = shape.groups, parts = shape.parts;
    float* room = temporaries.take(shape.room);
    for (int k = 0, at = 0; k < 2; ++k) totals.part[k] = a.part[k] = shape.sums[k] ? room + (size_t)at++ * parts * a.n : nullptr;
    a.means = temporaries.take(shape.means);
    if (shape.inside) {
        const dim3 block(w.threads, groups);
        const auto bytes = [&](int chunks) { return (size_t)V * 4 * w.threads * std::max<size_t>(2 * chunks, groups > 1 ? groups : 0); };
        if (w.threads <= kFewThreads && w.chunks == 1) block_back_rows_kernel<TX, TF, TD, 1, kFewThreads><<<parts, block, bytes(1), s>>>(a);
        else if constexpr (V == 4) {
            if (w.chunks == 1) block_back_rows_kernel<TX, TF, TD, 1, kMostThreads><<<parts, block, bytes(1), s>>>(a);
            else block_back_rows_kernel<TX, TF, TD, 2, kMostThreads><<<parts, block, bytes(2), s>>>(a);
        } else {
            return (int)hipErrorInvalidValue;
        }
    } else {
        block_back_means_kernel<TX, TF, TD><<<(unsigned)std::min<int64_t>(a.tokens, 1 << 20), 512, 0, s>>>(a);
        if (int e = (int)hipGetLastError()) return e;
        block_back_strips_kernel<TX, TF, TD><<<dim3((unsigned)((a.n + 64 * V - 1) / (64 * V)), parts), 256, 0, s>>>(a, shape.tokens_of_part);
    }
    if (int e = (int)hipGetLastError()) return e;
    if (!shape.sums[0] && !shape.sums[1]) return 0;
    block_back_totals_kernel<<<dim3((unsigned)((a.n + 63) / 64), 2), 1024, 0, s>>>(totals, parts, a.n);
    return (int)hipGetLastError();
}

template <class TX>
int block_back_of(const BlockBackwardCall& c, BlockBackArgs a, const Totals& outs, hipStream_t s) {
    const bool dy_columns = c.dy.order == CER_ORDER_COLUMNS, f_columns = c.f.order == CER_ORDER_COLUMNS;
    const BackShape shape(c);
    Room room(c.workspace, shape.bytes(c), s);
    if (room.error) return room.error;
    float *dy = room.take(dy_columns ? shape.turned : 0), *f = room.take(f_columns ? shape.turned : 0), *df = room.take(f_columns ? shape.turned : 0);
    Turns w{{}, c.n, c.tokens};
    unsigned many = 0;
    if (dy_columns) {
        a.dy = dy, a.lddy = c.n;
        w.each[many++] = {static_cast<const float*>(c.dy.data), dy, c.dy.ld, c.n};
    }
    if (f_columns) {
        a.f = f, a.df = df, a.ldf = a.lddf = c.n;
        w.each[many++] = {static_cast<const float*>(c.f.data), f, c.f.ld, c.n};
    }
    if (many)
        if (int e = turn(w, many, s)) return e;
    int e;
    if constexpr (sizeof(TX) == 4) {
        e = block_back_rows<float, float, float>(a, outs, shape, room, s);
    } else {
        const bool wide_f = c.f.type == CER_TYPE_F32, wide_dy = c.dy.type == CER_TYPE_F32;
        e = wide_f ? wide_dy ? block_back_rows<TX, float, float>(a, outs, shape, room, s) : block_back_rows<TX, float, TX>(a, outs, shape, room, s)
                   : wide_dy ? block_back_rows<TX, TX, float>(a, outs, shape, room, s) : block_back_rows<TX, TX, TX>(a, outs, shape, room, s);
    }
    if (e || !f_columns) return e;
    return turn({{{df, static_cast<float*>(c.df.data), c.n, c.df.ld}, {}}, c.tokens, c.n}, 1, s);
}
}  // namespace

int64_t block_room(const BlockCall& c) {
    return (int64_t)Room::rounded((size_t)c.tokens * c.n * 4) * ((c.f.order == CER_ORDER_COLUMNS) + (c.y.order == CER_ORDER_COLUMNS));
}
int64_t block_backward_room(const BlockBackwardCall& c) { return c.tokens ? BackShape(c).bytes(c) : 0; }
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
    const Totals outs{{nullptr, nullptr}, c.dpre_weight, c.dpost_weight, c.dgate_vector, {c.gate_vector, c.gate_vector_type}, {c.post_weight, c.post_weight_type}};
    if (c.tokens == 0) {
        if (!c.dpre_weight && !c.dpost_weight && !c.dgate_vector) return 0;
        block_back_totals_kernel<<<dim3((unsigned)((c.n + 63) / 64), 2), 1024, 0, s>>>(outs, 0, c.n);
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
