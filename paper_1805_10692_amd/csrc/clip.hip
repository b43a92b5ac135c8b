// The global norm over many gradient tensors, and clipping to it.
//
//   norm = sqrt(sum over all tensors, all elements, of g^2);   c = min(1, limit / (norm + 1e-6));   out = c g.
//
// The factor is known when every gradient has been read, so that they are read twice: two launches, a read and a read and a write per
// element, bytes bound.  All tensors are cut into chunks of kChunk elements; a workgroup takes chunks blockIdx.x, + gridDim.x, ... and
// finds a chunk's tensor in the table that comes with the launch's arguments (a table in device memory would have to be copied there
// at every call: gradients have other addresses in every step).  Squares are added in 64 bits: their conversion costs little beside
// the reads, and neither large gradients nor many of them spoil the sum.  A workgroup's sum goes to a place of its own and every
// workgroup of the second launch adds up all of them in the same order, so that the result does not depend on the order in which
// workgroups run.
//
// Measured: 48 M numbers in 56 tensors, fp32, 97.5 us (reads 35.7 us, 5.4 TB/s; read and write 61.8 us, 6.2 TB/s: a good part of what the first launch read
// is still in the memory-side cache); six tensors of 70 thousand together 9.2 us, the two launches.
#include <algorithm>

#include "operators.hpp"

namespace cer {
namespace {

constexpr int kEntries = 120, kThreads = 256, kPartsPerLaunch = 2048;
constexpr int64_t kChunk = 8192;

struct ClipTable {  // within the 4 KiB of arguments that a launch may have
    struct {
        const void* grad;
        void* out;
        int64_t numbers;
        uint32_t first;  // chunk
        int32_t type;
    } at[kEntries];
    uint32_t count, chunks;
};

__device__ __forceinline__ uint32_t tensor_of(const ClipTable& t, uint32_t chunk) {
    uint32_t lo = 0, hi = t.count;  // the last entry whose first chunk is not after this one
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (t.at[mid].first <= chunk) lo = mid;
        else hi = mid;
    }
    return lo;
}

template <class T>
__device__ __forceinline__ double chunk_squares(const T* g, int64_t left) {
    constexpr int V = 16 / sizeof(T);
    double sum = 0;
    constexpr int kSteps = kChunk / (kThreads * V);
    if (left >= kChunk) {
        Vec<float, V> v[kSteps];
#pragma unroll
        for (int s = 0; s < kSteps; ++s) v[s] = load_f32<T, V>(g + (s * kThreads + threadIdx.x) * V);
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int j = 0; j < V; ++j) sum = fma((double)v[s][j], (double)v[s][j], sum);
        return sum;
    }
    for (int64_t e = threadIdx.x * V; e < left; e += kThreads * V) {
        const Vec<float, V> v = load_some<T, V>(g + e, left - e);
#pragma unroll
        for (int j = 0; j < V; ++j) sum = fma((double)v[j], (double)v[j], sum);
    }
    return sum;
}

__device__ __forceinline__ double block_total_f64(double v, double* room) {
#pragma unroll
    for (int k = 32; k; k >>= 1) v += __shfl_xor(v, k);
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
    __syncthreads();
    double all = room[0];
    for (int k = 1; k < kThreads / 64; ++k) all += room[k];
    return all;
}

__global__ __launch_bounds__(kThreads) void clip_squares_kernel(ClipTable t, double* part) {
    __shared__ double room[kThreads / 64];
    double sum = 0;
    for (uint32_t c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        const uint32_t k = tensor_of(t, c);
        const int64_t at = (int64_t)(c - t.at[k].first) * kChunk, left = t.at[k].numbers - at;
        const void* g = t.at[k].grad;
        if (t.at[k].type == CER_TYPE_BF16) sum += chunk_squares(static_cast<const __bf16*>(g) + at, left);
        else if (t.at[k].type == CER_TYPE_F16) sum += chunk_squares(static_cast<const _Float16*>(g) + at, left);
        else sum += chunk_squares(static_cast<const float*>(g) + at, left);
    }
    sum = block_total_f64(sum, room);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

template <bool kOnce, class T>
__device__ __forceinline__ void chunk_scale(const T* g, T* out, int64_t left, float c) {
    constexpr int V = 16 / sizeof(T);
    constexpr int kSteps = kChunk / (kThreads * V);
    if (left >= kChunk) {
        Vec<float, V> v[kSteps];
#pragma unroll
        for (int s = 0; s < kSteps; ++s) v[s] = load_f32<T, V>(g + (s * kThreads + threadIdx.x) * V);
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            T* to = out + (s * kThreads + threadIdx.x) * V;
            if constexpr (kOnce) store_f32_once<T, V>(to, v[s] * c);
            else store_f32<T, V>(to, v[s] * c);
        }
        return;
    }
    for (int64_t e = threadIdx.x * V; e < left; e += kThreads * V) store_some<T, V>(out + e, load_some<T, V>(g + e, left - e) * c, left - e);
}

// The norm from the parts, then (`scale`) the table's gradients times the factor.
template <bool kOnce>
__global__ __launch_bounds__(kThreads) void clip_scale_kernel(ClipTable t, const double* part, uint32_t parts, float max_norm, float* norm, bool scale) {
    __shared__ double room[kThreads / 64];
    double sum = 0;
    for (uint32_t p = threadIdx.x; p < parts; p += kThreads) sum += part[p];
    const float all = (float)sqrt(block_total_f64(sum, room));
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = all;
    if (!scale) return;
    float c = max_norm / (all + 1e-6f);
    if (c > 1.f) c = 1.f;  // a NaN stays one
    for (uint32_t j = blockIdx.x; j < t.chunks; j += gridDim.x) {
        const uint32_t k = t.chunks - 1 - j;  // what was read last is in the caches still
        const uint32_t i = tensor_of(t, k);
        if (c == 1.f && t.at[i].grad == t.at[i].out) continue;
        const int64_t at = (int64_t)(k - t.at[i].first) * kChunk, left = t.at[i].numbers - at;
        const void* g = t.at[i].grad;
        void* out = t.at[i].out;
        if (t.at[i].type == CER_TYPE_BF16) chunk_scale<kOnce>(static_cast<const __bf16*>(g) + at, static_cast<__bf16*>(out) + at, left, c);
        else if (t.at[i].type == CER_TYPE_F16) chunk_scale<kOnce>(static_cast<const _Float16*>(g) + at, static_cast<_Float16*>(out) + at, left, c);
        else chunk_scale<kOnce>(static_cast<const float*>(g) + at, static_cast<float*>(out) + at, left, c);
    }
}

// The next table from grads[i ...]; tensors without elements are left out, larger ones than a table's chunk numbers hold are cut.
ClipTable next_table(const ClipCall& c, int64_t* i, int64_t* done) {
    ClipTable t;
    t.count = t.chunks = 0;
    constexpr int64_t most = 1 << 30;  // chunks
    while (*i < c.count && t.count < kEntries && t.chunks < most) {
        const cer_gradient_t& g = c.grads[*i];
        const int64_t left = g.numbers - *done, take = std::min(left, (most - (int64_t)t.chunks) * kChunk);
        const int64_t item = g.type == CER_TYPE_F32 ? 4 : 2;
        if (take > 0) {
            auto& e = t.at[t.count++];
            e.grad = static_cast<const char*>(g.grad) + *done * item;
            e.out = g.out ? static_cast<char*>(g.out) + *done * item : nullptr;
            e.numbers = take;
            e.first = t.chunks;
            e.type = g.type;
            t.chunks += (uint32_t)((take + kChunk - 1) / kChunk);
        }
        if (take == left) {
            ++*i;
            *done = 0;
        } else {
            *done += take;
        }
    }
    return t;
}
}  // namespace

int launch_clip(const ClipCall& c, hipStream_t s) {
    int64_t tables = 0;
    for (int64_t i = 0, done = 0; i < c.count; ++tables) (void)next_table(c, &i, &done);
    Temporary room((size_t)std::max<int64_t>(tables, 1) * kPartsPerLaunch * sizeof(double), s);
    if (room.error) return room.error;
    double* part = static_cast<double*>(room.p);
    uint32_t parts = 0;
    for (int64_t i = 0, done = 0; i < c.count;) {
        const ClipTable t = next_table(c, &i, &done);
        if (!t.count) continue;
        const unsigned grid = std::min<uint32_t>(t.chunks, kPartsPerLaunch);
        clip_squares_kernel<<<grid, kThreads, 0, s>>>(t, part + parts);
        if (int e = (int)hipGetLastError()) return e;
        parts += grid;
    }
    if (!c.scale || !parts) {
        ClipTable none;
        none.count = none.chunks = 0;
        clip_scale_kernel<false><<<1, kThreads, 0, s>>>(none, part, parts, 0.f, c.norm, false);
        return (int)hipGetLastError();
    }
    // Where gradients and outputs together are more than the memory-side cache of 256 MiB holds, none of the outputs is there when somebody wants them,
    // and stores that do not stay in the caches leave them to the gradients: 48 M numbers in 32 bits 98 us, with ordinary stores 116.
    int64_t bytes = 0;
    for (int64_t i = 0; i < c.count; ++i) bytes += c.grads[i].numbers * (c.grads[i].type == CER_TYPE_F32 ? 4 : 2) * (c.grads[i].out == c.grads[i].grad ? 1 : 2);
    const bool once = bytes > (int64_t)256 << 20;
    float* norm = c.norm;
    for (int64_t i = 0, done = 0; i < c.count;) {
        const ClipTable t = next_table(c, &i, &done);
        if (!t.count) continue;
        (once ? clip_scale_kernel<true> : clip_scale_kernel<false>)<<<std::min<uint32_t>(t.chunks, kPartsPerLaunch), kThreads, 0, s>>>(t, part, parts, c.max_norm, norm, true);
        if (int e = (int)hipGetLastError()) return e;
        norm = nullptr;  // written once
    }
    return 0;
}

}  // namespace cer
