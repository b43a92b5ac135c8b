// Shared by the operators beside a projection (norm.hip, adapter.hip, clip.hip): element types, loads and stores of several
// elements, sums over a wave and a workgroup, and the launchers that operators_capi.cpp calls after its checks.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/cer.h"
#include "cer_internal.hpp"

namespace cer {

// What a launcher returns where a temporary could not be had or a launch failed is a hipError_t value as int; 0: enqueued.
struct NormCall {
    cer_tokens_t x, r, sum, y;  // data == nullptr: not there
    int64_t tokens, n;
    const void* weight;
    int32_t weight_type;
    float eps;
    float *scale, *rstd;
};
int launch_norm(const NormCall& c, hipStream_t s);

struct NormBackwardCall {
    cer_tokens_t dy, h, dsum, dx;
    int64_t tokens, n;
    const float* rstd;
    const void* weight;
    int32_t weight_type;
    float* dweight;
};
int launch_norm_backward(const NormBackwardCall& c, hipStream_t s);

struct AdapterCall {
    cer_adapters_t w;
    const int32_t* index;
    int64_t tokens;
    cer_tokens_t x, base, y;
    float* hidden;
    void* workspace;
    int64_t workspace_bytes;
};
int64_t adapter_workspace(int64_t tokens, int64_t rank, int64_t in, int64_t out);
int launch_adapters(const AdapterCall& c, hipStream_t s);

struct AdapterBackwardCall {
    cer_adapters_t w;
    const int32_t* index;
    int64_t tokens;
    cer_tokens_t dy, x, base, dx;
    const float* hidden;
    float *dA, *dB;
};
int launch_adapters_backward(const AdapterBackwardCall& c, hipStream_t s);

struct ClipCall {
    const cer_gradient_t* grads;
    int64_t count;
    float max_norm;
    float* norm;
    bool scale;  // false: the norm alone
};
int launch_clip(const ClipCall& c, hipStream_t s);

// A temporary for the length of a call, ordered on the stream.
struct Temporary {
    Temporary(size_t bytes, hipStream_t s) : stream(s) { error = bytes ? temp_alloc(&p, bytes, s) : 0; }
    ~Temporary() {
        if (p) (void)temp_free(p, stream);
    }
    Temporary(const Temporary&) = delete;
    Temporary& operator=(const Temporary&) = delete;
    float* floats() const { return static_cast<float*>(p); }
    void* p = nullptr;
    hipStream_t stream;
    int error = 0;
};

#ifdef __HIPCC__

template <class T, int N>
using Vec = T __attribute__((ext_vector_type(N)));

// N elements at any address that an element may have: global loads and stores of gfx950 need no more.
template <class T, int N>
struct Packed {
    typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};
template <class T, int N>
__host__ __device__ __forceinline__ Vec<T, N> load(const T* p) {
    return *reinterpret_cast<const typename Packed<T, N>::type*>(p);
}
template <class T, int N>
__device__ __forceinline__ void store(T* p, Vec<T, N> v) {
    *reinterpret_cast<typename Packed<T, N>::type*>(p) = v;
}
template <class T, int N>
__device__ __forceinline__ Vec<float, N> load_f32(const T* p) {
    return __builtin_convertvector((load<T, N>(p)), Vec<float, N>);
}
template <class T, int N>
__device__ __forceinline__ void store_f32(T* p, Vec<float, N> v) {
    store<T, N>(p, __builtin_convertvector(v, Vec<T, N>));
}
// The same for what nobody reads soon: it does not take the place of other lines in the caches.
template <class T, int N>
__device__ __forceinline__ void store_f32_once(T* p, Vec<float, N> v) {
    __builtin_nontemporal_store(__builtin_convertvector(v, Vec<T, N>), reinterpret_cast<typename Packed<T, N>::type*>(p));
}
// The first `left` of N elements (left may be over N or below 1); the others are 0 and not read.
template <class T, int N>
__device__ __forceinline__ Vec<float, N> load_some(const T* p, int64_t left) {
    if (left >= N) return load_f32<T, N>(p);
    Vec<float, N> v;
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = j < left ? (float)p[j] : 0.f;
    return v;
}
template <class T, int N>
__device__ __forceinline__ void store_some(T* p, Vec<float, N> v, int64_t left) {
    if (left >= N) {
        store_f32<T, N>(p, v);
        return;
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (j < left) p[j] = (T)v[j];
}
// As they are in memory.
template <class T, int N>
__host__ __device__ __forceinline__ Vec<T, N> load_own(const T* p, int64_t left) {
    if (left >= N) return load<T, N>(p);
    Vec<T, N> v;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        v[j] = (T)0.f;
        if (j < left) v[j] = p[j];
    }
    return v;
}
// The same of an array whose type is an argument (one branch for a whole wave).
template <int N>
__device__ __forceinline__ Vec<float, N> load_some_of(const void* p, int type, int64_t at, int64_t left) {
    if (type == CER_TYPE_BF16) return load_some<__bf16, N>(static_cast<const __bf16*>(p) + at, left);
    if (type == CER_TYPE_F16) return load_some<_Float16, N>(static_cast<const _Float16*>(p) + at, left);
    return load_some<float, N>(static_cast<const float*>(p) + at, left);
}

__device__ __forceinline__ float wave_total(float v) {
#pragma unroll
    for (int k = 32; k; k >>= 1) v += __shfl_xor(v, k);
    return v;
}
// The larger one, and NaN if one is: a row with a NaN gets no scale that hides it.
__device__ __forceinline__ float larger(float a, float b) { return b > a || b != b ? b : a; }
__device__ __forceinline__ float wave_largest(float v) {
#pragma unroll
    for (int k = 32; k; k >>= 1) v = larger(v, __shfl_xor(v, k));
    return v;
}

// Over a workgroup of up to 16 waves; `room`: 16 floats of LDS that nothing else uses until the next barrier but one.
template <bool kLargest = false>
__device__ __forceinline__ float block_total(float v, float* room) {
    v = kLargest ? wave_largest(v) : wave_total(v);
    const unsigned waves = blockDim.x >> 6;
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
    __syncthreads();
    float all = room[0];
    for (unsigned k = 1; k < waves; ++k) all = kLargest ? larger(all, room[k]) : all + room[k];
    return all;
}

// The largest value that e4m3 without infinities (bias 7) holds.
constexpr float kLargestF8 = 448.f;

#endif  // __HIPCC__

}  // namespace cer
