// Which memory of an adapter's weights a lane of the many-token kernel reads: nothing of a rank past the adapter's own, whose memory need not
// exist.  For the device and, in the tests, for the host, where what lies behind the weights can be out of reach.
#pragma once

#include "operators.hpp"

namespace cer {

// Elements at a wave's own address (a scalar) and a lane's offset in bytes from it.
template <class T>
__host__ __device__ __forceinline__ const T* at(const T* base, uint32_t bytes) { return reinterpret_cast<const T*>(reinterpret_cast<const char*>(base) + bytes); }
template <class T>
__host__ __device__ __forceinline__ T* at(T* base, uint32_t bytes) { return reinterpret_cast<T*>(reinterpret_cast<char*>(base) + bytes); }

// The same offset, as a number of its own: sums with it are made where they stand, as a scalar and an offset that the load adds up, and not kept in two registers each
// through the loops around them (32 of those: 64 registers).
__host__ __device__ __forceinline__ uint32_t here(uint32_t bytes) {
#ifdef __HIP_DEVICE_COMPILE__
    asm volatile("" : "+v"(bytes));
#endif
    return bytes;
}

// Eight ranks from `low` on of four neighbours on the long axis, 0 from the adapter's `rank` on (over 0).  Element (neighbour j, rank r) at
// w[r * ld + j] (kAlong) or w[j * ld + r], `lane` bytes on.  Where the adapter has whole fours or eights of ranks they are loaded so, else one
// by one; in the place of ranks past the last one the first ones are read again.
template <class TW, bool kAlong>
__host__ __device__ __forceinline__ void weights_of(const TW* w, uint32_t lane, int64_t ld, int rank, int low, Vec<TW, 8> (&u)[4]) {
    auto place = [&](int r) { return here(lane) + (uint32_t)(r < rank ? kAlong ? r * ld : r : 0) * (uint32_t)sizeof(TW); };
    if constexpr (kAlong) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const Vec<TW, 4> v = load<TW, 4>(at(w, place(low + e)));
#pragma unroll
            for (int j = 0; j < 4; ++j) u[j][e] = v[j];
        }
    } else if (rank % 8 == 0) {
        const uint32_t first = place(low);
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = load<TW, 8>(at(w + j * ld, first));
    } else if (rank % 4 == 0) {
        const uint32_t first = place(low), second = place(low + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            u[j] = __builtin_shufflevector(load<TW, 4>(at(w + j * ld, first)), load<TW, 4>(at(w + j * ld, second)), 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) u[j][e] = *at(w + j * ld, place(low + e));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (rank % 8)
#pragma unroll
            for (int e = 0; e < 8; ++e) u[j][e] = low + e < rank ? u[j][e] : (TW)0.f;
        else if (low >= rank)
            u[j] = (TW)0.f;
    }
}

}  // namespace cer
