// Dropout with a mask that is formed again wherever it is needed and never stored.
//
// y = r + (keep ? x . 65536 / (65536 - d) : 0),   d = round(p . 65536),   keep = a 16-bit random number of the element's own is at least d.
// The numbers are those of Philox 4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011): eight features of
// a token share a counter of 128 bits -- which eight of the tensor, and which call -- so that the mask depends on the key, the token and
// the feature alone, not on types, orders, strides or the launch, and the backward pass is the same call on the gradient.
//
// 16 bits per element and not 32: the generator's 20 wide products per eight elements are then hidden behind the bytes; the probability is a
// multiple of 2^-16, and the factor is that multiple's, so that the mean stays x.
#include <algorithm>

#include "operators.hpp"

namespace cer {
namespace {

// Quotients of numbers below 2^31 by d (1 <= d < 2^31): (a . multiplier) >> shift, exact because multiplier . d - 2^shift < 2^(shift - 31).
struct Divide {
    uint32_t multiplier, shift;
    explicit Divide(uint32_t d) {
        uint32_t up = 0;
        while (((uint64_t)1 << up) < d) ++up;
        shift = 31 + up;
        multiplier = (uint32_t)((((uint64_t)1 << shift) + d - 1) / d);
    }
    __device__ __forceinline__ uint32_t operator()(uint32_t a) const { return (uint32_t)(((uint64_t)a * multiplier) >> shift); }
};

struct DropArgs {
    const void *x, *r;
    void* y;
    int64_t ldx, ldr, ldy;
    int64_t n, first_block;           // of the launch's tokens
    uint32_t tokens, blocks, dropped;  // of this launch; blocks of eight features of a token
    float factor;
    Divide by;
    const uint64_t* key;  // seed, offset
    uint64_t call;
};

// Eight 16-bit numbers of block `at`, two to a word, the earlier one in the lower half.
__device__ __forceinline__ Vec<uint32_t, 4> random_block(uint64_t at, uint64_t seed, uint64_t which) {
    uint32_t a = (uint32_t)at, b = (uint32_t)(at >> 32), c = (uint32_t)which, d = (uint32_t)(which >> 32);
    uint32_t k = (uint32_t)seed, l = (uint32_t)(seed >> 32);
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t p = (uint64_t)a * 0xD2511F53u, q = (uint64_t)c * 0xCD9E8D57u;
        a = (uint32_t)(q >> 32) ^ b ^ k;
        b = (uint32_t)q;
        c = (uint32_t)(p >> 32) ^ d ^ l;
        d = (uint32_t)p;
        k += 0x9E3779B9u;
        l += 0xBB67AE85u;
    }
    return {a, b, c, d};
}

// A thread for eight features of a token: in rows neighbouring threads have neighbouring features, in columns neighbouring tokens.
template <class T, bool kColumns>
__global__ __launch_bounds__(256) void dropout_kernel(DropArgs a) {
    const uint32_t g = blockIdx.x * 256u + threadIdx.x;
    if (g >= a.tokens * a.blocks) return;
    const uint32_t slow = a.by(g), quick = g - slow * (kColumns ? a.tokens : a.blocks);
    const uint32_t t = kColumns ? quick : slow, block = kColumns ? slow : quick;
    const int64_t i = (int64_t)block * 8, left = a.n - i;
    Vec<float, 8> x, r = 0.f;
    if constexpr (kColumns) {
        const T* from = static_cast<const T*>(a.x) + i * a.ldx + t;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = j < left ? (float)from[j * a.ldx] : 0.f;
        if (a.r) {
            const T* add = static_cast<const T*>(a.r) + i * a.ldr + t;
#pragma unroll
            for (int j = 0; j < 8; ++j) r[j] = j < left ? (float)add[j * a.ldr] : 0.f;
        }
    } else {
        x = load_some<T, 8>(static_cast<const T*>(a.x) + (int64_t)t * a.ldx + i, left);
        if (a.r) r = load_some<T, 8>(static_cast<const T*>(a.r) + (int64_t)t * a.ldr + i, left);
    }
    const Vec<uint32_t, 4> words = random_block((uint64_t)a.first_block + (uint64_t)t * a.blocks + block, a.key[0], a.key[1] + a.call);
    Vec<float, 8> y;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t number = j % 2 ? words[j / 2] >> 16 : words[j / 2] & 0xFFFFu;
        y[j] = number >= a.dropped ? x[j] * a.factor : 0.f;  // a dropped NaN or infinity is 0 too
    }
    if (a.r) y += r;
    if constexpr (kColumns) {
        T* to = static_cast<T*>(a.y) + i * a.ldy + t;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < left) to[j * a.ldy] = (T)y[j];
    } else {
        store_some<T, 8>(static_cast<T*>(a.y) + (int64_t)t * a.ldy + i, y, left);
    }
}

template <class T, bool kColumns>
int dropout_of(const DropoutCall& c, hipStream_t s) {
    const int64_t blocks = (c.n + 7) / 8, at_once = std::max<int64_t>(1, ((int64_t)1 << 30) / blocks);  // a launch's blocks fit 31 bits
    const int32_t item = (int32_t)sizeof(T);
    for (int64_t t = 0; t < c.tokens; t += at_once) {
        const uint32_t tokens = (uint32_t)std::min(at_once, c.tokens - t);
        auto from = [&](const cer_tokens_t& m) { return m.data ? static_cast<char*>(m.data) + t * (kColumns ? 1 : m.ld) * item : nullptr; };
        DropArgs a{from(c.x), from(c.r), from(c.y), c.x.ld, c.r.ld, c.y.ld, c.n, t * blocks, tokens, (uint32_t)blocks, c.dropped,
                   c.dropped < 65536 ? 65536.f / (float)(65536 - c.dropped) : 0.f, Divide(kColumns ? tokens : (uint32_t)blocks), reinterpret_cast<const uint64_t*>(c.key),
                   (uint64_t)c.call};
        dropout_kernel<T, kColumns><<<(unsigned)((tokens * blocks + 255) / 256), 256, 0, s>>>(a);
        if (int e = (int)hipGetLastError()) return e;
    }
    return 0;
}
}  // namespace

int launch_dropout(const DropoutCall& c, hipStream_t s) {
    if (c.x.order == CER_ORDER_COLUMNS) return dropout_of<float, true>(c, s);
    if (c.x.type == CER_TYPE_BF16) return dropout_of<__bf16, false>(c, s);
    if (c.x.type == CER_TYPE_F16) return dropout_of<_Float16, false>(c, s);
    return dropout_of<float, false>(c, s);
}

}  // namespace cer
