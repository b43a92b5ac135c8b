// C entry points of the operators beside a projection (include/cer.h): every argument is checked here, the launchers rely on it.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <limits>

#include "operators.hpp"

namespace {
using namespace cer;

constexpr int64_t kMostTokens = (int64_t)1 << 28, kMostAdapterTokens = (int64_t)1 << 24, kMostNormFeatures = 65536, kMostFeatures = (int64_t)1 << 22, kMostRank = 256, kMostAdapters = 65535, kMostLd = (int64_t)1 << 22;

int bytes_of(int type) { return type == CER_TYPE_F32 ? 4 : type == CER_TYPE_F8 ? 1 : 2; }
bool number_type(int type) { return type == CER_TYPE_F32 || type == CER_TYPE_BF16 || type == CER_TYPE_F16; }

bool there(const cer_tokens_t* m) { return m && m->data; }

// A matrix that the call reads or (output) writes.
bool good(const cer_tokens_t* m, int64_t tokens, int64_t features, bool output, bool eight_bits = false) {
    if (!there(m)) return false;
    if (!number_type(m->type) && !(eight_bits && m->type == CER_TYPE_F8)) return false;
    if (m->order != CER_ORDER_ROWS && m->order != CER_ORDER_COLUMNS) return false;
    if (m->order == CER_ORDER_COLUMNS && m->type != CER_TYPE_F32) return false;
    if (reinterpret_cast<uintptr_t>(m->data) % bytes_of(m->type)) return false;
    const int64_t vectors = m->order == CER_ORDER_ROWS ? tokens : features, length = m->order == CER_ORDER_ROWS ? features : tokens;
    if (m->ld < 0 || (output && vectors > 1 && m->ld < length)) return false;
    return vectors <= 1 || m->ld <= std::numeric_limits<int64_t>::max() / 8 / vectors;
}
bool alike(const cer_tokens_t* a, const cer_tokens_t* b) { return a->type == b->type && a->order == b->order; }
// Whether two matrices share their place, if they do, in the way that is allowed.
bool same_or_apart(const cer_tokens_t* a, const cer_tokens_t* b) { return a->data != b->data || (a->ld == b->ld && alike(a, b)); }

cer_tokens_t or_none(const cer_tokens_t* m) { return there(m) ? *m : cer_tokens_t{nullptr, 0, 0, 0}; }

int result(int hip) { return hip ? record_hip_error(hip) : CER_OK; }

int check_adapters(const cer_adapters_t* w, int64_t tokens) {
    if (!w || !w->A || !w->B || !number_type(w->type)) return CER_E_INVALID;
    if (w->adapters < 1 || w->rank < 1 || w->in < 1 || w->out < 1 || tokens < 0) return CER_E_INVALID;
    if (w->rank > kMostRank || w->adapters > kMostAdapters || w->in > kMostFeatures || w->out > kMostFeatures || tokens > kMostAdapterTokens) return CER_E_TOO_LARGE;
    if (tokens * w->rank >= (int64_t)1 << 31 || w->adapters * w->rank * std::max(w->in, w->out) > (int64_t)1 << 33) return CER_E_TOO_LARGE;
    if (reinterpret_cast<uintptr_t>(w->A) % bytes_of(w->type) || reinterpret_cast<uintptr_t>(w->B) % bytes_of(w->type)) return CER_E_INVALID;
    if (w->stride_a < 0 || w->stride_b < 0 || w->ld_a < 0 || w->ld_b < 0) return CER_E_INVALID;
    // of strides: no product of one with an index overflows, and the kernels' offsets within a tile fit 32 bits
    if (std::max(w->stride_a, w->stride_b) > (int64_t)1 << 40 || std::max(w->ld_a, w->ld_b) > kMostLd) return CER_E_TOO_LARGE;
    return CER_OK;
}
// Offsets within a tile of 64 vectors fit 32 bits.  Columns of the most tokens lie as far apart as there are tokens: a lane's offset there is at most 48 columns.
bool near(const cer_tokens_t* m) { return !there(m) || m->ld <= (m->order == CER_ORDER_COLUMNS ? kMostAdapterTokens : kMostLd); }
// Activations beside adapters of this type.
bool fits(const cer_tokens_t* m, const cer_adapters_t* w) { return m->type == CER_TYPE_F32 || m->type == w->type; }
}  // namespace

extern "C" {

int rms_norm(const cer_tokens_t* X, const cer_tokens_t* residual, const cer_tokens_t* sum, const cer_tokens_t* Y, int64_t tokens, int64_t n,
             const void* weight, int32_t weight_type, float eps, float* scale, float* rstd, void* stream) {
    if (tokens < 0 || n < 1 || !(eps >= 0.f) || std::isinf(eps)) return CER_E_INVALID;
    if (tokens > kMostTokens || n > kMostNormFeatures) return CER_E_TOO_LARGE;
    if (tokens == 0) return CER_OK;
    if (!good(X, tokens, n, false) || !good(Y, tokens, n, true, true)) return CER_E_INVALID;
    if (there(residual) && !(good(residual, tokens, n, false) && alike(residual, X))) return CER_E_INVALID;
    if (there(sum) && !(good(sum, tokens, n, true) && alike(sum, X) && same_or_apart(sum, X) && (!there(residual) || same_or_apart(sum, residual)))) return CER_E_INVALID;
    if (Y->type != CER_TYPE_F32 && Y->type != CER_TYPE_F8 && Y->type != X->type) return CER_E_INVALID;
    if (Y->type == CER_TYPE_F8 ? X->order != CER_ORDER_ROWS || Y->order != CER_ORDER_ROWS || !scale : scale != nullptr) return CER_E_INVALID;
    if (X->order == CER_ORDER_COLUMNS && Y->type != CER_TYPE_F32) return CER_E_INVALID;
    if (weight && !number_type(weight_type)) return CER_E_INVALID;
    NormCall c{*X, or_none(residual), or_none(sum), *Y, tokens, n, weight, weight_type, eps, scale, rstd};
    return result(launch_norm(c, static_cast<hipStream_t>(stream)));
}

int rms_norm_backward(const cer_tokens_t* dY, const cer_tokens_t* H, const cer_tokens_t* dsum, const cer_tokens_t* dX, int64_t tokens, int64_t n,
                      const float* rstd, const void* weight, int32_t weight_type, float* dweight, void* stream) {
    if (tokens < 0 || n < 1) return CER_E_INVALID;
    if (tokens > kMostTokens || n > kMostNormFeatures) return CER_E_TOO_LARGE;
    if (tokens) {
        if (!good(dY, tokens, n, false) || !good(H, tokens, n, false) || !good(dX, tokens, n, true) || !rstd) return CER_E_INVALID;
        if (!alike(H, dX) || (there(dsum) && !(good(dsum, tokens, n, false) && alike(dsum, H)))) return CER_E_INVALID;
        if (dY->type != CER_TYPE_F32 && dY->type != H->type) return CER_E_INVALID;
        if (H->order == CER_ORDER_COLUMNS && dY->order != CER_ORDER_COLUMNS) return CER_E_INVALID;
        if (!same_or_apart(dX, dY) || !same_or_apart(dX, H) || (there(dsum) && !same_or_apart(dX, dsum))) return CER_E_INVALID;
    }
    if (weight && !number_type(weight_type)) return CER_E_INVALID;
    NormBackwardCall c{or_none(dY), or_none(H), or_none(dsum), or_none(dX), tokens, n, rstd, weight, weight_type, dweight};
    return result(launch_norm_backward(c, static_cast<hipStream_t>(stream)));
}

int64_t adapter_workspace_bytes(int64_t tokens, int64_t rank, int64_t in, int64_t out) {
    if (tokens < 0 || rank < 1 || in < 1 || out < 1) return CER_E_INVALID;
    if (tokens > kMostAdapterTokens || rank > kMostRank || in > kMostFeatures || out > kMostFeatures) return CER_E_TOO_LARGE;
    return tokens ? adapter_workspace(tokens, rank, in, out) : 0;
}

int adapter_matmul(const cer_adapters_t* w, const int32_t* index, int64_t tokens, const cer_tokens_t* X, const cer_tokens_t* base,
                   const cer_tokens_t* Y, float* hidden, void* workspace, int64_t workspace_bytes, void* stream) {
    if (int e = check_adapters(w, tokens)) return e;
    if (tokens == 0) return CER_OK;
    if (!index || !good(X, tokens, w->in, false) || !good(Y, tokens, w->out, true) || !alike(X, Y) || !fits(X, w)) return CER_E_INVALID;
    if (there(base) && !(good(base, tokens, w->out, false) && alike(base, Y) && same_or_apart(base, Y))) return CER_E_INVALID;
    if (!near(X) || !near(base) || !near(Y)) return CER_E_TOO_LARGE;
    if (workspace && (workspace_bytes < adapter_workspace(tokens, w->rank, w->in, w->out) || reinterpret_cast<uintptr_t>(workspace) % 4)) return CER_E_INVALID;
    AdapterCall c{*w, index, tokens, *X, or_none(base), *Y, hidden, workspace, workspace_bytes};
    return result(launch_adapters(c, static_cast<hipStream_t>(stream)));
}

int adapter_backward(const cer_adapters_t* w, const int32_t* index, int64_t tokens, const cer_tokens_t* dY, const cer_tokens_t* X,
                     const float* hidden, const cer_tokens_t* base, const cer_tokens_t* dX, float* dA, float* dB, void* stream) {
    if (int e = check_adapters(w, tokens)) return e;
    if (tokens) {
        if (!index || !good(dY, tokens, w->out, false) || !fits(dY, w)) return CER_E_INVALID;
        if (dA && !(good(X, tokens, w->in, false) && alike(X, dY))) return CER_E_INVALID;
        if (dB && !hidden) return CER_E_INVALID;
        if (there(dX) && !(good(dX, tokens, w->in, true) && alike(dX, dY))) return CER_E_INVALID;
        if (there(dX) && there(base) && !(good(base, tokens, w->in, false) && alike(base, dX) && same_or_apart(base, dX))) return CER_E_INVALID;
        if (!near(dY) || !near(X) || !near(base) || !near(dX)) return CER_E_TOO_LARGE;
    }
    AdapterBackwardCall c{*w, index, tokens, or_none(dY), or_none(X), or_none(base), or_none(dX), hidden, dA, dB};
    return result(launch_adapters_backward(c, static_cast<hipStream_t>(stream)));
}

static int clip(const cer_gradient_t* grads, int64_t count, float max_norm, float* norm, bool scale, void* stream) {
    if (count < 0 || (count && !grads) || !norm || !(max_norm >= 0.f) || std::isinf(max_norm)) return CER_E_INVALID;
    for (int64_t i = 0; i < count; ++i) {
        const cer_gradient_t& g = grads[i];
        if (g.numbers < 0 || !number_type(g.type)) return CER_E_INVALID;
        if (g.numbers > (int64_t)1 << 48) return CER_E_TOO_LARGE;
        if (g.numbers == 0) continue;
        if (!g.grad || reinterpret_cast<uintptr_t>(g.grad) % bytes_of(g.type)) return CER_E_INVALID;
        if (scale && (!g.out || reinterpret_cast<uintptr_t>(g.out) % bytes_of(g.type))) return CER_E_INVALID;
    }
    ClipCall c{grads, count, max_norm, norm, scale};
    return result(launch_clip(c, static_cast<hipStream_t>(stream)));
}
int grad_norm(const cer_gradient_t* grads, int64_t count, float* norm, void* stream) { return clip(grads, count, 0.f, norm, false, stream); }
int grad_clip(const cer_gradient_t* grads, int64_t count, float max_norm, float* norm, void* stream) {
    return clip(grads, count, max_norm, norm, true, stream);
}

}  // extern "C"
