// C entry points of the operators beside a projection (include/cer.h): every argument is checked here, the launchers rely on it.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <limits>

#include "operators.hpp"

namespace {
using namespace cer;

constexpr int64_t kMostBlockFeatures = 32768, kMostNumbers = (int64_t)1 << 40;
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
// An input, or one that may be missing, of another matrix' type and order.
bool like(const cer_tokens_t* m, const cer_tokens_t* as, int64_t tokens, int64_t features, bool output) { return good(m, tokens, features, output) && alike(m, as); }
bool none_or_like(const cer_tokens_t* m, const cer_tokens_t* as, int64_t tokens, int64_t features, bool output) { return !there(m) || like(m, as, tokens, features, output); }
bool rows_of(const cer_tokens_t* m, int type) { return m->order == CER_ORDER_ROWS && m->type == type; }
bool apart(const void* out, std::initializer_list<const cer_tokens_t*> others) {
    return !out || std::none_of(others.begin(), others.end(), [&](const cer_tokens_t* m) { return there(m) && m->data == out; });
}
bool vector(const void* p, int type) { return !p || (number_type(type) && reinterpret_cast<uintptr_t>(p) % bytes_of(type) == 0); }
bool room_enough(const void* workspace, int64_t have, int64_t need) { return have >= need && reinterpret_cast<uintptr_t>(workspace) % 16 == 0; }

int check_linear(const void* W, int64_t ldw, int32_t type, int64_t tokens, int64_t in, int64_t out, int32_t activation) {
    if (!W || !number_type(type) || tokens < 0 || in < 1 || out < 1 || ldw < 0) return CER_E_INVALID;
    if (activation < CER_ACTIVATION_NONE || activation > CER_ACTIVATION_SILU || reinterpret_cast<uintptr_t>(W) % bytes_of(type)) return CER_E_INVALID;
    if (tokens > kMostAdapterTokens || in > kMostFeatures || out > kMostFeatures || tokens * std::max(in, out) > kMostNumbers || in * out > kMostNumbers) return CER_E_TOO_LARGE;
    return out > 1 && ldw > std::numeric_limits<int64_t>::max() / 8 / out ? CER_E_INVALID : CER_OK;
}
// What block_norm and its gradient have in common.
int check_block(int64_t tokens, int64_t n, const void* gate_vector, int32_t gate_type, const void* post_weight, int32_t post_type, const void* pre_weight, int32_t pre_type, float scale) {
    if (tokens < 0 || n < 1 || !std::isfinite(scale)) return CER_E_INVALID;
    if (tokens > kMostTokens || n > kMostBlockFeatures || tokens * n > kMostNumbers) return CER_E_TOO_LARGE;
    return vector(gate_vector, gate_type) && vector(post_weight, post_type) && vector(pre_weight, pre_type) ? CER_OK : CER_E_INVALID;
}
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


int64_t linear_workspace_bytes(int64_t tokens, int64_t in, int64_t out, int32_t type, int32_t order, int32_t backward) {
    if (tokens < 0 || in < 1 || out < 1 || !number_type(type) || (order != CER_ORDER_ROWS && !(order == CER_ORDER_COLUMNS && type == CER_TYPE_F32))) return CER_E_INVALID;
    if (int e = check_linear(&type, in, type, tokens, in, out, CER_ACTIVATION_NONE)) return e == CER_E_TOO_LARGE ? e : CER_E_INVALID;
    void* some = &type;  // everything is there
    const cer_tokens_t m{some, 0, type, order};
    if (!backward) return linear_room({some, in, type, tokens, in, out, m, m, m, m, some, type, CER_ACTIVATION_SILU, nullptr});
    float all = 0;
    return linear_backward_room({some, in, type, tokens, in, out, m, m, m, m, m, CER_ACTIVATION_SILU, some, in, &all, nullptr});
}

int64_t block_workspace_bytes(int64_t tokens, int64_t n, int32_t type, int32_t columns, int32_t backward) {
    if (!number_type(type)) return CER_E_INVALID;
    if (int e = check_block(tokens, n, nullptr, 0, nullptr, 0, nullptr, 0, 1.f)) return e;
    float all = 0;
    const cer_tokens_t stream{&all, 0, type, CER_ORDER_ROWS}, branch{&all, 0, columns ? CER_TYPE_F32 : type, columns ? CER_ORDER_COLUMNS : CER_ORDER_ROWS}, none{nullptr, 0, 0, 0};
    if (!backward) return block_room({stream, branch, stream, branch, none, tokens, n, nullptr, 0, nullptr, nullptr, 0, 0, 1.f, 0.f, true, nullptr, nullptr, nullptr});
    return block_backward_room({branch, stream, branch, none, none, stream, branch, none, tokens, n, &all, &all, &all, 0, nullptr, nullptr, 0, 0, 1.f, &all, &all, &all, nullptr});
}

int linear_matmul(const void* W, int64_t ldw, int32_t type, int64_t tokens, int64_t in, int64_t out, const cer_tokens_t* X, const cer_tokens_t* Y,
                  const void* bias, int32_t bias_type, const cer_tokens_t* residual, int32_t activation, const cer_tokens_t* pre, void* workspace,
                  int64_t workspace_bytes, void* stream) {
    if (int e = check_linear(W, ldw, type, tokens, in, out, activation)) return e;
    if (!vector(bias, bias_type)) return CER_E_INVALID;
    if (tokens == 0) return CER_OK;
    if (!good(X, tokens, in, false) || X->type != type || !like(Y, X, tokens, out, true)) return CER_E_INVALID;
    if (!none_or_like(residual, X, tokens, out, false) || !none_or_like(pre, X, tokens, out, true)) return CER_E_INVALID;
    if (there(residual) && !same_or_apart(residual, Y)) return CER_E_INVALID;
    if (Y->data == W || !apart(Y->data, {X, pre}) || (there(pre) && (pre->data == W || !apart(pre->data, {X, residual})))) return CER_E_INVALID;
    LinearCall c{W, ldw, type, tokens, in, out, *X, or_none(residual), *Y, or_none(pre), bias, bias_type, activation, workspace};
    if (workspace && !room_enough(workspace, workspace_bytes, linear_room(c))) return CER_E_INVALID;
    return result(launch_linear(c, static_cast<hipStream_t>(stream)));
}

int linear_backward(const void* W, int64_t ldw, int32_t type, int64_t tokens, int64_t in, int64_t out, const cer_tokens_t* dY, const cer_tokens_t* X,
                    int32_t activation, const cer_tokens_t* pre, const cer_tokens_t* base, const cer_tokens_t* dX, void* dW, int64_t lddw, float* dbias,
                    void* workspace, int64_t workspace_bytes, void* stream) {
    if (int e = check_linear(W, ldw, type, tokens, in, out, activation)) return e;
    if (dW && (lddw < in || (out > 1 && lddw > std::numeric_limits<int64_t>::max() / 8 / out) || reinterpret_cast<uintptr_t>(dW) % bytes_of(type) || dW == W)) return CER_E_INVALID;
    if (reinterpret_cast<uintptr_t>(dbias) % 4) return CER_E_INVALID;
    if (tokens) {
        if (!good(dY, tokens, out, false) || dY->type != type) return CER_E_INVALID;
        if (activation != CER_ACTIVATION_NONE && !like(pre, dY, tokens, out, false)) return CER_E_INVALID;
        if (dW && !like(X, dY, tokens, in, false)) return CER_E_INVALID;
        if (!none_or_like(dX, dY, tokens, in, true) || (there(dX) && !none_or_like(base, dX, tokens, in, false))) return CER_E_INVALID;
        if (there(dX) && there(base) && !same_or_apart(base, dX)) return CER_E_INVALID;
        if (there(dX) && (dX->data == W || dX->data == dW || !apart(dX->data, {dY, X, pre}))) return CER_E_INVALID;
        if (!apart(dW, {dY, X, pre, base}) || !apart(dbias, {dY, X, pre, base, dX})) return CER_E_INVALID;
    }
    const cer_tokens_t none{nullptr, 0, 0, 0};
    LinearBackwardCall c{W, ldw, type, tokens, in, out, or_none(dY), or_none(X), activation != CER_ACTIVATION_NONE ? or_none(pre) : none, or_none(base), or_none(dX), activation, dW, lddw, dbias, workspace};
    if (workspace && !room_enough(workspace, workspace_bytes, linear_backward_room(c))) return CER_E_INVALID;
    return result(launch_linear_backward(c, static_cast<hipStream_t>(stream)));
}

int block_norm(const cer_tokens_t* X, const cer_tokens_t* F, const cer_tokens_t* H, const cer_tokens_t* Y, int64_t tokens, int64_t n, const cer_tokens_t* gate,
               const void* gate_vector, int32_t gate_type, const void* post_weight, int32_t post_type, const void* pre_weight, int32_t pre_type, float scale,
               float eps, int32_t post, float* rstd_post, float* rstd_pre, void* workspace, int64_t workspace_bytes, void* stream) {
    if (int e = check_block(tokens, n, gate_vector, gate_type, post_weight, post_type, pre_weight, pre_type, scale)) return e;
    if (!(eps >= 0.f) || std::isinf(eps) || (!post && (post_weight || rstd_post)) || (gate_vector && there(gate))) return CER_E_INVALID;
    if (tokens == 0) return CER_OK;
    if (!good(X, tokens, n, false) || X->order != CER_ORDER_ROWS || !like(H, X, tokens, n, true) || !same_or_apart(H, X)) return CER_E_INVALID;
    if (!good(F, tokens, n, false) || !good(Y, tokens, n, true)) return CER_E_INVALID;
    if ((F->type != CER_TYPE_F32 && F->type != X->type) || (Y->type != CER_TYPE_F32 && Y->type != X->type)) return CER_E_INVALID;
    if (F->data == Y->data && (!same_or_apart(F, Y) || F->order != CER_ORDER_ROWS)) return CER_E_INVALID;
    if (!none_or_like(gate, X, tokens, n, false)) return CER_E_INVALID;
    if (!apart(H->data, {F, Y, gate}) || !apart(Y->data, {X, gate})) return CER_E_INVALID;
    BlockCall c{*X, *F, *H, *Y, or_none(gate), tokens, n, gate_vector, gate_type, post_weight, pre_weight, post_type, pre_type, scale, eps, post != 0, rstd_post, rstd_pre, workspace};
    if (workspace && !room_enough(workspace, workspace_bytes, block_room(c))) return CER_E_INVALID;
    return result(launch_block_norm(c, static_cast<hipStream_t>(stream)));
}

int block_norm_backward(const cer_tokens_t* dY, const cer_tokens_t* H, const cer_tokens_t* F, const float* rstd_pre, const float* rstd_post,
                        const cer_tokens_t* dX, const cer_tokens_t* dF, int64_t tokens, int64_t n, const cer_tokens_t* gate, const void* gate_vector,
                        int32_t gate_type, const void* post_weight, int32_t post_type, const void* pre_weight, int32_t pre_type, float scale,
                        const cer_tokens_t* dsum, const cer_tokens_t* dgate, float* dgate_vector, float* dpost_weight, float* dpre_weight, void* workspace,
                        int64_t workspace_bytes, void* stream) {
    if (int e = check_block(tokens, n, gate_vector, gate_type, post_weight, post_type, pre_weight, pre_type, scale)) return e;
    if (gate_vector && there(gate)) return CER_E_INVALID;
    if (dgate_vector && !gate_vector) return CER_E_INVALID;
    if (tokens) {
        if (!rstd_pre || (!rstd_post && (post_weight || dpost_weight))) return CER_E_INVALID;
        if (!good(H, tokens, n, false) || H->order != CER_ORDER_ROWS || !like(dX, H, tokens, n, true)) return CER_E_INVALID;
        if (!good(dY, tokens, n, false) || (dY->type != CER_TYPE_F32 && dY->type != H->type)) return CER_E_INVALID;
        if (!good(F, tokens, n, false) || (F->type != CER_TYPE_F32 && F->type != H->type) || !like(dF, F, tokens, n, true)) return CER_E_INVALID;
        if (!none_or_like(dsum, H, tokens, n, false) || !none_or_like(gate, H, tokens, n, false) || !none_or_like(dgate, H, tokens, n, true)) return CER_E_INVALID;
        if (there(dgate) && !there(gate)) return CER_E_INVALID;
        if (!apart(dX->data, {dY, H, F, gate, dsum, dF, dgate}) || !apart(dF->data, {dY, H, F, gate, dsum, dgate})) return CER_E_INVALID;
        if (there(dgate) && !apart(dgate->data, {dY, H, F, gate, dsum})) return CER_E_INVALID;
    }
    BlockBackwardCall c{or_none(dY), or_none(H), or_none(F), or_none(gate), or_none(dsum), or_none(dX), or_none(dF), or_none(dgate), tokens, n, rstd_post, rstd_pre,
                        gate_vector, gate_type, post_weight, pre_weight, post_type, pre_type, scale, dgate_vector, dpost_weight, dpre_weight, workspace};
    if (workspace && !room_enough(workspace, workspace_bytes, block_backward_room(c))) return CER_E_INVALID;
    return result(launch_block_norm_backward(c, static_cast<hipStream_t>(stream)));
}

int dropout_add(const cer_tokens_t* X, const cer_tokens_t* residual, const cer_tokens_t* Y, int64_t tokens, int64_t n, const int64_t* key, double p, int64_t call,
                void* stream) {
    if (tokens < 0 || n < 1 || !(p >= 0.0 && p <= 1.0)) return CER_E_INVALID;
    if (tokens > kMostTokens || n > kMostFeatures || tokens * n > kMostNumbers) return CER_E_TOO_LARGE;
    if (tokens == 0) return CER_OK;
    if (!good(X, tokens, n, false) || !like(Y, X, tokens, n, true) || !none_or_like(residual, X, tokens, n, false)) return CER_E_INVALID;
    if (!same_or_apart(Y, X) || (there(residual) && !same_or_apart(Y, residual))) return CER_E_INVALID;
    if (!key || reinterpret_cast<uintptr_t>(key) % 8) return CER_E_INVALID;
    DropoutCall c{*X, or_none(residual), *Y, tokens, n, key, (uint32_t)std::nearbyint(p * 65536.0), call};
    return result(launch_dropout(c, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
