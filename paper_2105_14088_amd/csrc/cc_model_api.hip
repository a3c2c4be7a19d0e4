// C ABI of the order model: argument checks, launches.  Declarations and contracts: include/cc.h.
#include <hip/hip_runtime.h>

#include <cmath>

#include "../../include/cc.h"
#include "cc_internal.h"

namespace {

#define CC_HIP(expr)                                      \
    do {                                                  \
        hipError_t e_ = (expr);                           \
        if (e_ != hipSuccess) return cc::hip_fail(e_);    \
    } while (0)

static_assert(CC_SCAN_CHUNK == cc::kScanChunk, "the kernels keep states as the header says");
static_assert(CC_F32 == cc::kF32 && CC_F16 == cc::kF16 && CC_BF16 == cc::kBF16, "element types");

constexpr int64_t kMaxRow = 1 << 24, kMaxRows = 1 << 30, kMaxPositions = (int64_t)1 << 31, kMaxChannels = (int64_t)1 << 32, kMaxProduct = (int64_t)1 << 38;

bool is_dtype(int d) { return d == CC_F32 || d == CC_F16 || d == CC_BF16; }
uintptr_t below(int dtype) { return dtype == CC_F32 ? 3u : 1u; }
bool aligned(const void* p, uintptr_t mask) { return ((uintptr_t)p & mask) == 0; }
// A required pointer at its element's alignment; an optional one that may be null.
bool have(const void* p, uintptr_t mask) { return p && aligned(p, mask); }
// A scale of logits: with room on both sides for its products in 32 bits.
bool scale_ok(float v) { return v >= 0x1p-64f && v <= 0x1p64f; }

bool workspace_ok(const void* p, size_t bytes, size_t need) {
    return need == 0 || (p && bytes >= need && aligned(p, 255u));
}

// Rows of an output must not overlap: a dimension of more than one entry steps over what lies inside it.
bool separate(int64_t outer, int64_t outer_stride, int64_t inner, int64_t inner_stride, int64_t row) {
    if (inner > 1 && inner_stride < row) return false;
    return outer <= 1 || outer_stride >= (inner - 1) * inner_stride + row || (inner > 1 && outer_stride >= row && inner_stride >= (outer - 1) * outer_stride + row);
}
bool strides_ok(int64_t a, int64_t b) { return a >= 0 && b >= 0; }

bool scan_sizes(int64_t B, int64_t T, int64_t D) {
    return B >= 0 && T >= 0 && D >= 1 && D <= kMaxRow && B < kMaxPositions && T < kMaxPositions && B * T < kMaxPositions && B * D < kMaxChannels;
}
bool token_sizes(int64_t B, int64_t T, int64_t V) {
    return B >= 0 && T >= 0 && V >= 1 && V <= kMaxRow && B < kMaxPositions && T < kMaxPositions && B * T < kMaxPositions;
}

// Rows that are stored where others are read: in the same places.
bool in_place_ok(const void* out, int64_t out_stride, const void* in, int64_t in_stride) { return out != in || out_stride == in_stride; }
bool norm_sizes(int64_t n, int64_t D) { return n >= 0 && n < kMaxPositions && D >= 1 && D <= kMaxRow; }
bool product_sizes(int64_t M, int64_t N, int64_t K) {
    return M >= 0 && M < kMaxPositions && N >= 0 && N <= kMaxRow && K >= 0 && K <= CC_PRODUCT_MAX_K && M * N <= kMaxProduct;
}

// What the two calls that shape logits share.
int check_shape(const void* logits, int32_t dtype, int64_t B, int64_t T, int64_t V, int64_t stride_b, int64_t stride_t, const int32_t* history,
                int64_t L, int64_t history_stride, const int32_t* lengths, const int32_t* starts, const float* penalties, const float* bias,
                int64_t bias_stride, const uint32_t* allowed, int64_t allowed_stride_b, int64_t allowed_stride_t, const void* out,
                int64_t out_stride_b, int64_t out_stride_t) {
    if (!is_dtype(dtype) || !token_sizes(B, T, V) || !strides_ok(stride_b, stride_t)) return CC_ERR_INVALID_ARG;
    if (L < 0 || L >= kMaxPositions || !strides_ok(history_stride, bias_stride) || !strides_ok(allowed_stride_b, allowed_stride_t))
        return CC_ERR_INVALID_ARG;
    if (B == 0 || T == 0) return CC_OK;
    if (!have(logits, below(dtype)) || !have(out, below(dtype)) || !separate(B, out_stride_b, T, out_stride_t, V)) return CC_ERR_INVALID_ARG;
    if ((L > 0 && !history) || !aligned(history, 3u) || !aligned(lengths, 3u) || !aligned(starts, 3u) || !aligned(penalties, 3u) ||
        !aligned(bias, 3u) || !aligned(allowed, 3u))
        return CC_ERR_INVALID_ARG;
    return CC_OK;
}

cc::ShapeCall shape_call(const void* logits, int32_t dtype, int64_t B, int64_t T, int64_t V, int64_t stride_b, int64_t stride_t,
                         const int32_t* history, int64_t L, int64_t history_stride, const int32_t* lengths, const int32_t* starts,
                         const float* penalties, const float* bias, int64_t bias_stride, const uint32_t* allowed, int64_t allowed_stride_b,
                         int64_t allowed_stride_t, void* out, int64_t out_stride_b, int64_t out_stride_t) {
    cc::ShapeCall c = {};
    c.logits = logits;
    c.dtype = dtype;
    c.B = B;
    c.T = T;
    c.V = V;
    c.stride_b = stride_b;
    c.stride_t = stride_t;
    c.history = L > 0 ? history : nullptr;
    c.L = L;
    c.history_stride = history_stride;
    c.lengths = lengths;
    c.starts = starts;
    c.penalties = penalties;
    c.bias = bias;
    c.bias_stride = bias_stride;
    c.allowed = allowed;
    c.allowed_stride_b = allowed_stride_b;
    c.allowed_stride_t = allowed_stride_t;
    c.out = out;
    c.out_stride_b = out_stride_b;
    c.out_stride_t = out_stride_t;
    return c;
}

// What the four calls on logits share.
int check_tokens(const void* logits, int32_t dtype, int64_t B, int64_t T, int64_t V, int64_t stride_b, int64_t stride_t,
                 const int32_t* tokens, int32_t placed, float scale, const void* grad, int64_t gsb, int64_t gst) {
    if (!is_dtype(dtype) || !token_sizes(B, T, V) || !strides_ok(stride_b, stride_t) || !scale_ok(scale)) return CC_ERR_INVALID_ARG;
    if (placed && (V > CC_MAX_N || T > CC_MAX_N)) return CC_ERR_UNSUPPORTED_N;
    if (B == 0 || T == 0) return CC_OK;
    if (!have(logits, below(dtype)) || !have(tokens, 3u)) return CC_ERR_INVALID_ARG;
    if (grad) {
        if (!aligned(grad, below(dtype)) || !separate(B, gsb, T, gst, V)) return CC_ERR_INVALID_ARG;
        // in place: an element's gradient goes where the element was
        if (grad == logits && (gsb != stride_b || gst != stride_t)) return CC_ERR_INVALID_ARG;
    }
    return CC_OK;
}

cc::TokenCall token_call(const void* logits, int32_t dtype, int64_t B, int64_t T, int64_t V, int64_t stride_b, int64_t stride_t,
                         const int32_t* tokens, const uint8_t* mask, int32_t placed, float scale) {
    cc::TokenCall c = {};
    c.logits = logits;
    c.dtype = dtype;
    c.B = B;
    c.T = T;
    c.V = V;
    c.stride_b = stride_b;
    c.stride_t = stride_t;
    c.tokens = tokens;
    c.mask = mask;
    c.placed = placed != 0;
    c.scale = scale;
    c.grad_scale = 1.0f;
    return c;
}

}  // namespace

extern "C" {

int cc_embed(const void* table, int32_t dtype, int64_t V, int64_t D, int64_t table_stride, const int32_t* ids, int64_t n,
             float scale, void* out, int64_t out_stride, void* stream) {
    if (!is_dtype(dtype) || V < 1 || V >= kMaxRows || D < 1 || D > kMaxRow || n < 0 || n >= kMaxRows) return CC_ERR_INVALID_ARG;
    if (table_stride < 0 || !separate(1, 0, n, out_stride, D) || !std::isfinite(scale)) return CC_ERR_INVALID_ARG;
    if (n == 0) return CC_OK;
    if (!have(table, below(dtype)) || !have(ids, 3u) || !have(out, below(dtype))) return CC_ERR_INVALID_ARG;
    cc::EmbedCall c = {};
    c.table = table;
    c.ids = ids;
    c.out = out;
    c.dtype = dtype;
    c.V = V;
    c.D = D;
    c.n = n;
    c.table_stride = table_stride;
    c.out_stride = out_stride;
    c.scale = scale;
    CC_HIP(cc::poison_lds_if_asked((hipStream_t)stream));
    CC_HIP(cc::launch_embed(c, (hipStream_t)stream));
    return CC_OK;
}

size_t cc_embed_workspace_bytes(int64_t V, int64_t D, int64_t n) {
    if (V < 1 || V >= kMaxRows || D < 1 || D > kMaxRow || n < 0 || n >= kMaxRows) return 0;
    return cc::embed_workspace_bytes(V, D, n);
}

int cc_embed_backward(const void* grad, int32_t dtype, int64_t n, int64_t D, int64_t grad_stride, const int32_t* ids, int64_t V,
                      float scale, void* grad_table, int32_t grad_dtype, int64_t grad_table_stride, int32_t accumulate,
                      void* workspace, size_t workspace_bytes, void* stream) {
    if (!is_dtype(dtype) || V < 1 || V >= kMaxRows || D < 1 || D > kMaxRow || n < 0 || n >= kMaxRows) return CC_ERR_INVALID_ARG;
    if ((grad_dtype != CC_F32 && grad_dtype != dtype) || grad_stride < 0 || !separate(1, 0, V, grad_table_stride, D) || !std::isfinite(scale))
        return CC_ERR_INVALID_ARG;
    if (n == 0 && accumulate) return CC_OK;
    if (!have(grad_table, below(grad_dtype))) return CC_ERR_INVALID_ARG;
    if (n > 0 && (!have(grad, below(dtype)) || !have(ids, 3u))) return CC_ERR_INVALID_ARG;
    if (!workspace_ok(workspace, workspace_bytes, cc::embed_workspace_bytes(V, D, n))) return CC_ERR_WORKSPACE;
    cc::EmbedCall c = {};
    c.grad_table = grad_table;
    c.ids = ids;
    c.out = const_cast<void*>(grad);
    c.dtype = dtype;
    c.grad_dtype = grad_dtype;
    c.accumulate = accumulate != 0;
    c.V = V;
    c.D = D;
    c.n = n;
    c.table_stride = grad_table_stride;
    c.out_stride = grad_stride;
    c.scale = scale;
    c.workspace = workspace;
    CC_HIP(cc::poison_lds_if_asked((hipStream_t)stream));
    CC_HIP(cc::launch_embed_backward(c, (hipStream_t)stream));
    return CC_OK;
}

size_t cc_gated_scan_workspace_bytes(int64_t B, int64_t T, int64_t D) {
    return scan_sizes(B, T, D) ? cc::scan_workspace_bytes(B, T, D) : 0;
}

int cc_gated_scan(const void* x, int64_t x_stride_b, int64_t x_stride_t, const void* gate, int64_t gate_stride_b,
                  int64_t gate_stride_t, int32_t dtype, int64_t B, int64_t T, int64_t D, const int32_t* lengths, const float* h0,
                  void* h, int64_t h_stride_b, int64_t h_stride_t, float* last, float* states, void* workspace,
                  size_t workspace_bytes, void* stream) {
    if (!is_dtype(dtype) || !scan_sizes(B, T, D)) return CC_ERR_INVALID_ARG;
    if (!strides_ok(x_stride_b, x_stride_t) || !strides_ok(gate_stride_b, gate_stride_t) || !separate(B, h_stride_b, T, h_stride_t, D))
        return CC_ERR_INVALID_ARG;
    if (B == 0) return CC_OK;
    if (T > 0 && (!have(x, below(dtype)) || !have(gate, below(dtype)) || !have(h, below(dtype)))) return CC_ERR_INVALID_ARG;
    if (!aligned(lengths, 3u) || !aligned(h0, 3u) || !aligned(last, 3u) || !aligned(states, 3u)) return CC_ERR_INVALID_ARG;
    if (!workspace_ok(workspace, workspace_bytes, cc::scan_workspace_bytes(B, T, D))) return CC_ERR_WORKSPACE;
    cc::ScanCall c = {};
    c.x = {const_cast<void*>(x), x_stride_b, x_stride_t};
    c.gate = {const_cast<void*>(gate), gate_stride_b, gate_stride_t};
    c.dtype = dtype;
    c.B = B;
    c.T = T;
    c.D = D;
    c.lengths = lengths;
    c.h0 = h0;
    c.h = {h, h_stride_b, h_stride_t};
    c.last = last;
    c.states = states;
    c.workspace = workspace;
    CC_HIP(cc::poison_lds_if_asked((hipStream_t)stream));
    CC_HIP(cc::launch_scan(c, (hipStream_t)stream));
    return CC_OK;
}

int cc_gated_scan_backward(const void* x, int64_t x_stride_b, int64_t x_stride_t, const void* gate, int64_t gate_stride_b,
                           int64_t gate_stride_t, int32_t dtype, int64_t B, int64_t T, int64_t D, const int32_t* lengths,
                           const float* states, const void* grad_h, int64_t grad_h_stride_b, int64_t grad_h_stride_t,
                           const float* grad_last, void* grad_x, int64_t grad_x_stride_b, int64_t grad_x_stride_t,
                           void* grad_gate, int64_t grad_gate_stride_b, int64_t grad_gate_stride_t, float* grad_h0,
                           void* workspace, size_t workspace_bytes, void* stream) {
    if (!is_dtype(dtype) || !scan_sizes(B, T, D)) return CC_ERR_INVALID_ARG;
    if (!strides_ok(x_stride_b, x_stride_t) || !strides_ok(gate_stride_b, gate_stride_t) || !strides_ok(grad_h_stride_b, grad_h_stride_t) ||
        !separate(B, grad_x_stride_b, T, grad_x_stride_t, D) || !separate(B, grad_gate_stride_b, T, grad_gate_stride_t, D))
        return CC_ERR_INVALID_ARG;
    if (B == 0) return CC_OK;
    const uintptr_t e = below(dtype);
    if (T > 0 && (!have(x, e) || !have(gate, e) || !have(grad_h, e) || !have(grad_x, e) || !have(grad_gate, e) || !have(states, 3u)))
        return CC_ERR_INVALID_ARG;
    if (!aligned(lengths, 3u) || !aligned(grad_last, 3u) || !aligned(grad_h0, 3u)) return CC_ERR_INVALID_ARG;
    if (!workspace_ok(workspace, workspace_bytes, cc::scan_workspace_bytes(B, T, D))) return CC_ERR_WORKSPACE;
    cc::ScanCall c = {};
    c.x = {const_cast<void*>(x), x_stride_b, x_stride_t};
    c.gate = {const_cast<void*>(gate), gate_stride_b, gate_stride_t};
    c.dtype = dtype;
    c.B = B;
    c.T = T;
    c.D = D;
    c.lengths = lengths;
    c.h = {const_cast<void*>(grad_h), grad_h_stride_b, grad_h_stride_t};
    c.last = const_cast<float*>(grad_last);
    c.states = const_cast<float*>(states);
    c.grad_x = {grad_x, grad_x_stride_b, grad_x_stride_t};
    c.grad_gate = {grad_gate, grad_gate_stride_b, grad_gate_stride_t};
    c.grad_h0 = grad_h0;
    c.workspace = workspace;
    CC_HIP(cc::poison_lds_if_asked((hipStream_t)stream));
    CC_HIP(cc::launch_scan_backward(c, (hipStream_t)stream));
    return CC_OK;
}

int cc_token_logprob(const void* logits, int32_t dtype, int64_t B, int64_t T, int64_t V, int64_t stride_b, int64_t stride_t,
                     const int32_t* tokens, const uint8_t* mask, int32_t placed, float scale, float* logprob, float* rows,
                     void* stream) {
    if (int rc = check_tokens(logits, dtype, B, T, V, stride_b, stride_t, tokens, placed, scale, nullptr, 0, 0)) return rc;
    if (B == 0 || T == 0) return CC_OK;
    if (!have(logprob, 3u) || !aligned(rows, 7u)) return CC_ERR_INVALID_ARG;
    cc::TokenCall c = token_call(logits, dtype, B, T, V, stride_b, stride_t, tokens, mask, placed, scale);
    c.logprob = logprob;
    c.rows = rows;
    CC_HIP(cc::poison_lds_if_asked((hipStream_t)stream));
    CC_HIP(cc::launch_token(cc::kTokenForward, c, (hipStream_t)stream));
    return CC_OK;
}

int cc_token_logprob_backward(const void* logits, int32_t dtype, int64_t B, int64_t T, int64_t V, int64_t stride_b,
                              int64_t stride_t, const int32_t* tokens, const uint8_t* mask, int32_t placed, float scale,
                              const float* rows, const float* grad_logprob, float grad_scale, void* grad_logits,
                              int64_t grad_stride_b, int64_t grad_stride_t, void* stream) {
    if (int rc = check_tokens(logits, dtype, B, T, V, stride_b, stride_t, tokens, placed, scale, grad_logits, grad_stride_b, grad_stride_t))
        return rc;
    if (!std::isfinite(grad_scale)) return CC_ERR_INVALID_ARG;
    if (B == 0 || T == 0) return CC_OK;
    if (!have(rows, 7u) || !have(grad_logprob, 3u) || !grad_logits) return CC_ERR_INVALID_ARG;
    cc::TokenCall c = token_call(logits, dtype, B, T, V, stride_b, stride_t, tokens, mask, placed, scale);
    c.rows = const_cast<float*>(rows);
    c.slope = grad_logprob;
    c.grad_scale = grad_scale;
    c.grad = grad_logits;
    c.grad_stride_b = grad_stride_b;
    c.grad_stride_t = grad_stride_t;
    CC_HIP(cc::poison_lds_if_asked((hipStream_t)stream));
    CC_HIP(cc::launch_token(cc::kTokenBackward, c, (hipStream_t)stream));
    return CC_OK;
}

size_t cc_token_workspace_bytes(int64_t B, int64_t T) { return token_sizes(B, T, 1) ? cc::token_workspace_bytes(B, T) : 0; }

int cc_policy_loss(const void* logits, int32_t dtype, int64_t B, int64_t T, int64_t V, int64_t stride_b, int64_t stride_t,
                   const int32_t* tokens, const uint8_t* mask, int32_t placed, float scale, const float* old_logprob,
                   const float* ref_logprob, const float* advantage, int32_t advantage_per_token, float clip_low,
                   float clip_high, float kl_coef, int32_t mean, float grad_scale, float* stats, float* logprob,
                   void* grad_logits, int64_t grad_stride_b, int64_t grad_stride_t, void* workspace, size_t workspace_bytes,
                   void* stream) {
    if (int rc = check_tokens(logits, dtype, B, T, V, stride_b, stride_t, tokens, placed, scale, grad_logits, grad_stride_b, grad_stride_t))
        return rc;
    if (!(clip_low >= 0.0f) || !(clip_low <= 1.0f) || !(clip_high >= 0.0f) || !std::isfinite(clip_high) || !std::isfinite(kl_coef) ||
        !std::isfinite(grad_scale) || (mean != CC_MEAN_TOKENS && mean != CC_MEAN_ORDERS))
        return CC_ERR_INVALID_ARG;
    if (!have(stats, 3u)) return CC_ERR_INVALID_ARG;
    if (B > 0 && T > 0 && (!have(old_logprob, 3u) || !aligned(ref_logprob, 3u) || !have(advantage, 3u) || !have(logprob, 3u)))
        return CC_ERR_INVALID_ARG;
    if (!workspace_ok(workspace, workspace_bytes, cc::token_workspace_bytes(B, T))) return CC_ERR_WORKSPACE;
    cc::TokenCall c = token_call(logits, dtype, B, T, V, stride_b, stride_t, tokens, mask, placed, scale);
    c.old = old_logprob;
    c.ref = ref_logprob;
    c.advantage = advantage;
    c.advantage_per_token = advantage_per_token != 0;
    c.clip_low = clip_low;
    c.clip_high = clip_high;
    c.kl_coef = kl_coef;
    c.mean_of_orders = mean == CC_MEAN_ORDERS;
    c.grad_scale = grad_scale;
    c.stats = stats;
    c.logprob = logprob;
    c.grad = grad_logits;
    c.grad_stride_b = grad_stride_b;
    c.grad_stride_t = grad_stride_t;
    c.workspace = workspace;
    CC_HIP(cc::poison_lds_if_asked((hipStream_t)stream));
    CC_HIP(cc::launch_token(cc::kTokenPolicy, c, (hipStream_t)stream));
    return CC_OK;
}

int cc_preference_loss(const void* logits, int32_t dtype, int64_t B, int64_t T, int64_t V, int64_t stride_b, int64_t stride_t,
                       const int32_t* tokens, const uint8_t* mask, int32_t placed, float scale, const float* ref_logprob,
                       float beta, float label_smoothing, float grad_scale, float* loss, float* margin, float* logprob,
                       void* grad_logits, int64_t grad_stride_b, int64_t grad_stride_t, void* workspace,
                       size_t workspace_bytes, void* stream) {
    if (int rc = check_tokens(logits, dtype, B, T, V, stride_b, stride_t, tokens, placed, scale, grad_logits, grad_stride_b, grad_stride_t))
        return rc;
    if ((B & 1) || !std::isfinite(beta) || !(label_smoothing >= 0.0f) || !(label_smoothing <= 1.0f) || !std::isfinite(grad_scale))
        return CC_ERR_INVALID_ARG;
    if (!have(loss, 3u) || (B > 0 && !have(margin, 3u))) return CC_ERR_INVALID_ARG;
    if (B > 0 && T > 0 && (!aligned(ref_logprob, 3u) || !have(logprob, 3u))) return CC_ERR_INVALID_ARG;
    if (!workspace_ok(workspace, workspace_bytes, cc::token_workspace_bytes(B, T))) return CC_ERR_WORKSPACE;
    cc::TokenCall c = token_call(logits, dtype, B, T, V, stride_b, stride_t, tokens, mask, placed, scale);
    c.ref = ref_logprob;
    c.beta = beta;
    c.smoothing = label_smoothing;
    c.grad_scale = grad_scale;
    c.stats = loss;
    c.margin = margin;
    c.logprob = logprob;
    c.grad = grad_logits;
    c.grad_stride_b = grad_stride_b;
    c.grad_stride_t = grad_stride_t;
    c.workspace = workspace;
    CC_HIP(cc::poison_lds_if_asked((hipStream_t)stream));
    CC_HIP(cc::launch_token(cc::kTokenPreference, c, (hipStream_t)stream));
    return CC_OK;
}

int cc_rms_norm(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, int32_t dtype, int64_t n,
                int64_t D, const void* weight, int32_t weight_dtype, float eps, void* sum, int64_t sum_stride, void* out,
                int64_t out_stride, int8_t* q, int64_t q_stride, float* scale, float* rstd, void* stream) {
    if (!is_dtype(dtype) || !norm_sizes(n, D) || !strides_ok(x_stride, residual_stride) || !(eps > 0.0f) || !std::isfinite(eps))
        return CC_ERR_INVALID_ARG;
    if (weight && weight_dtype != CC_F32 && weight_dtype != dtype) return CC_ERR_INVALID_ARG;
    if ((q == nullptr) != (scale == nullptr)) return CC_ERR_INVALID_ARG;
    if (n == 0) return CC_OK;
    const uintptr_t e = below(dtype);
    if (!have(x, e) || !aligned(residual, e) || !aligned(weight, below(weight_dtype)) || !aligned(sum, e) || !aligned(out, e) ||
        !aligned(scale, 3u) || !aligned(rstd, 3u))
        return CC_ERR_INVALID_ARG;
    if ((sum && !separate(1, 0, n, sum_stride, D)) || (out && !separate(1, 0, n, out_stride, D)) || (q && !separate(1, 0, n, q_stride, D)))
        return CC_ERR_INVALID_ARG;
    if (sum && (!in_place_ok(sum, sum_stride, x, x_stride) || !in_place_ok(sum, sum_stride, residual, residual_stride))) return CC_ERR_INVALID_ARG;
    cc::NormCall c = {};
    c.x = x;
    c.residual = residual;
    c.weight = weight;
    c.dtype = dtype;
    c.weight_dtype = weight ? weight_dtype : dtype;
    c.n = n;
    c.D = D;
    c.x_stride = x_stride;
    c.residual_stride = residual_stride;
    c.sum_stride = sum_stride;
    c.out_stride = out_stride;
    c.q_stride = q_stride;
    c.eps = eps;
    c.sum = sum;
    c.out = out;
    c.q = q;
    c.scale = scale;
    c.rstd = rstd;
    CC_HIP(cc::poison_lds_if_asked((hipStream_t)stream));
    CC_HIP(cc::launch_norm(c, (hipStream_t)stream));
    return CC_OK;
}

size_t cc_rms_norm_workspace_bytes(int64_t n, int64_t D) { return norm_sizes(n, D) ? cc::norm_workspace_bytes(n, D) : 0; }

int cc_rms_norm_backward(const void* grad_out, int64_t grad_out_stride, const void* h, int64_t h_stride, int32_t dtype, int64_t n,
                         int64_t D, const void* weight, int32_t weight_dtype, const float* rstd, const void* grad_sum,
                         int64_t grad_sum_stride, void* grad_h, int64_t grad_h_stride, void* grad_weight,
                         int32_t grad_weight_dtype, int32_t accumulate, void* workspace, size_t workspace_bytes, void* stream) {
    if (!is_dtype(dtype) || !norm_sizes(n, D) || !strides_ok(grad_out_stride, h_stride) || grad_sum_stride < 0) return CC_ERR_INVALID_ARG;
    if (weight && weight_dtype != CC_F32 && weight_dtype != dtype) return CC_ERR_INVALID_ARG;
    if (grad_weight && (!weight || (grad_weight_dtype != CC_F32 && grad_weight_dtype != weight_dtype) || !aligned(grad_weight, below(grad_weight_dtype))))
        return CC_ERR_INVALID_ARG;
    const uintptr_t e = below(dtype);
    if (n > 0) {
        if (!have(grad_out, e) || !have(h, e) || !aligned(weight, below(weight_dtype)) || !have(rstd, 3u) || !aligned(grad_sum, e) || !have(grad_h, e))
            return CC_ERR_INVALID_ARG;
        if (!separate(1, 0, n, grad_h_stride, D) || !in_place_ok(grad_h, grad_h_stride, grad_out, grad_out_stride) ||
            !in_place_ok(grad_h, grad_h_stride, grad_sum, grad_sum_stride))
            return CC_ERR_INVALID_ARG;
        if (grad_weight && !workspace_ok(workspace, workspace_bytes, cc::norm_workspace_bytes(n, D))) return CC_ERR_WORKSPACE;
    }
    if (n == 0 && (!grad_weight || accumulate)) return CC_OK;
    cc::NormBackwardCall c = {};
    c.grad = grad_out;
    c.h = h;
    c.weight = weight;
    c.grad_sum = grad_sum;
    c.rstd = rstd;
    c.dtype = dtype;
    c.weight_dtype = weight ? weight_dtype : dtype;
    c.grad_weight_dtype = grad_weight_dtype;
    c.n = n;
    c.D = D;
    c.grad_stride = grad_out_stride;
    c.h_stride = h_stride;
    c.grad_sum_stride = grad_sum_stride;
    c.grad_h_stride = grad_h_stride;
    c.grad_h = grad_h;
    c.grad_weight = grad_weight;
    c.accumulate = accumulate != 0;
    c.workspace = workspace;
    CC_HIP(cc::poison_lds_if_asked((hipStream_t)stream));
    CC_HIP(cc::launch_norm_backward(c, (hipStream_t)stream));
    return CC_OK;
}

int cc_quantize_rows(const void* x, int64_t x_stride, int32_t dtype, int64_t n, int64_t D, int8_t* q, int64_t q_stride,
                     float* scale, void* stream) {
    if (!is_dtype(dtype) || !norm_sizes(n, D) || x_stride < 0 || !separate(1, 0, n, q_stride, D)) return CC_ERR_INVALID_ARG;
    if (n == 0) return CC_OK;
    if (!have(x, below(dtype)) || !q || !have(scale, 3u)) return CC_ERR_INVALID_ARG;
    cc::NormCall c = {};
    c.x = x;
    c.dtype = dtype;
    c.n = n;
    c.D = D;
    c.x_stride = x_stride;
    c.q_stride = q_stride;
    c.q = q;
    c.scale = scale;
    CC_HIP(cc::poison_lds_if_asked((hipStream_t)stream));
    CC_HIP(cc::launch_quantize(c, (hipStream_t)stream));
    return CC_OK;
}

size_t cc_product_i8_workspace_bytes(int64_t M, int64_t N, int64_t K) { return product_sizes(M, N, K) ? cc::product_workspace_bytes(M, N, K) : 0; }

int cc_product_i8(const int8_t* x, int64_t x_stride, const float* x_scale, const int8_t* w, int64_t w_stride, const float* w_scale,
                  const float* bias, int64_t M, int64_t N, int64_t K, void* out, int64_t out_stride, int32_t dtype,
                  void* workspace, size_t workspace_bytes, void* stream) {
    if (!is_dtype(dtype) || !product_sizes(M, N, K) || !strides_ok(x_stride, w_stride) || !separate(1, 0, M, out_stride, N))
        return CC_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return CC_OK;
    if ((K > 0 && (!x || !w)) || !have(x_scale, 3u) || !have(w_scale, 3u) || !aligned(bias, 3u) || !have(out, below(dtype))) return CC_ERR_INVALID_ARG;
    if (!workspace_ok(workspace, workspace_bytes, cc::product_workspace_bytes(M, N, K))) return CC_ERR_WORKSPACE;
    cc::ProductCall c = {};
    c.x = x;
    c.w = w;
    c.x_scale = x_scale;
    c.w_scale = w_scale;
    c.bias = bias;
    c.M = M;
    c.N = N;
    c.K = K;
    c.x_stride = x_stride;
    c.w_stride = w_stride;
    c.out = out;
    c.out_stride = out_stride;
    c.dtype = dtype;
    c.workspace = workspace;
    CC_HIP(cc::poison_lds_if_asked((hipStream_t)stream));
    CC_HIP(cc::launch_product(c, (hipStream_t)stream));
    return CC_OK;
}

int cc_shape_logits(const void* logits, int32_t dtype, int64_t B, int64_t T, int64_t V, int64_t stride_b, int64_t stride_t,
                    const int32_t* history, int64_t L, int64_t history_stride, const int32_t* lengths, const int32_t* starts,
                    const float* penalties, const float* bias, int64_t bias_stride, const uint32_t* allowed,
                    int64_t allowed_stride_b, int64_t allowed_stride_t, void* out, int64_t out_stride_b, int64_t out_stride_t,
                    void* stream) {
    if (int rc = check_shape(logits, dtype, B, T, V, stride_b, stride_t, history, L, history_stride, lengths, starts, penalties, bias, bias_stride,
                             allowed, allowed_stride_b, allowed_stride_t, out, out_stride_b, out_stride_t))
        return rc;
    if (B == 0 || T == 0) return CC_OK;
    if (out == logits && (out_stride_b != stride_b || out_stride_t != stride_t)) return CC_ERR_INVALID_ARG;
    const cc::ShapeCall c = shape_call(logits, dtype, B, T, V, stride_b, stride_t, history, L, history_stride, lengths, starts, penalties, bias,
                                       bias_stride, allowed, allowed_stride_b, allowed_stride_t, out, out_stride_b, out_stride_t);
    CC_HIP(cc::poison_lds_if_asked((hipStream_t)stream));
    CC_HIP(cc::launch_shape(c, (hipStream_t)stream));
    return CC_OK;
}

int cc_shape_logits_backward(const void* grad_out, int64_t grad_stride_b, int64_t grad_stride_t, const void* logits, int32_t dtype,
                             int64_t B, int64_t T, int64_t V, int64_t stride_b, int64_t stride_t, const int32_t* history, int64_t L,
                             int64_t history_stride, const int32_t* lengths, const int32_t* starts, const float* penalties,
                             const float* bias, int64_t bias_stride, const uint32_t* allowed, int64_t allowed_stride_b,
                             int64_t allowed_stride_t, void* grad_logits, int64_t out_stride_b, int64_t out_stride_t, void* stream) {
    if (int rc = check_shape(logits, dtype, B, T, V, stride_b, stride_t, history, L, history_stride, lengths, starts, penalties, bias, bias_stride,
                             allowed, allowed_stride_b, allowed_stride_t, grad_logits, out_stride_b, out_stride_t))
        return rc;
    if (!strides_ok(grad_stride_b, grad_stride_t)) return CC_ERR_INVALID_ARG;
    if (B == 0 || T == 0) return CC_OK;
    if (!have(grad_out, below(dtype))) return CC_ERR_INVALID_ARG;
    if (grad_logits == grad_out && (out_stride_b != grad_stride_b || out_stride_t != grad_stride_t)) return CC_ERR_INVALID_ARG;
    cc::ShapeCall c = shape_call(logits, dtype, B, T, V, stride_b, stride_t, history, L, history_stride, lengths, starts, penalties, bias,
                                 bias_stride, allowed, allowed_stride_b, allowed_stride_t, grad_logits, out_stride_b, out_stride_t);
    c.grad = grad_out;
    c.grad_stride_b = grad_stride_b;
    c.grad_stride_t = grad_stride_t;
    CC_HIP(cc::poison_lds_if_asked((hipStream_t)stream));
    CC_HIP(cc::launch_shape(c, (hipStream_t)stream));
    return CC_OK;
}

}  // extern "C"
