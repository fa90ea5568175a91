// C ABI of the history encoder's operators: argument checks and dispatch.
#include "../../include/lime.h"

#include <stdarg.h>
#include <stdio.h>

#include <algorithm>

#include "encoder.hpp"

namespace {

int32_t fail(int32_t status, const char* fmt, ...) {
  char text[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(text, sizeof(text), fmt, ap);
  va_end(ap);
  return lime::set_error(status, text);
}

int32_t launched(const char* fn, hipError_t e) { return e == hipSuccess ? LIME_OK : fail(LIME_LAUNCH_FAILED, "%s: %s", fn, hipGetErrorString(e)); }

constexpr int64_t kMostRows = (int64_t{1} << 31) - 1, kMostStrideBytes = (int64_t{1} << 24) - 1;
bool known(int32_t dtype) { return dtype == LIME_F32 || dtype == LIME_BF16; }
int64_t bytes_of(int32_t dtype) { return dtype == LIME_BF16 ? 2 : 4; }

int32_t check_stride(const char* fn, const char* what, int64_t stride, int64_t width, int32_t dtype) {
  if (stride < width) return fail(LIME_INVALID_ARG, "%s: the rows of %s overlap (%lld elements apart, %lld wide)", fn, what, static_cast<long long>(stride), static_cast<long long>(width));
  if (stride * bytes_of(dtype) > kMostStrideBytes) return fail(LIME_UNSUPPORTED, "%s: the rows of %s are %lld elements apart: at most %lld bytes are", fn, what, static_cast<long long>(stride), static_cast<long long>(kMostStrideBytes));
  return LIME_OK;
}
int32_t check_workspace(const char* fn, const void* workspace, size_t given, size_t need) {
  if (!workspace || given < need) return fail(LIME_WORKSPACE_TOO_SMALL, "%s: workspace of %zu bytes needed, %zu given", fn, need, workspace ? given : 0);
  if (reinterpret_cast<uintptr_t>(workspace) % 256 != 0) return fail(LIME_INVALID_ARG, "%s: the workspace is not 256-byte aligned", fn);
  return LIME_OK;
}
#define CHECK(expr)                     \
  do {                                  \
    if (int32_t st_ = (expr)) return st_; \
  } while (0)

// ----------------------------------------------------------------------------- norms and rotation
int32_t check_rotary(const char* fn, int64_t rows, int32_t hq, int32_t hk, int32_t dh, float base, float eps, int32_t dtype) {
  if (!known(dtype)) return fail(LIME_INVALID_ARG, "%s: unknown dtype %d", fn, dtype);
  if (rows <= 0 || hq <= 0 || hk < 0 || dh <= 0) return fail(LIME_INVALID_ARG, "%s: rows, hq and dh must be positive, hk not negative (rows=%lld hq=%d hk=%d dh=%d)", fn, static_cast<long long>(rows), hq, hk, dh);
  if (dh % 2 != 0) return fail(LIME_INVALID_ARG, "%s: dh=%d is odd: its elements are turned in pairs", fn, dh);
  if (!(base > 0.f) || !(eps >= 0.f)) return fail(LIME_INVALID_ARG, "%s: base must be positive and eps not negative", fn);
  if (dh > lime::kMaxRotaryHead) return fail(LIME_UNSUPPORTED, "%s: dh=%d exceeds %d", fn, dh, lime::kMaxRotaryHead);
  if (rows > kMostRows || std::max(hq, hk) > 65535) return fail(LIME_UNSUPPORTED, "%s: rows or heads beyond the limit", fn);
  return LIME_OK;
}

// ----------------------------------------------------------------------------- attention
int32_t check_sequences(const char* fn, const lime_sequences* w, int32_t hq, int32_t hk, int32_t dh, int32_t dtype) {
  if (!known(dtype)) return fail(LIME_INVALID_ARG, "%s: unknown dtype %d", fn, dtype);
  if (!w) return fail(LIME_INVALID_ARG, "%s: a required pointer is NULL", fn);
  if (w->B <= 0 || hq <= 0 || hk <= 0 || dh <= 0) return fail(LIME_INVALID_ARG, "%s: B, hq, hk, dh must be positive (B=%d hq=%d hk=%d dh=%d)", fn, w->B, hq, hk, dh);
  if (w->q_rows < 0 || w->k_rows < 0 || w->max_q < 0 || w->max_k < 0) return fail(LIME_INVALID_ARG, "%s: rows and longest slots must not be negative", fn);
  if (hq % hk != 0) return fail(LIME_INVALID_ARG, "%s: hq=%d is not a multiple of hk=%d", fn, hq, hk);
  if (dh > lime::kMaxSequenceHead) return fail(LIME_UNSUPPORTED, "%s: dh=%d exceeds %d", fn, dh, lime::kMaxSequenceHead);
  if (w->q_rows > kMostRows || w->k_rows > kMostRows) return fail(LIME_UNSUPPORTED, "%s: at most %lld rows", fn, static_cast<long long>(kMostRows));
  if (w->B > 65535 || hq > 65535) return fail(LIME_UNSUPPORTED, "%s: B=%d or hq=%d exceeds 65535", fn, w->B, hq);
  if (!w->q_offsets || !w->k_offsets) return fail(LIME_INVALID_ARG, "%s: offsets are required", fn);
  return LIME_OK;
}

lime::SequenceAttention describe(const lime_sequences* w, int32_t hq, int32_t hk, int32_t dh, float scale, int32_t causal, int32_t dtype) {
  lime::SequenceAttention a{};
  a.q_offsets = w->q_offsets, a.q_lens = w->q_lens, a.k_offsets = w->k_offsets, a.k_lens = w->k_lens;
  // (a slot is no longer than its tensor)
  a.q_rows = w->q_rows, a.k_rows = w->k_rows, a.B = w->B;
  a.max_q = static_cast<int>(std::min<int64_t>(w->max_q, w->q_rows)), a.max_k = static_cast<int>(std::min<int64_t>(w->max_k, w->k_rows));
  a.hq = hq, a.hk = hk, a.dh = dh, a.scale = scale, a.causal = causal, a.dtype = dtype;
  return a;
}

// ----------------------------------------------------------------------------- the loss
int32_t check_catalogue(const char* fn, int64_t rows, int32_t n_items, int32_t d, int32_t dtype) {
  if (!known(dtype)) return fail(LIME_INVALID_ARG, "%s: unknown dtype %d", fn, dtype);
  if (rows <= 0 || n_items <= 0 || d <= 0) return fail(LIME_INVALID_ARG, "%s: rows, n_items and d must be positive (rows=%lld n_items=%d d=%d)", fn, static_cast<long long>(rows), n_items, d);
  if (d > lime::kMaxCatalogueWidth) return fail(LIME_UNSUPPORTED, "%s: d=%d exceeds %d", fn, d, lime::kMaxCatalogueWidth);
  if (!lime::catalogue_loss_fits(rows, n_items)) return fail(LIME_UNSUPPORTED, "%s: rows=%lld or n_items=%d beyond the limit", fn, static_cast<long long>(rows), n_items);
  return LIME_OK;
}

}  // namespace

extern "C" {
#pragma GCC visibility push(default)

int32_t lime_norm_rotary(const void* Q, int64_t q_stride, const void* K, int64_t k_stride, const void* gamma_q, const void* gamma_k,
                         const int32_t* positions, float base, float eps, void* QO, int64_t qo_stride, void* KO, int64_t ko_stride,
                         int64_t rows, int32_t hq, int32_t hk, int32_t dh, int32_t dtype, void* stream) {
  const char* fn = "lime_norm_rotary";
  CHECK(check_rotary(fn, rows, hq, hk, dh, base, eps, dtype));
  if (!Q || !QO || (hk > 0 && (!K || !KO))) return fail(LIME_INVALID_ARG, "%s: a required pointer is NULL", fn);
  CHECK(check_stride(fn, "Q", q_stride, int64_t{hq} * dh, dtype));
  CHECK(check_stride(fn, "QO", qo_stride, int64_t{hq} * dh, dtype));
  if (hk > 0) {
    CHECK(check_stride(fn, "K", k_stride, int64_t{hk} * dh, dtype));
    CHECK(check_stride(fn, "KO", ko_stride, int64_t{hk} * dh, dtype));
  }
  lime::NormRotary a{};
  a.x[0] = Q, a.x[1] = K, a.out[0] = QO, a.out[1] = KO, a.gamma[0] = gamma_q, a.gamma[1] = gamma_k;
  a.x_stride[0] = q_stride, a.x_stride[1] = k_stride, a.out_stride[0] = qo_stride, a.out_stride[1] = ko_stride;
  a.heads[0] = hq, a.heads[1] = hk, a.positions = positions, a.rows = rows, a.dh = dh, a.dtype = dtype, a.base = base, a.eps = eps;
  if (!lime::norm_rotary_fits(a)) return fail(LIME_UNSUPPORTED, "%s: rows=%lld beyond the limit", fn, static_cast<long long>(rows));
  return launched(fn, lime::norm_rotary(a, static_cast<hipStream_t>(stream)));
}

size_t lime_norm_rotary_backward_workspace_bytes(int64_t rows, int32_t dh) {
  return rows <= 0 || dh <= 0 || dh % 2 != 0 || dh > lime::kMaxRotaryHead ? 0 : lime::norm_rotary_backward_workspace(rows, dh);
}

int32_t lime_norm_rotary_backward(const void* dQO, int64_t dqo_stride, const void* dKO, int64_t dko_stride, const void* Q, int64_t q_stride,
                                  const void* K, int64_t k_stride, const void* gamma_q, const void* gamma_k, const int32_t* positions,
                                  float base, float eps, void* dQ, int64_t dq_stride, void* dK, int64_t dk_stride, void* dgamma_q,
                                  void* dgamma_k, int64_t rows, int32_t hq, int32_t hk, int32_t dh, int32_t dtype, void* workspace,
                                  size_t ws_bytes, void* stream) {
  const char* fn = "lime_norm_rotary_backward";
  CHECK(check_rotary(fn, rows, hq, hk, dh, base, eps, dtype));
  if (!dQO || !Q || !dQ || (hk > 0 && (!dKO || !K || !dK))) return fail(LIME_INVALID_ARG, "%s: a required pointer is NULL", fn);
  CHECK(check_stride(fn, "dQO", dqo_stride, int64_t{hq} * dh, dtype));
  CHECK(check_stride(fn, "Q", q_stride, int64_t{hq} * dh, dtype));
  CHECK(check_stride(fn, "dQ", dq_stride, int64_t{hq} * dh, dtype));
  if (hk > 0) {
    CHECK(check_stride(fn, "dKO", dko_stride, int64_t{hk} * dh, dtype));
    CHECK(check_stride(fn, "K", k_stride, int64_t{hk} * dh, dtype));
    CHECK(check_stride(fn, "dK", dk_stride, int64_t{hk} * dh, dtype));
  }
  CHECK(check_workspace(fn, workspace, ws_bytes, lime::norm_rotary_backward_workspace(rows, dh)));
  lime::NormRotary a{};
  a.x[0] = Q, a.x[1] = K, a.dy[0] = dQO, a.dy[1] = dKO, a.out[0] = dQ, a.out[1] = dK, a.gamma[0] = gamma_q, a.gamma[1] = gamma_k;
  a.dgamma[0] = dgamma_q, a.dgamma[1] = hk > 0 ? dgamma_k : nullptr;
  a.x_stride[0] = q_stride, a.x_stride[1] = k_stride, a.dy_stride[0] = dqo_stride, a.dy_stride[1] = dko_stride, a.out_stride[0] = dq_stride, a.out_stride[1] = dk_stride;
  a.heads[0] = hq, a.heads[1] = hk, a.positions = positions, a.rows = rows, a.dh = dh, a.dtype = dtype, a.base = base, a.eps = eps;
  if (!lime::norm_rotary_fits(a)) return fail(LIME_UNSUPPORTED, "%s: rows=%lld beyond the limit", fn, static_cast<long long>(rows));
  return launched(fn, lime::norm_rotary_backward(a, workspace, static_cast<hipStream_t>(stream)));
}

size_t lime_sequence_attention_workspace_bytes(const lime_sequences* where, int32_t hq, int32_t hk, int32_t dh, int32_t dtype, int32_t backward) {
  if (!where || !known(dtype) || where->B <= 0 || hq <= 0 || hk <= 0 || hq % hk != 0 || dh <= 0 || dh > lime::kMaxSequenceHead || where->q_rows < 0 || where->k_rows < 0 ||
      where->max_q < 0 || where->max_k < 0 || where->q_rows > kMostRows || where->k_rows > kMostRows || where->B > 65535 || hq > 65535)
    return 0;  // (within these the plan's products stay in 64 bits)
  const lime::SequenceAttention a = describe(where, hq, hk, dh, 1.f, 1, dtype);
  return backward ? lime::sequence_attention_backward_workspace(a) : lime::sequence_attention_workspace(a);
}

int32_t lime_sequence_attention(const lime_sequences* where, const void* Q, int64_t q_stride, const void* K, int64_t k_stride,
                                const void* V, int64_t v_stride, void* O, float* lse, int32_t hq, int32_t hk, int32_t dh, float scale,
                                int32_t causal, int32_t dtype, void* workspace, size_t ws_bytes, void* stream) {
  const char* fn = "lime_sequence_attention";
  CHECK(check_sequences(fn, where, hq, hk, dh, dtype));
  if ((where->q_rows > 0 && (!Q || !O)) || (where->k_rows > 0 && (!K || !V))) return fail(LIME_INVALID_ARG, "%s: a required pointer is NULL", fn);
  CHECK(check_stride(fn, "Q", q_stride, int64_t{hq} * dh, dtype));
  CHECK(check_stride(fn, "K", k_stride, int64_t{hk} * dh, dtype));
  CHECK(check_stride(fn, "V", v_stride, int64_t{hk} * dh, dtype));
  lime::SequenceAttention a = describe(where, hq, hk, dh, scale, causal, dtype);
  if (!lime::sequence_attention_fits(a)) return fail(LIME_UNSUPPORTED, "%s: more work than one launch takes (B=%d max_q=%d max_k=%d hq=%d)", fn, a.B, a.max_q, a.max_k, hq);
  CHECK(check_workspace(fn, workspace, ws_bytes, lime::sequence_attention_workspace(a)));
  a.Q = Q, a.K = K, a.V = V, a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride, a.O = O, a.lse = lse;
  if (a.max_q == 0) return LIME_OK;  // no queries
  return launched(fn, lime::sequence_attention(a, workspace, static_cast<hipStream_t>(stream)));
}

int32_t lime_sequence_attention_backward(const lime_sequences* where, const void* dO, const void* Q, int64_t q_stride, const void* K,
                                         int64_t k_stride, const void* V, int64_t v_stride, const void* O, const float* lse, void* dQ,
                                         int64_t dq_stride, void* dK, int64_t dk_stride, void* dV, int64_t dv_stride, int32_t hq,
                                         int32_t hk, int32_t dh, float scale, int32_t causal, int32_t dtype, void* workspace,
                                         size_t ws_bytes, void* stream) {
  const char* fn = "lime_sequence_attention_backward";
  CHECK(check_sequences(fn, where, hq, hk, dh, dtype));
  if ((where->q_rows > 0 && (!Q || !O || !dO || !dQ || !lse)) || (where->k_rows > 0 && (!K || !V || !dK || !dV)))
    return fail(LIME_INVALID_ARG, "%s: a required pointer is NULL", fn);
  CHECK(check_stride(fn, "Q", q_stride, int64_t{hq} * dh, dtype));
  CHECK(check_stride(fn, "K", k_stride, int64_t{hk} * dh, dtype));
  CHECK(check_stride(fn, "V", v_stride, int64_t{hk} * dh, dtype));
  CHECK(check_stride(fn, "dQ", dq_stride, int64_t{hq} * dh, dtype));
  CHECK(check_stride(fn, "dK", dk_stride, int64_t{hk} * dh, dtype));
  CHECK(check_stride(fn, "dV", dv_stride, int64_t{hk} * dh, dtype));
  CHECK(check_stride(fn, "dO", int64_t{hq} * dh, int64_t{hq} * dh, dtype));
  lime::SequenceAttention a = describe(where, hq, hk, dh, scale, causal, dtype);
  if (!lime::sequence_attention_backward_fits(a)) return fail(LIME_UNSUPPORTED, "%s: more work than one launch takes (B=%d max_q=%d max_k=%d hq=%d)", fn, a.B, a.max_q, a.max_k, hq);
  CHECK(check_workspace(fn, workspace, ws_bytes, lime::sequence_attention_backward_workspace(a)));
  a.Q = Q, a.K = K, a.V = V, a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride, a.O = const_cast<void*>(O), a.lse = const_cast<float*>(lse);
  a.dO = dO, a.dQ = dQ, a.dK = dK, a.dV = dV, a.dq_stride = dq_stride, a.dk_stride = dk_stride, a.dv_stride = dv_stride;
  return launched(fn, lime::sequence_attention_backward(a, workspace, static_cast<hipStream_t>(stream)));
}

size_t lime_catalogue_loss_workspace_bytes(int64_t rows, int32_t n_items, int32_t d, int32_t dtype, int32_t backward) {
  if (!known(dtype) || rows <= 0 || n_items <= 0 || d <= 0 || d > lime::kMaxCatalogueWidth || !lime::catalogue_loss_fits(rows, n_items)) return 0;
  return lime::catalogue_loss_workspace(rows, n_items, d, dtype, backward != 0);
}

int32_t lime_catalogue_loss(const void* X, const void* W, const int32_t* targets, float* loss, float* lse, int64_t rows, int32_t n_items,
                            int32_t d, float scale, int32_t dtype, void* workspace, size_t ws_bytes, void* stream) {
  const char* fn = "lime_catalogue_loss";
  CHECK(check_catalogue(fn, rows, n_items, d, dtype));
  if (!X || !W || !targets || !loss || !lse) return fail(LIME_INVALID_ARG, "%s: a required pointer is NULL", fn);
  CHECK(check_workspace(fn, workspace, ws_bytes, lime::catalogue_loss_workspace(rows, n_items, d, dtype, false)));
  lime::CatalogueLoss a{};
  a.X = X, a.W = W, a.targets = targets, a.loss = loss, a.lse = lse, a.rows = rows, a.items = n_items, a.d = d, a.dtype = dtype, a.scale = scale;
  return launched(fn, lime::catalogue_loss(a, workspace, static_cast<hipStream_t>(stream)));
}

int32_t lime_catalogue_loss_backward(const float* dloss, const void* X, const void* W, const int32_t* targets, const float* lse, void* dX,
                                     void* dW, int64_t rows, int32_t n_items, int32_t d, float scale, int32_t dtype, void* workspace,
                                     size_t ws_bytes, void* stream) {
  const char* fn = "lime_catalogue_loss_backward";
  CHECK(check_catalogue(fn, rows, n_items, d, dtype));
  if (!dloss || !X || !W || !targets || !lse || (!dX && !dW)) return fail(LIME_INVALID_ARG, "%s: a required pointer is NULL", fn);
  CHECK(check_workspace(fn, workspace, ws_bytes, lime::catalogue_loss_workspace(rows, n_items, d, dtype, true)));
  lime::CatalogueLoss a{};
  a.X = X, a.W = W, a.targets = targets, a.lse = const_cast<float*>(lse), a.dloss = dloss, a.dX = dX, a.dW = dW, a.rows = rows, a.items = n_items, a.d = d;
  a.dtype = dtype, a.scale = scale;
  return launched(fn, lime::catalogue_loss_backward(a, workspace, static_cast<hipStream_t>(stream)));
}

#pragma GCC visibility pop
}  // extern "C"
