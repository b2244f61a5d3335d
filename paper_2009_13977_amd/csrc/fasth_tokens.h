// C entry points of the operators around the layers of a token model: argument checks, then the launchers of
// fasth_embed.h, fasth_norm.h, fasth_log_prob.h and fasth_grad.h. Included by fasth.hip behind its own entry points.
#pragma once
#include <algorithm>
#include <cstdint>
#include <vector>

#include "fasth_embed.h"
#include "fasth_norm.h"
#include "fasth_log_prob.h"
#include "fasth_grad.h"

namespace fasth {

constexpr int kMaxColumns = 65535;  // as the layers take

static bool known_dtype(int dtype) { return dtype == FASTH_F32 || dtype == FASTH_BF16 || dtype == FASTH_F16; }

static int check_embed_shape(const fasth_embed_shape* s) {
  if (!s || s->vocab < 1 || s->d < 1 || s->m < 1 || !known_dtype(s->dtype) || (s->id_bits != 32 && s->id_bits != 64)) return FASTH_EINVAL;
  return s->vocab > kEmbedMaxVocab || s->d > kMaxD || s->m > kMaxColumns ? FASTH_EUNSUPPORTED : FASTH_OK;
}
static int check_norm_shape(const fasth_norm_shape* s) {
  if (!s || s->d < 1 || s->m < 1 || !known_dtype(s->dtype) || !(s->eps > 0.f) || !(s->eps < INFINITY)) return FASTH_EINVAL;
  return s->d > kMaxD || s->m > kMaxColumns ? FASTH_EUNSUPPORTED : FASTH_OK;
}
static int check_log_prob_shape(const fasth_log_prob_shape* s) {
  if (!s || s->vocab < 1 || s->m < 1 || s->top < 0 || !known_dtype(s->dtype) || (s->id_bits != 32 && s->id_bits != 64)) return FASTH_EINVAL;
  return s->vocab > kLogitMaxVocab || s->m > kMaxColumns || s->top > FASTH_MAX_TOP ? FASTH_EUNSUPPORTED : FASTH_OK;
}
static int check_tensors(const fasth_tensor* t, int n) {
  if (n < 0 || (n > 0 && !t)) return FASTH_EINVAL;
  for (int i = 0; i < n; ++i) {
    if (!known_dtype(t[i].dtype) || (t[i].count > 0 && !t[i].data)) return FASTH_EINVAL;
    if (!aligned16(t[i].data)) return FASTH_EALIGN;
    if (t[i].count > kGradMaxCount) return FASTH_EUNSUPPORTED;
  }
  return FASTH_OK;
}

struct Span {
  uintptr_t begin, end;
  int tensor;
  bool written;
};
// Whether a written tensor overlaps anything but its own input at the very same place: the result would depend on
// which of the two came first.
static bool clip_overlaps(const fasth_tensor* t, void* const* out, int n) {
  std::vector<Span> spans;
  spans.reserve(2 * (size_t)n);
  for (int i = 0; i < n; ++i) {
    if (!t[i].count) continue;
    const size_t bytes = t[i].count * (t[i].dtype == FASTH_F32 ? 4 : 2);
    const uintptr_t src = reinterpret_cast<uintptr_t>(t[i].data), dst = out ? reinterpret_cast<uintptr_t>(out[i]) : src;
    spans.push_back({dst, dst + bytes, i, true});
    if (dst != src) spans.push_back({src, src + bytes, i, false});
  }
  std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.begin < b.begin; });
  uintptr_t written_to = 0, any_to = 0;  // the furthest ends so far
  for (const Span& s : spans) {
    if (s.begin < written_to || (s.written && s.begin < any_to)) return true;
    any_to = std::max(any_to, s.end);
    if (s.written) written_to = std::max(written_to, s.end);
  }
  return false;
}

}  // namespace fasth

using namespace fasth;

#define FASTH_BY_TYPE(dtype, CALL)                 \
  switch (dtype) {                                 \
    case FASTH_F32: { typedef float T; return CALL; }   \
    case FASTH_BF16: { typedef bf16_t T; return CALL; } \
    default: { typedef f16_t T; return CALL; }          \
  }

extern "C" {

int fasth_embed(const fasth_embed_shape* shape, const void* table, const void* ids, float scale, float* X, void* stream) {
  const int rc = check_embed_shape(shape);
  if (rc != FASTH_OK) return rc;
  if (!table || !ids || !X) return FASTH_EINVAL;
  if (!aligned16(table) || !aligned16(ids) || !aligned16(X)) return FASTH_EALIGN;
  FASTH_BY_TYPE(shape->dtype, launch_embed<T>(*shape, table, ids, scale, X, static_cast<hipStream_t>(stream)))
}

size_t fasth_embed_workspace_bytes(const fasth_embed_shape* shape) {
  return check_embed_shape(shape) == FASTH_OK ? make_embed_layout(*shape).total : 0;
}

int fasth_embed_backward(const fasth_embed_shape* shape, const void* ids, const float* G, float scale, void* dTable, void* workspace,
                         size_t workspace_bytes, void* stream) {
  const int rc = check_embed_shape(shape);
  if (rc != FASTH_OK) return rc;
  if (!ids || !G || !dTable || !workspace) return FASTH_EINVAL;
  if (!aligned16(ids) || !aligned16(G) || !aligned16(dTable) || !aligned16(workspace)) return FASTH_EALIGN;
  if (workspace_bytes < make_embed_layout(*shape).total) return FASTH_EWORKSPACE;
  FASTH_BY_TYPE(shape->dtype, launch_embed_grad<T>(*shape, ids, G, scale, dTable, workspace, static_cast<hipStream_t>(stream)))
}

int fasth_norm(const fasth_norm_shape* shape, const float* X, const float* R, const float* weight, float* S, void* Y, float* rstd,
               void* stream) {
  const int rc = check_norm_shape(shape);
  if (rc != FASTH_OK) return rc;
  if (!X || !weight || !Y || !rstd || !R != !S) return FASTH_EINVAL;
  if (!aligned16(X) || !aligned16(R) || !aligned16(weight) || !aligned16(S) || !aligned16(Y) || !aligned16(rstd)) return FASTH_EALIGN;
  NormArgs a;
  a.X = X; a.R = R; a.w = weight; a.S = S; a.Y = Y; a.rstd = rstd;
  a.d = shape->d; a.m = shape->m; a.eps = shape->eps;
  FASTH_BY_TYPE(shape->dtype, launch_norm<T>(a, static_cast<hipStream_t>(stream)))
}

size_t fasth_norm_workspace_bytes(const fasth_norm_shape* shape) {
  return check_norm_shape(shape) == FASTH_OK ? norm_workspace(*shape) : 0;
}

int fasth_norm_backward(const fasth_norm_shape* shape, const void* G, const float* S, const float* weight, const float* rstd,
                        const float* dS, float* dX, float* dweight, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_norm_shape(shape);
  if (rc != FASTH_OK) return rc;
  if (!G || !S || !weight || !rstd || !dX || !workspace) return FASTH_EINVAL;
  if (!aligned16(G) || !aligned16(S) || !aligned16(weight) || !aligned16(rstd) || !aligned16(dS) || !aligned16(dX) ||
      !aligned16(dweight) || !aligned16(workspace))
    return FASTH_EALIGN;
  if (workspace_bytes < norm_workspace(*shape)) return FASTH_EWORKSPACE;
  NormGradArgs a;
  a.G = G; a.S = S; a.w = weight; a.rstd = rstd; a.dS = dS; a.dX = dX;
  a.d = shape->d; a.m = shape->m;
  FASTH_BY_TYPE(shape->dtype, launch_norm_grad<T>(a, dweight, workspace, static_cast<hipStream_t>(stream)))
}

size_t fasth_log_prob_workspace_bytes(const fasth_log_prob_shape* shape) {
  return check_log_prob_shape(shape) == FASTH_OK ? log_prob_workspace(*shape) : 0;
}

int fasth_log_prob(const fasth_log_prob_shape* shape, const void* logits, const void* ids, float* logp, float* entropy, float* stats,
                   float* top_logp, int* top_ids, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_log_prob_shape(shape);
  if (rc != FASTH_OK) return rc;
  if (!logits || !logp || !entropy || !stats || !workspace || (shape->top > 0) != (top_logp != nullptr) || !top_logp != !top_ids)
    return FASTH_EINVAL;
  if (!aligned16(logits) || !aligned16(ids) || !aligned16(logp) || !aligned16(entropy) || !aligned16(stats) || !aligned16(top_logp) ||
      !aligned16(top_ids) || !aligned16(workspace))
    return FASTH_EALIGN;
  if (workspace_bytes < log_prob_workspace(*shape)) return FASTH_EWORKSPACE;
  LogProbArgs a;
  a.logits = logits; a.ids = ids; a.logp = logp; a.entropy = entropy; a.stats = stats; a.top_logp = top_logp; a.top_ids = top_ids;
  a.id_bits = shape->id_bits; a.vocab = shape->vocab; a.m = shape->m; a.top = shape->top;
  FASTH_BY_TYPE(shape->dtype, launch_log_prob<T>(a, workspace, static_cast<hipStream_t>(stream)))
}

int fasth_log_prob_backward(const fasth_log_prob_shape* shape, const void* logits, const void* ids, const float* stats,
                            const float* entropy, const float* g_logp, const float* g_entropy, void* dlogits, void* stream) {
  const int rc = check_log_prob_shape(shape);
  if (rc != FASTH_OK) return rc;
  if (!logits || !stats || !dlogits || (!g_logp && !g_entropy) || (g_logp && !ids) || (g_entropy && !entropy)) return FASTH_EINVAL;
  if (!aligned16(logits) || !aligned16(ids) || !aligned16(stats) || !aligned16(entropy) || !aligned16(g_logp) ||
      !aligned16(g_entropy) || !aligned16(dlogits))
    return FASTH_EALIGN;
  LogProbGradArgs a;
  a.logits = logits; a.ids = ids; a.stats = stats; a.entropy = entropy; a.g_logp = g_logp; a.g_entropy = g_entropy; a.dlogits = dlogits;
  a.id_bits = shape->id_bits; a.vocab = shape->vocab; a.m = shape->m;
  FASTH_BY_TYPE(shape->dtype, launch_log_prob_grad<T>(a, static_cast<hipStream_t>(stream)))
}

size_t fasth_grad_workspace_bytes(const fasth_tensor* tensors, int n) {
  return check_tensors(tensors, n) == FASTH_OK ? grad_workspace(n) : 0;
}

int fasth_grad_norm(const fasth_tensor* tensors, int n, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_tensors(tensors, n);
  if (rc != FASTH_OK) return rc;
  if (!norm || !workspace) return FASTH_EINVAL;
  if (!aligned16(norm) || !aligned16(workspace)) return FASTH_EALIGN;
  if (workspace_bytes < grad_workspace(n)) return FASTH_EWORKSPACE;
  return launch_grads(tensors, nullptr, n, false, 0.f, norm, workspace, static_cast<hipStream_t>(stream));
}

int fasth_grad_clip(const fasth_tensor* tensors, void* const* out, int n, float max_norm, float* norm, void* workspace,
                    size_t workspace_bytes, void* stream) {
  const int rc = check_tensors(tensors, n);
  if (rc != FASTH_OK) return rc;
  if (!norm || !workspace || !(max_norm >= 0.f)) return FASTH_EINVAL;
  if (!aligned16(norm) || !aligned16(workspace)) return FASTH_EALIGN;
  for (int i = 0; out && i < n; ++i) {
    if (tensors[i].count > 0 && !out[i]) return FASTH_EINVAL;
    if (!aligned16(out[i])) return FASTH_EALIGN;
  }
  if (workspace_bytes < grad_workspace(n)) return FASTH_EWORKSPACE;
  try {
    if (clip_overlaps(tensors, out, n)) return FASTH_EINVAL;
  } catch (...) {  // no host memory for the comparison
    std::snprintf(g_hip_error_text, sizeof(g_hip_error_text), "fasth_grad_clip: out of host memory");
    return FASTH_EHIP;
  }
  return launch_grads(tensors, out, n, true, max_norm, norm, workspace, static_cast<hipStream_t>(stream));
}

}  // extern "C"
