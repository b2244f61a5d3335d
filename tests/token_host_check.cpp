// Host-only exerciser of the argument checks of the operators around the layers, built with AddressSanitizer and
// UndefinedBehaviorSanitizer on the host side (tests/test_token_sanitizers.py compiles and runs it). Every call below is
// refused before any GPU call.
#include <climits>
#include <cmath>
#include <cstdio>
#include <vector>

#include "fasth.h"

static int failures = 0;
#define EXPECT(call, want)                                                              \
  do {                                                                                  \
    const long long got_ = (long long)(call);                                           \
    if (got_ != (long long)(want)) {                                                    \
      std::printf("FAIL %s: got %lld, want %lld\n", #call, got_, (long long)(want));    \
      ++failures;                                                                       \
    }                                                                                   \
  } while (0)

int main() {
  float* p = reinterpret_cast<float*>(256);    // aligned, never dereferenced on the host
  float* odd = reinterpret_cast<float*>(260);  // not 16-byte aligned
  int* pi = reinterpret_cast<int*>(256);
  const size_t big = (size_t)1 << 50;

  const fasth_embed_shape embed = {100, 64, 32, FASTH_BF16, 64}, most = {1 << 24, 16384, 65535, FASTH_F32, 64};
  EXPECT(fasth_embed_workspace_bytes(&most) > (size_t)16384 * 65535 * 4, 1);
  EXPECT(fasth_embed_workspace_bytes(nullptr), 0);
  for (int v : {INT_MIN, -1, 0}) {
    const fasth_embed_shape a = {v, 64, 32, 0, 64}, b = {100, v, 32, 0, 64}, c = {100, 64, v, 0, 64};
    for (const fasth_embed_shape* s : {&a, &b, &c}) {
      EXPECT(fasth_embed_workspace_bytes(s), 0);
      EXPECT(fasth_embed(s, p, p, 1.f, p, nullptr), FASTH_EINVAL);
      EXPECT(fasth_embed_backward(s, p, p, 1.f, p, p, big, nullptr), FASTH_EINVAL);
    }
  }
  const fasth_embed_shape huge = {INT_MAX, INT_MAX, INT_MAX, 0, 64};
  EXPECT(fasth_embed(&huge, p, p, 1.f, p, nullptr), FASTH_EUNSUPPORTED);
  EXPECT(fasth_embed(nullptr, p, p, 1.f, p, nullptr), FASTH_EINVAL);
  EXPECT(fasth_embed(&embed, p, nullptr, 1.f, p, nullptr), FASTH_EINVAL);
  EXPECT(fasth_embed(&embed, odd, p, 1.f, p, nullptr), FASTH_EALIGN);
  EXPECT(fasth_embed_backward(&embed, p, p, 1.f, p, p, fasth_embed_workspace_bytes(&embed) - 1, nullptr), FASTH_EWORKSPACE);

  const fasth_norm_shape norm = {64, 32, FASTH_F16, 1e-5f}, largest = {16384, 65535, FASTH_F32, 1e-5f};
  EXPECT(fasth_norm_workspace_bytes(&largest) > 0, 1);
  for (float eps : {0.f, -1.f, INFINITY, -INFINITY, NAN}) {
    const fasth_norm_shape s = {64, 32, 0, eps};
    EXPECT(fasth_norm_workspace_bytes(&s), 0);
    EXPECT(fasth_norm(&s, p, nullptr, p, nullptr, p, p, nullptr), FASTH_EINVAL);
  }
  const fasth_norm_shape wide = {64, INT_MAX, 0, 1e-5f}, tall = {INT_MAX, 4, 0, 1e-5f};
  EXPECT(fasth_norm(&wide, p, nullptr, p, nullptr, p, p, nullptr), FASTH_EUNSUPPORTED);
  EXPECT(fasth_norm(&tall, p, nullptr, p, nullptr, p, p, nullptr), FASTH_EUNSUPPORTED);
  EXPECT(fasth_norm(&norm, p, p, p, nullptr, p, p, nullptr), FASTH_EINVAL);
  EXPECT(fasth_norm(&norm, p, nullptr, p, p, p, p, nullptr), FASTH_EINVAL);
  EXPECT(fasth_norm(&norm, p, odd, p, p, p, p, nullptr), FASTH_EALIGN);
  EXPECT(fasth_norm_backward(&norm, p, p, p, p, odd, p, nullptr, p, big, nullptr), FASTH_EALIGN);
  EXPECT(fasth_norm_backward(&norm, p, p, p, p, nullptr, p, p, p, 0, nullptr), FASTH_EWORKSPACE);

  const fasth_log_prob_shape prob = {1000, 32, FASTH_F32, 32, 3}, last = {1 << 21, 65535, FASTH_BF16, 64, 32};
  EXPECT(fasth_log_prob_workspace_bytes(&last) > 0, 1);
  for (int top : {INT_MIN, -1, 33, INT_MAX}) {
    const fasth_log_prob_shape s = {1000, 32, 0, 64, top};
    EXPECT(fasth_log_prob_workspace_bytes(&s), 0);
    EXPECT(fasth_log_prob(&s, p, p, p, p, p, p, pi, p, big, nullptr), top < 0 ? FASTH_EINVAL : FASTH_EUNSUPPORTED);
  }
  EXPECT(fasth_log_prob(&prob, p, p, p, p, p, nullptr, nullptr, p, big, nullptr), FASTH_EINVAL);
  EXPECT(fasth_log_prob(&prob, p, p, p, p, p, p, pi, p, 64, nullptr), FASTH_EWORKSPACE);
  EXPECT(fasth_log_prob(&prob, p, odd, p, p, p, p, pi, p, big, nullptr), FASTH_EALIGN);
  EXPECT(fasth_log_prob_backward(&prob, p, p, p, p, nullptr, nullptr, p, nullptr), FASTH_EINVAL);
  EXPECT(fasth_log_prob_backward(&prob, p, nullptr, p, p, p, nullptr, p, nullptr), FASTH_EINVAL);

  std::vector<fasth_tensor> many(1000);  // 16 MiB apart
  for (size_t i = 0; i < many.size(); ++i) many[i] = {reinterpret_cast<void*>((i + 1) << 24), 1000, FASTH_F32};
  std::vector<void*> out(many.size());
  for (size_t i = 0; i < many.size(); ++i) out[i] = reinterpret_cast<void*>(((i + 1) << 24) + (1 << 20));
  EXPECT(fasth_grad_workspace_bytes(many.data(), 1000) > 0, 1);
  EXPECT(fasth_grad_workspace_bytes(nullptr, 3), 0);
  EXPECT(fasth_grad_norm(many.data(), INT_MIN, p, p, big, nullptr), FASTH_EINVAL);
  EXPECT(fasth_grad_norm(many.data(), 1000, p, p, 8, nullptr), FASTH_EWORKSPACE);
  out[999] = reinterpret_cast<void*>(((size_t)500 << 24) + 3984);  // the last entries of the 500th tensor
  EXPECT(fasth_grad_clip(many.data(), out.data(), 1000, 1.f, p, p, big, nullptr), FASTH_EINVAL);
  out[999] = out[0];
  EXPECT(fasth_grad_clip(many.data(), out.data(), 1000, 1.f, p, p, big, nullptr), FASTH_EINVAL);
  out[999] = nullptr;
  EXPECT(fasth_grad_clip(many.data(), out.data(), 1000, 1.f, p, p, big, nullptr), FASTH_EINVAL);
  many[3].data = many[2].data;
  EXPECT(fasth_grad_clip(many.data(), nullptr, 1000, 1.f, p, p, big, nullptr), FASTH_EINVAL);
  many[3].count = ~0ull;
  EXPECT(fasth_grad_clip(many.data(), nullptr, 1000, 1.f, p, p, big, nullptr), FASTH_EUNSUPPORTED);
  EXPECT(fasth_grad_clip(many.data(), nullptr, 3, NAN, p, p, big, nullptr), FASTH_EINVAL);
  EXPECT(fasth_grad_clip(many.data(), nullptr, 3, -1.f, p, p, big, nullptr), FASTH_EINVAL);

  if (failures) return 1;
  std::printf("token_host_check: ok\n");
  return 0;
}
