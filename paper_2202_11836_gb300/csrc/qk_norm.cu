// The C ABI of the head norms (kernels: qk_norm.cuh).
#include <initializer_list>

#include "abi.h"
#include "qk_norm.cuh"

namespace sky {
namespace qkn {

extern template sky_status forward<__nv_bfloat16>(const sky_qk_norm_shape&, Params&, cudaStream_t);
extern template sky_status forward<float>(const sky_qk_norm_shape&, Params&, cudaStream_t);
extern template sky_status backward<__nv_bfloat16>(const sky_qk_norm_shape&, Params&, float*, float*, cudaStream_t);
extern template sky_status backward<float>(const sky_qk_norm_shape&, Params&, float*, float*, cudaStream_t);

sky_status check(const sky_qk_norm_shape* s) {
  SKY_CHECK(s, SKY_ERR_INVALID_ARG, "null shape");
  SKY_CHECK(s->rows > 0 && s->q_heads >= 0 && s->k_heads >= 0 && s->head_dim > 0 &&
                static_cast<int64_t>(s->q_heads) + s->k_heads > 0,
            SKY_ERR_INVALID_ARG, "bad sizes");
  SKY_CHECK(s->dtype == SKY_DTYPE_BF16 || s->dtype == SKY_DTYPE_FP32, SKY_ERR_INVALID_ARG, "unknown dtype");
  SKY_CHECK(s->rotation >= SKY_ROTATE_NONE && s->rotation <= SKY_ROTATE_PAIRS, SKY_ERR_INVALID_ARG,
            "unknown rotation");
  SKY_CHECK(s->eps >= 0.f && std::isfinite(s->eps), SKY_ERR_INVALID_ARG, "eps must be finite and not negative");
  SKY_CHECK(s->rotation == SKY_ROTATE_NONE || (s->theta > 0. && std::isfinite(s->theta)), SKY_ERR_INVALID_ARG,
            "theta must be finite and positive");
  const int64_t width = (static_cast<int64_t>(s->q_heads) + s->k_heads) * s->head_dim;
  SKY_CHECK(s->ldx >= width && s->ldy >= width, SKY_ERR_INVALID_ARG, "rows shorter than their heads");
  SKY_CHECK(s->head_dim % 16 == 0 && s->head_dim <= MAX_D, SKY_ERR_UNSUPPORTED,
            "head norms need a head dim that is a multiple of 16, up to %d (got %d)", MAX_D, s->head_dim);
  const int vec = s->dtype == SKY_DTYPE_BF16 ? 8 : 4;
  SKY_CHECK(s->ldx % vec == 0 && s->ldy % vec == 0, SKY_ERR_UNSUPPORTED,
            "head norms need rows that are multiples of 16 bytes apart");
  SKY_CHECK(width <= (1 << 24), SKY_ERR_UNSUPPORTED, "rows of more than 2^24 values");
  return SKY_OK;
}

Params params(const sky_qk_norm_shape& s, const void* q_gain, const void* k_gain, const int32_t* pos) {
  Params p = {};
  p.gain[0] = q_gain;
  p.gain[1] = k_gain;
  p.pos = pos;
  p.ldx = s.ldx;
  p.ldy = s.ldy;
  p.rows = s.rows;
  p.D = s.head_dim;
  p.heads[0] = s.q_heads;
  p.heads[1] = s.k_heads;
  p.eps = s.eps;
  if (s.rotation != SKY_ROTATE_NONE) {
    // theta^(-2 i / D) as the product of two powers, i = 16 a + b: half the calls of pow
    double fine[16], coarse = 1.0;
    for (int b = 0; b < 16; ++b) fine[b] = std::pow(s.theta, -2.0 * b / s.head_dim);
    for (int i = 0; i < s.head_dim / 2; ++i) {
      if (i > 0 && i % 16 == 0) coarse = std::pow(s.theta, -2.0 * i / s.head_dim);
      const double f = coarse * fine[i % 16] / 6.283185307179586476925;
      double whole;  // (whole turns a position change nothing; they arise for theta < 1)
      // (to nearest; below 1 a double is at most 1 - 2^-53, so 2^64 is never reached)
      p.turn[i] = static_cast<uint64_t>(std::nearbyint(std::modf(f, &whole) * 18446744073709551616.0));
    }
  }
  return p;
}

// Gains on their type's grid, positions and gain gradients on 4 bytes.
bool small_on_grid(const sky_qk_norm_shape& s, std::initializer_list<const void*> gains,
                   std::initializer_list<const void*> words) {
  for (const void* p : gains)
    if (reinterpret_cast<uintptr_t>(p) % (s.dtype == SKY_DTYPE_BF16 ? 2 : 4)) return false;
  for (const void* p : words)
    if (reinterpret_cast<uintptr_t>(p) & 3) return false;
  return true;
}

bool a16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

size_t workspace(const sky_qk_norm_shape& s) {  // 2 rows a CTA, of as many as any plan makes
  const int most = std::max(max_ctas(true), ceil_div(static_cast<int64_t>(s.q_heads) + s.k_heads + 2, WARPS));
  return static_cast<size_t>(2) * most * s.head_dim * sizeof(float);
}

}  // namespace qkn
}  // namespace sky

using namespace sky;

extern "C" {

sky_status sky_qk_norm_fwd(const sky_qk_norm_shape* shape, const void* x, const void* q_gain, const void* k_gain,
                           const int32_t* d_pos, void* y, void* stream) {
  ABI_GUARD_BEGIN
  const sky_status ok = qkn::check(shape);
  if (ok != SKY_OK) return ok;
  SKY_CHECK(x && y, SKY_ERR_INVALID_ARG, "null argument");
  SKY_CHECK(d_pos || shape->rotation == SKY_ROTATE_NONE, SKY_ERR_INVALID_ARG, "a rotation needs positions");
  SKY_CHECK(x != y || shape->ldx == shape->ldy, SKY_ERR_INVALID_ARG, "in place needs ldx == ldy");
  SKY_CHECK(qkn::small_on_grid(*shape, {q_gain, k_gain}, {d_pos}), SKY_ERR_INVALID_ARG,
            "gains or positions off their type's grid");
  SKY_CHECK(qkn::a16(x) && qkn::a16(y), SKY_ERR_UNSUPPORTED, "head norm tensors must be 16-byte aligned");
  qkn::Params p = qkn::params(*shape, q_gain, k_gain, d_pos);
  p.x = x;
  p.out = y;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return shape->dtype == SKY_DTYPE_BF16 ? qkn::forward<__nv_bfloat16>(*shape, p, st) : qkn::forward<float>(*shape, p, st);
  ABI_GUARD_END
}

size_t sky_qk_norm_bwd_workspace_bytes(const sky_qk_norm_shape* shape) {
  return shape && qkn::check(shape) == SKY_OK ? qkn::workspace(*shape) : 0;
}

sky_status sky_qk_norm_bwd(const sky_qk_norm_shape* shape, const void* x, const void* dy, const void* q_gain,
                           const void* k_gain, const int32_t* d_pos, void* dx, float* dq_gain, float* dk_gain,
                           void* workspace, size_t workspace_bytes, void* stream) {
  ABI_GUARD_BEGIN
  const sky_status ok = qkn::check(shape);
  if (ok != SKY_OK) return ok;
  SKY_CHECK(x && dy && dx && workspace, SKY_ERR_INVALID_ARG, "null argument");
  SKY_CHECK(d_pos || shape->rotation == SKY_ROTATE_NONE, SKY_ERR_INVALID_ARG, "a rotation needs positions");
  SKY_CHECK(dx != dy || shape->ldx == shape->ldy, SKY_ERR_INVALID_ARG, "in place needs ldx == ldy");
  SKY_CHECK(qkn::small_on_grid(*shape, {q_gain, k_gain}, {d_pos, dq_gain, dk_gain}), SKY_ERR_INVALID_ARG,
            "gains, positions or gain gradients off their type's grid");
  SKY_CHECK(qkn::a16(x) && qkn::a16(dy) && qkn::a16(dx), SKY_ERR_UNSUPPORTED,
            "head norm tensors must be 16-byte aligned");
  SKY_CHECK((reinterpret_cast<uintptr_t>(workspace) & 3) == 0, SKY_ERR_INVALID_ARG,
            "workspace must be 4-byte aligned");
  SKY_CHECK(workspace_bytes >= qkn::workspace(*shape), SKY_ERR_INVALID_ARG, "workspace too small");
  qkn::Params p = qkn::params(*shape, q_gain, k_gain, d_pos);
  p.x = x;
  p.dy = dy;
  p.out = dx;
  p.part = static_cast<float*>(workspace);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return shape->dtype == SKY_DTYPE_BF16 ? qkn::backward<__nv_bfloat16>(*shape, p, dq_gain, dk_gain, st)
                                        : qkn::backward<float>(*shape, p, dq_gain, dk_gain, st);
  ABI_GUARD_END
}

}  // extern "C"
