// Attention of a decoder's queries over an encoder's states: the C ABI of
// sky_cross_attention_* and its choice of kernels.  Per sequence b and query head a,
// with the key head a / (heads / kv_heads):
//   P = softmax_j(Q K^T / sqrt(D)) over the valid keys j < len[b],  ctx = P V,
// and with dP = dctx V^T, delta = rowsum(P dP) = rowsum(dctx ctx), dS = P (dP - delta)
//   dQ = dS K / sqrt(D),  dK = sum of dS^T Q / sqrt(D),  dV = sum of P^T dctx
// over the query heads of a key head.
#include <algorithm>
#include <initializer_list>
#include <type_traits>

#include "abi.h"
#include "attention_few.h"
#include "attention_simt.h"
#include "attention_tc.h"
#include "common.cuh"

namespace sky {
namespace cross {

sky_status check(const sky_cross_shape* s) {
  SKY_CHECK(s, SKY_ERR_INVALID_ARG, "null shape");
  SKY_CHECK(s->batch > 0 && s->q_len > 0 && s->kv_len > 0 && s->heads > 0 && s->kv_heads > 0 && s->head_dim > 0 &&
                s->heads % s->kv_heads == 0,
            SKY_ERR_INVALID_ARG, "bad sizes");
  SKY_CHECK(s->dtype == SKY_DTYPE_BF16 || s->dtype == SKY_DTYPE_FP32, SKY_ERR_INVALID_ARG, "unknown dtype");
  SKY_CHECK(s->head_dim <= 128, SKY_ERR_UNSUPPORTED, "cross attention needs a head dim up to 128 (got %d)", s->head_dim);
  const int64_t qw = static_cast<int64_t>(s->heads) * s->head_dim, kw = static_cast<int64_t>(s->kv_heads) * s->head_dim;
  SKY_CHECK(s->ldq >= qw && s->ldo >= qw && s->ldk >= kw && s->ldv >= kw, SKY_ERR_INVALID_ARG,
            "rows shorter than their heads");
  // grid dimensions and the kernels' row and column numbers, which are 32 bits
  SKY_CHECK(s->batch <= 65535 && s->q_len <= (1 << 24) && s->kv_len <= (1 << 24) && s->heads <= (1 << 10) &&
                std::max(std::max(s->ldq, s->ldo), std::max(s->ldk, s->ldv)) <= (int64_t{1} << 30),
            SKY_ERR_UNSUPPORTED, "cross attention of more than 65535 sequences, 2^24 rows, 1024 heads or 2^30 values a row");
  SKY_CHECK(static_cast<int64_t>(s->batch) * s->q_len * s->heads < (int64_t{1} << 33), SKY_ERR_UNSUPPORTED,
            "cross attention of 2^33 query rows and heads or more");
  return SKY_OK;
}

// Tensors start on their type's grid (the tensor-core kernels ask for more, and the
// others serve what does not meet it).
bool on_grid(const sky_cross_shape& s, const void* p) {
  return reinterpret_cast<uintptr_t>(p) % (s.dtype == SKY_DTYPE_BF16 ? 2 : 4) == 0;
}
bool words(std::initializer_list<const void*> ps) {  // lengths, log-sum-exps, status: 4 bytes
  for (const void* p : ps)
    if (reinterpret_cast<uintptr_t>(p) & 3) return false;
  return true;
}

attn::Geometry geometry(const sky_cross_shape& s, const void* q, const void* k, const void* v, const int32_t* len,
                        int32_t* status) {
  return {q,        k,       v,       s.ldq, s.ldk, s.ldv, s.ldo, s.q_len, s.kv_len, s.heads, s.heads / s.kv_heads,
          s.head_dim, 0, false, len, status};
}

// delta, 4 bytes a row and head, and where the shape allows the tensor-core kernels (the
// pointers, which may rule them out still, are not known) their table rows, 32 more.
size_t workspace(const sky_cross_shape& s) {
  const attn::Geometry g = geometry(s, nullptr, nullptr, nullptr, nullptr, nullptr);
  if (s.dtype == SKY_DTYPE_BF16 && cross_attention_tc_fits(g, {})) return cross_attention_bwd_tc_ws(g, s.batch);
  return (static_cast<size_t>(s.batch) * s.heads * s.q_len * sizeof(float) + 15) & ~size_t{15};
}

template <typename T>
sky_status forward(const sky_cross_shape& s, const attn::Geometry& g, void* ctx, float* lse, cudaStream_t st) {
  if (std::is_same<T, __nv_bfloat16>::value && cross_attention_tc_fits(g, {g.q, g.k, g.v, ctx}))
    return cross_attention_few_fits(g) ? cross_attention_few(g, s.batch, ctx, lse, st)
                                       : cross_attention_fwd_tc(g, s.batch, ctx, lse, st);
  if (cross_attention_few_simt_pays(g, s.batch)) return cross_attention_few_simt(g, s.batch, static_cast<T*>(ctx), lse, st);
  const cudaError_t e = attn::launch_fwd_simt(g, s.batch, static_cast<T*>(ctx), lse, st);
  return e == cudaSuccess ? SKY_OK : cuda_fail(e, "cross attention forward launch");
}

template <typename T>
sky_status backward(const sky_cross_shape& s, const attn::Geometry& g, const void* ctx, const void* dctx,
                    const float* lse, void* dq, void* dk, void* dv, void* ws, cudaStream_t st) {
  if (std::is_same<T, __nv_bfloat16>::value && cross_attention_tc_fits(g, {g.q, g.k, g.v, dctx, dq, dk, dv}))
    return cross_attention_bwd_tc(g, s.batch, dctx, lse, dq, dk, dv, ws, st);
  const cudaError_t e =
      attn::launch_bwd_simt(g, s.batch, static_cast<const T*>(ctx), static_cast<const T*>(dctx), lse,
                            static_cast<float*>(ws), static_cast<T*>(dq), static_cast<T*>(dk), static_cast<T*>(dv), st);
  return e == cudaSuccess ? SKY_OK : cuda_fail(e, "cross attention backward launch");
}

}  // namespace cross
}  // namespace sky

using namespace sky;

extern "C" {

sky_status sky_cross_attention_fwd(const sky_cross_shape* shape, const void* q, const void* k, const void* v,
                                   const int32_t* d_len, void* ctx, float* lse, int32_t* d_status, void* stream) {
  ABI_GUARD_BEGIN
  const sky_status ok = cross::check(shape);
  if (ok != SKY_OK) return ok;
  SKY_CHECK(q && k && v && d_len && ctx, SKY_ERR_INVALID_ARG, "null argument");
  for (const void* p : {q, k, v, static_cast<const void*>(ctx)})
    SKY_CHECK(cross::on_grid(*shape, p), SKY_ERR_INVALID_ARG, "a tensor off its type's grid");
  SKY_CHECK(cross::words({d_len, lse, d_status}), SKY_ERR_INVALID_ARG, "lengths, lse or status off the 4-byte grid");
  const attn::Geometry g = cross::geometry(*shape, q, k, v, d_len, d_status);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return shape->dtype == SKY_DTYPE_BF16 ? cross::forward<__nv_bfloat16>(*shape, g, ctx, lse, st)
                                        : cross::forward<float>(*shape, g, ctx, lse, st);
  ABI_GUARD_END
}

size_t sky_cross_attention_bwd_workspace_bytes(const sky_cross_shape* shape) {
  return shape && cross::check(shape) == SKY_OK ? cross::workspace(*shape) : 0;
}

sky_status sky_cross_attention_bwd(const sky_cross_shape* shape, const void* q, const void* k, const void* v,
                                   const void* ctx, const void* dctx, const float* lse, const int32_t* d_len, void* dq,
                                   void* dk, void* dv, void* workspace, size_t workspace_bytes, int32_t* d_status,
                                   void* stream) {
  ABI_GUARD_BEGIN
  const sky_status ok = cross::check(shape);
  if (ok != SKY_OK) return ok;
  SKY_CHECK(q && k && v && ctx && dctx && lse && d_len && dq && dk && dv && workspace, SKY_ERR_INVALID_ARG,
            "null argument");
  for (const void* p : {q, k, v, ctx, dctx, static_cast<const void*>(dq), static_cast<const void*>(dk),
                        static_cast<const void*>(dv)})
    SKY_CHECK(cross::on_grid(*shape, p), SKY_ERR_INVALID_ARG, "a tensor off its type's grid");
  SKY_CHECK(cross::words({d_len, lse, d_status}), SKY_ERR_INVALID_ARG, "lengths, lse or status off the 4-byte grid");
  SKY_CHECK((reinterpret_cast<uintptr_t>(workspace) & 15) == 0, SKY_ERR_INVALID_ARG,
            "workspace must be 16-byte aligned");
  SKY_CHECK(workspace_bytes >= cross::workspace(*shape), SKY_ERR_INVALID_ARG, "workspace too small");
  const attn::Geometry g = cross::geometry(*shape, q, k, v, d_len, d_status);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return shape->dtype == SKY_DTYPE_BF16
             ? cross::backward<__nv_bfloat16>(*shape, g, ctx, dctx, lse, dq, dk, dv, workspace, st)
             : cross::backward<float>(*shape, g, ctx, dctx, lse, dq, dk, dv, workspace, st);
  ABI_GUARD_END
}

}  // extern "C"
