// Attention on the CUDA cores (attention_simt.cu): any head dim up to 128 and any
// strides, fp32 arithmetic on fp32 or bf16 storage, queries of one length over keys of
// another.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"

namespace sky {
namespace attn {

// Where a call's tensors are.  Rows of q, dq (ldq), k, dk (ldk), v, dv (ldv) and ctx,
// dctx (ldo) hold their heads side by side; head a reads key head a / group.
struct Geometry {
  const void *q, *k, *v;
  int64_t ldq, ldk, ldv, ldo;
  int Sq, Skv, A, group, D;
  int LD;                 // row stride in shared memory, and whether heads allow
  bool vec;               // 4-value accesses: the launchers' own
  const int32_t* lens;
  int32_t* status;
};

// The valid keys of sequence b, in [least, most]; a bad length is clamped and reported.
__device__ __forceinline__ int valid_keys(const int32_t* lens, int b, int least, int most, int32_t* status) {
  int len = lens[b];
  if (len < least || len > most) {
    if (status && threadIdx.x == 0) atomicOr(status, kStatusBadLength);
    len = len < least ? least : most;
  }
  return len;
}

// T: float or __nv_bfloat16.  lse may be null.
template <typename T>
cudaError_t launch_fwd_simt(const Geometry& g, int B, T* ctx, float* lse, cudaStream_t stream);
// delta: [B][A][Sq] floats of scratch.  ctx: read for fp32 only.
template <typename T>
cudaError_t launch_bwd_simt(const Geometry& g, int B, const T* ctx, const T* dctx, const float* lse, float* delta, T* dq,
                            T* dk, T* dv, cudaStream_t stream);
// Self attention over packed QKV rows.
cudaError_t launch_fwd_self(const float* qkv, const int32_t* lens, int B, int S, int H, int A, float* ctx, float* lse,
                            int32_t* status, cudaStream_t stream);
cudaError_t launch_bwd_self(const float* qkv, const float* ctx, const float* dctx, const float* lse, const int32_t* lens,
                            int B, int S, int H, int A, float* delta, float* dqkv, cudaStream_t stream);

}  // namespace attn
}  // namespace sky
