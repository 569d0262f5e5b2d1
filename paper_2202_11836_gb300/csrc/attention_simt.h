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
  int least;              // of a length: 1, or 0 where a sequence may have no keys
  int32_t* status;
};

// The valid keys of sequence b; a bad length is clamped and reported.
__device__ __forceinline__ int valid_keys(const Geometry& g, int b) {
  int len = g.lens[b];
  if (len < g.least || len > g.Skv) {
    if (g.status && threadIdx.x == 0) atomicOr(g.status, kStatusBadLength);
    len = len < g.least ? g.least : g.Skv;
  }
  return len;
}

// T: float or __nv_bfloat16.  lse may be null.
template <typename T>
cudaError_t launch_fwd_simt(Geometry g, int B, T* ctx, float* lse, cudaStream_t stream);
// delta: [B][A][Sq] floats of scratch.
template <typename T>
cudaError_t launch_bwd_simt(Geometry g, int B, const T* ctx, const T* dctx, const float* lse, float* delta, T* dq, T* dk,
                            T* dv, cudaStream_t stream);

}  // namespace attn
}  // namespace sky
