// Cross attention on the tensor cores (attention_tc.cu): bf16, head dim 64, every tensor
// and row distance on the 16-byte grid.
#pragma once
#include <cuda.h>

#include <initializer_list>

#include "../../include/sky_ops.h"
#include "attention_simt.h"

namespace sky {

namespace attn_tc {
// Heads of 64 of [B][rows] rows `ld` values apart: box {64 values, `take_heads` heads,
// `take` rows of one sequence}, 128B swizzle; what lies outside is read as zeros and not
// written.
bool cross_map(CUtensorMap* map, const void* base, int heads, int rows, int B, int64_t ld, int take_heads, int take);
}  // namespace attn_tc

bool cross_attention_tc_fits(const attn::Geometry& g, std::initializer_list<const void*> tensors);
sky_status cross_attention_fwd_tc(const attn::Geometry& g, int B, void* ctx, float* lse, cudaStream_t stream);
// Scratch of the backward (16-byte aligned): delta, then the dK/dV kernel's per-query rows.
size_t cross_attention_bwd_tc_ws(const attn::Geometry& g, int B);
sky_status cross_attention_bwd_tc(const attn::Geometry& g, int B, const void* dctx, const float* lse, void* dq, void* dk,
                                  void* dv, void* ws, cudaStream_t stream);

}  // namespace sky
