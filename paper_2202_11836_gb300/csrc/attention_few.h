// Cross attention of few query rows (attention_few.cu): bf16 with head dim 64, where
// cross_attention_tc_fits; and any type (T: float or __nv_bfloat16), head dim and alignment.
#pragma once
#include "../../include/sky_ops.h"
#include "attention_simt.h"

namespace sky {

bool cross_attention_few_fits(const attn::Geometry& g);
sky_status cross_attention_few(const attn::Geometry& g, int B, void* ctx, float* lse, cudaStream_t stream);

bool cross_attention_few_simt_pays(const attn::Geometry& g, int B);
template <typename T>
sky_status cross_attention_few_simt(const attn::Geometry& g, int B, T* ctx, float* lse, cudaStream_t stream);

}  // namespace sky
