// Masked scaled dot-product attention, Eq. 1: per sequence b and head a,
//   P = softmax_j(Q K^T / sqrt(D)) over the valid keys j < len[b],
//   ctx = P V,
// and its backward (dQ, dK, dV).  All S query rows are computed; padded keys
// get probability exactly 0.
//
// bf16 (D = 64): the tensor-core kernels of attention_tc.cu, plus the
// vectorised delta = rowsum(dO * O) pre-pass here (sequences over 128; shorter
// ones form it in their one backward launch).
// fp32: the kernels of attention_simt.cu.
#include "attention_simt.h"
#include "common.cuh"

namespace sky {
namespace attn {

constexpr int HD = 64;

using bf16 = __nv_bfloat16;

// delta[b,a,s] = sum_d dctx[b,s,a,d] * ctx[b,s,a,d]  (equals sum_j P_sj dP_sj)
// One warp per token row; each lane takes 8 consecutive elements (16 bytes
// of bf16) per 256-column group, and the 8 lanes covering one 64-wide head
// reduce with shuffles.  NV > 0: the row has exactly NV groups, and every
// load of the row is issued before the first product (more bytes in flight
// per warp); NV == 0: any H that is a multiple of 64, one group at a time.
// Requires D == 64.
// Beside delta it writes the per-query terms the tensor-core dK/dV kernel
// adds inside its score products: xtab[(b*A + a)*2 + 0][s] = lse2 / c and
// xtab[(b*A + a)*2 + 1][s] = delta (c = log2(e)/sqrt(D)), each negated and
// split into a bf16 high and low part, as 16-byte rows [hi, lo, 0 x 6].
template <int NV>
__global__ void attn_delta_bf16(const bf16* __restrict__ ctx, const bf16* __restrict__ dctx, int S,
                                int H, int A, int64_t rows, float* __restrict__ delta,
                                const float* __restrict__ lse, uint4* __restrict__ xtab) {
  pdl_wait();
  pdl_trigger();
  const int64_t row = (blockIdx.x * (int64_t)blockDim.x + threadIdx.x) >> 5;
  const int l = threadIdx.x & 31;
  if (row >= rows) return;
  const int64_t b = row / S, s = row % S;
  auto dot8 = [](const uint4& x, const uint4& y) {
    const __nv_bfloat162* xs = reinterpret_cast<const __nv_bfloat162*>(&x);
    const __nv_bfloat162* ys = reinterpret_cast<const __nv_bfloat162*>(&y);
    float acc = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 p = __bfloat1622float2(xs[i]), q = __bfloat1622float2(ys[i]);
      acc += p.x * q.x + p.y * q.y;
    }
    return acc;
  };
  // lz: the row's lse of this lane's head, loaded beside ctx / dctx (NV > 0)
  auto finish = [&](float acc, int col, float lz) {
    acc += __shfl_xor_sync(0xffffffffu, acc, 1);
    acc += __shfl_xor_sync(0xffffffffu, acc, 2);
    acc += __shfl_xor_sync(0xffffffffu, acc, 4);
    if ((l & 7) == 0 && col < H) {
      const int64_t bh = b * A + col / HD;
      delta[bh * S + s] = acc;
      auto row16 = [](float x) {  // -x as [hi, lo, 0, ...] in bf16
        const bf16 hi = __float2bfloat16_rn(-x);
        const bf16 lo = __float2bfloat16_rn(-x - __bfloat162float(hi));
        return make_uint4(static_cast<uint32_t>(__bfloat16_as_ushort(hi)) |
                              (static_cast<uint32_t>(__bfloat16_as_ushort(lo)) << 16),
                          0u, 0u, 0u);
      };
      constexpr float kC = 1.4426950408889634f * 0.125f;  // log2(e) / sqrt(64)
      xtab[(bh * 2) * S + s] = row16(__fdiv_rn(lz, kC));
      xtab[(bh * 2 + 1) * S + s] = row16(acc);
    }
  };
  if constexpr (NV > 0) {
    uint4 x[NV], y[NV];
    float lz[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      x[v] = *reinterpret_cast<const uint4*>(ctx + row * H + v * 256 + l * 8);
      y[v] = *reinterpret_cast<const uint4*>(dctx + row * H + v * 256 + l * 8);
      lz[v] = (l & 7) == 0 ? lse[(b * A + (v * 256 + l * 8) / HD) * S + s] : 0.f;
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) finish(dot8(x[v], y[v]), v * 256 + l * 8, lz[v]);
  } else {
    for (int c0 = 0; c0 < H; c0 += 256) {
      const int col = c0 + l * 8;
      float acc = 0.f, lz = 0.f;
      if (col < H) {
        acc = dot8(*reinterpret_cast<const uint4*>(ctx + row * H + col),
                   *reinterpret_cast<const uint4*>(dctx + row * H + col));
        if ((l & 7) == 0) lz = lse[(b * A + col / HD) * S + s];
      }
      finish(acc, col, lz);
    }
  }
}

}  // namespace attn

// ------------------------------------------------------------------- host
sky_status attention_fwd_tc(const void* qkv, const int32_t* lens, int B, int S, int H, int A,
                            void* ctx, float* lse, int32_t* status, uint64_t timeout_ns,
                            cudaStream_t stream);

sky_status attention_bwd_short_tc(const void* qkv, const void* ctx, const void* dctx, const float* lse,
                                  const int32_t* lens, int B, int S, int H, int A, void* dqkv, int32_t* status,
                                  uint64_t timeout_ns, cudaStream_t stream, float* colpart);

sky_status attention_bwd_tc(const void* qkv, const void* dctx, const float* lse, const float* delta,
                            const uint4* xtab, const int32_t* lens, int B, int S, int H, int A, void* dqkv,
                            int32_t* status, uint64_t timeout_ns, cudaStream_t stream,
                            float* colpart);

sky_status attention_fwd(const void* qkv, const int32_t* lens, int B, int S, int H, int A,
                         sky_dtype dt, void* ctx, float* lse, int32_t* status,
                         cudaStream_t stream) {
  const int D = H / A;
  if (dt == SKY_DTYPE_BF16) {
    SKY_CHECK(D == attn::HD, SKY_ERR_UNSUPPORTED, "bf16 attention needs head dim 64 (got %d)", D);
    return attention_fwd_tc(qkv, lens, B, S, H, A, ctx, lse, status, 2000000000ull, stream);
  }
  SKY_CHECK(D <= 128, SKY_ERR_UNSUPPORTED, "fp32 attention needs head dim <= 128");
  SKY_CHECK(S <= 3072, SKY_ERR_UNSUPPORTED, "fp32 attention: sequence too long");
  const cudaError_t e = attn::launch_fwd_self(static_cast<const float*>(qkv), lens, B, S, H, A, static_cast<float*>(ctx),
                                              lse, status, stream);
  return e == cudaSuccess ? SKY_OK : cuda_fail(e, "attention forward launch");
}

// delta [B][A][S] floats, then (bf16 path) the dK/dV kernel's per-query rows
// [B][A][2][S] x 16 bytes, 16-byte aligned.
static size_t delta_bytes(int B, int S, int A) { return ((size_t)B * A * S * sizeof(float) + 15) & ~(size_t)15; }
size_t attention_bwd_ws(int B, int S, int A) { return delta_bytes(B, S, A) + (size_t)B * A * 2 * S * 16; }

sky_status attention_bwd(const void* qkv, const void* ctx, const void* dctx, const float* lse,
                         const int32_t* lens, int B, int S, int H, int A, sky_dtype dt, void* dqkv,
                         float* delta, int32_t* status, cudaStream_t stream, float* colpart) {
  const int D = H / A;
  const int64_t rows = (int64_t)B * S;
  if (dt == SKY_DTYPE_BF16) {
    SKY_CHECK(D == attn::HD, SKY_ERR_UNSUPPORTED, "bf16 attention needs head dim 64 (got %d)", D);
    // every kernel below moves 16-byte vectors of these buffers (checked
    // before the first launch)
    const auto a16 = [](const void* q) { return (reinterpret_cast<uintptr_t>(q) & 15) == 0; };
    SKY_CHECK(a16(qkv) && a16(ctx) && a16(dctx) && a16(dqkv) && a16(delta), SKY_ERR_INVALID_ARG,
              "bf16 attention backward buffers and workspace must be 16-byte aligned");
    // one tile a sequence: everything in one launch (grid y is the batch, at most
    // 65535 as for the kernels below)
    if (S <= 128 && B <= 65535)
      return attention_bwd_short_tc(qkv, ctx, dctx, lse, lens, B, S, H, A, dqkv, status, 2000000000ull, stream,
                                    colpart);
    const auto* c = static_cast<const __nv_bfloat16*>(ctx);
    const auto* dc = static_cast<const __nv_bfloat16*>(dctx);
    const dim3 g(ceil_div(rows * 32, 256)), blk(256);
    uint4* xtab = reinterpret_cast<uint4*>(reinterpret_cast<char*>(delta) + delta_bytes(B, S, A));
    cudaError_t le;
    switch (H % 256 == 0 ? H / 256 : 0) {
      case 3: le = launch_pdl(attn::attn_delta_bf16<3>, g, blk, 0, stream, 1, c, dc, S, H, A, rows, delta, lse, xtab); break;
      case 4: le = launch_pdl(attn::attn_delta_bf16<4>, g, blk, 0, stream, 1, c, dc, S, H, A, rows, delta, lse, xtab); break;
      case 8: le = launch_pdl(attn::attn_delta_bf16<8>, g, blk, 0, stream, 1, c, dc, S, H, A, rows, delta, lse, xtab); break;
      default: le = launch_pdl(attn::attn_delta_bf16<0>, g, blk, 0, stream, 1, c, dc, S, H, A, rows, delta, lse, xtab); break;
    }
    count_launches(1);
    if (le != cudaSuccess) return cuda_fail(le, "attention delta launch");
    return attention_bwd_tc(qkv, dctx, lse, delta, xtab, lens, B, S, H, A, dqkv, status, 2000000000ull,
                            stream, colpart);
  }
  SKY_CHECK(D <= 128, SKY_ERR_UNSUPPORTED, "fp32 attention needs head dim <= 128");
  const cudaError_t e =
      attn::launch_bwd_self(static_cast<const float*>(qkv), static_cast<const float*>(ctx), static_cast<const float*>(dctx),
                            lse, lens, B, S, H, A, delta, static_cast<float*>(dqkv), stream);
  return e == cudaSuccess ? SKY_OK : cuda_fail(e, "attention backward launch");
}

}  // namespace sky
