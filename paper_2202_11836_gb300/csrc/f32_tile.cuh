// A 64 x 64 tile of a product in fp32 arithmetic on the CUDA cores, shared by the fp32 GEMM
// (gemm_f32.cu, which says why it looks like this and what it measured) and the products
// grouped by expert (grouped_f32.cu).
#pragma once
#include "common.cuh"
#include "ptx.cuh"

namespace sky {
namespace gemm {

constexpr int TM = 64, TN = 64, TK = 32;
constexpr int RM = 8, RN = 4;                        // a thread's rows and columns
constexpr int F_THREADS = TM * TN / (RM * RN);
constexpr int LD4 = TK * 64 / 4 / F_THREADS;         // 16-byte groups a thread loads per slab

// One operand pair of a tile: element (i, k) of A at i * lda + k where it is K-major, else
// at k * lda + i, likewise B; rows m < M, columns n < N, and K of the sum.
struct F32Operands {
  const float *A, *B;
  int64_t lda, ldb;
  int M, N, K;
};

// Slab layout: element (k, i) of a TK x 64 slab at k * 64 + (i ^ swz(k)), which
// keeps 4-float groups together and spreads both kinds of store over the banks.
__device__ __forceinline__ constexpr int swz(int k) { return ((k >> 2) & 7) << 2; }

// One operand's slab: 64 rows (M or N index) from i0, k from k0.  KMAJ: element
// (i, k) at i * ld + k, else at k * ld + i.  VEC: 16-byte loads (ld % 4 == 0 and
// an aligned base, so a group of four is inside or outside as a whole).
template <bool KMAJ, bool VEC>
__device__ __forceinline__ void load_slab(const float* __restrict__ X, int64_t ld, int i0, int I, int k0,
                                          int K, float (&r)[4 * LD4]) {
  const int t = threadIdx.x;
#pragma unroll
  for (int j = 0; j < LD4; ++j) {
    const int i = i0 + (KMAJ ? t / (TK / 4) + F_THREADS / (TK / 4) * j : (t & 15) * 4);
    const int k = k0 + (KMAJ ? t % (TK / 4) * 4 : (t >> 4) + F_THREADS / 16 * j);
    const float* p = X + (KMAJ ? static_cast<int64_t>(i) * ld + k : static_cast<int64_t>(k) * ld + i);
    if constexpr (VEC) {
      const float4 v = i < I && k < K ? __ldg(reinterpret_cast<const float4*>(p)) : make_float4(0.f, 0.f, 0.f, 0.f);
      r[4 * j] = v.x; r[4 * j + 1] = v.y; r[4 * j + 2] = v.z; r[4 * j + 3] = v.w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        r[4 * j + e] = (KMAJ ? i < I && k + e < K : i + e < I && k < K) ? __ldg(p + e) : 0.f;
    }
  }
}
template <bool KMAJ>
__device__ __forceinline__ void store_slab(float* s, const float (&r)[4 * LD4]) {
  const int t = threadIdx.x;
#pragma unroll
  for (int j = 0; j < LD4; ++j) {
    if constexpr (KMAJ) {
      const int i = t / (TK / 4) + F_THREADS / (TK / 4) * j, k = t % (TK / 4) * 4;
#pragma unroll
      for (int e = 0; e < 4; ++e) s[(k + e) * 64 + (i ^ swz(k))] = r[4 * j + e];
    } else {
      const int i = (t & 15) * 4, k = (t >> 4) + F_THREADS / 16 * j;
      *reinterpret_cast<float4*>(s + k * 64 + (i ^ swz(k))) =
          make_float4(r[4 * j], r[4 * j + 1], r[4 * j + 2], r[4 * j + 3]);
    }
  }
}

// The tile at (m0, n0) over the slabs [s0, s1) of the sum, one of `ks` splits over a cluster:
// finish(m, n, value) is called once for every element of the tile, those outside the
// matrix included.  Each CTA of a split first says that it runs (cluster_arrive).
template <bool AK, bool BK, bool VEC, typename F>
__device__ __forceinline__ void f32_tile(const F32Operands& o, int m0, int n0, int ks, int split, int s0, int s1,
                                         const F& finish) {
  __shared__ __align__(16) float sm[2][2][TK * 64];  // [buffer][A, B]; later, unsplit, the 64 x 64 tile
  __shared__ __align__(16) float recv[TM * TN];      // split: this CTA's rows from every split
  const int t = threadIdx.x;
  // thread (rg, cg): rows {rg * 4 .., 32 + rg * 4 ..}, columns cg * 4 ..
  constexpr int CG = TN / RN;
  const int rg = t / CG, cg = t % CG;
  uint64_t acc[RM][RN / 2] = {};  // pairs of adjacent columns
  float ra[4 * LD4], rb[4 * LD4];
  load_slab<AK, VEC>(o.A, o.lda, m0, o.M, s0 * TK, o.K, ra);
  load_slab<BK, VEC>(o.B, o.ldb, n0, o.N, s0 * TK, o.K, rb);
  for (int s = s0; s < s1; ++s) {
    float* sa = sm[(s - s0) & 1][0];
    float* sb = sm[(s - s0) & 1][1];
    store_slab<AK>(sa, ra);
    store_slab<BK>(sb, rb);
    __syncthreads();
    if (s + 1 < s1) {
      load_slab<AK, VEC>(o.A, o.lda, m0, o.M, (s + 1) * TK, o.K, ra);
      load_slab<BK, VEC>(o.B, o.ldb, n0, o.N, (s + 1) * TK, o.K, rb);
    }
#pragma unroll
    for (int k = 0; k < TK; ++k) {
      float a[RM];
      uint64_t b[RN / 2];
      *reinterpret_cast<float4*>(a) = *reinterpret_cast<const float4*>(sa + k * 64 + ((rg * 4) ^ swz(k)));
      *reinterpret_cast<float4*>(a + 4) = *reinterpret_cast<const float4*>(sa + k * 64 + ((32 + rg * 4) ^ swz(k)));
      *reinterpret_cast<ulonglong2*>(b) = *reinterpret_cast<const ulonglong2*>(sb + k * 64 + ((cg * 4) ^ swz(k)));
#pragma unroll
      for (int i = 0; i < RM; ++i) {
        const uint64_t aa = pack2(a[i], a[i]);
#pragma unroll
        for (int j = 0; j < RN / 2; ++j) acc[i][j] = fma2(aa, b[j], acc[i][j]);
      }
    }
  }
  pdl_trigger();
  if (ks == 1) {
    // through shared memory (row r at r * 64), so that a warp stores 32 consecutive
    // columns of a row
    float* st = &sm[0][0][0];
    const int c = t & 63;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < RM; ++i) {
      const int r = (i < 4 ? 0 : 32) + rg * 4 + (i & 3);
      *reinterpret_cast<ulonglong2*>(st + r * 64 + cg * 4) = make_ulonglong2(acc[i][0], acc[i][1]);
    }
    __syncthreads();
#pragma unroll 4
    for (int r = t / 64; r < TM; r += F_THREADS / 64) finish(m0 + r, n0 + c, st[r * 64 + c]);
    return;
  }
  // Each CTA owns 64 / ks rows of the tile: every split sends it its partial rows,
  // half a warp a row, and it adds them in split order.
  const int own = TM / ks;
  ptx::cluster_wait();  // every peer runs
  const uint32_t base = ptx::smem_u32(recv);
#pragma unroll
  for (int i = 0; i < RM; ++i) {
    const int r = (i < 4 ? 0 : 32) + rg * 4 + (i & 3);
    const float2 lo = unpack2(acc[i][0]), hi = unpack2(acc[i][1]);
    ptx::st_cluster_v4(ptx::mapa_shared(base, r / own) + ((split * own + r % own) * 64 + cg * 4) * 4,
                       __float_as_uint(lo.x), __float_as_uint(lo.y), __float_as_uint(hi.x), __float_as_uint(hi.y));
  }
  ptx::cluster_sync();
  for (int g = t; g < own * 16; g += F_THREADS) {
    const int r = g >> 4, c = (g & 15) * 4;
    float4 part[8];
#pragma unroll
    for (int s = 0; s < 8; ++s)
      part[s] = s < ks ? *reinterpret_cast<const float4*>(recv + (s * own + r) * 64 + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    float4 v = part[0];
#pragma unroll
    for (int s = 1; s < 8; ++s)
      if (s < ks) { v.x += part[s].x; v.y += part[s].y; v.z += part[s].z; v.w += part[s].w; }
    const int m = m0 + split * own + r;
    finish(m, n0 + c, v.x);
    finish(m, n0 + c + 1, v.y);
    finish(m, n0 + c + 2, v.z);
    finish(m, n0 + c + 3, v.w);
  }
}

}  // namespace gemm
}  // namespace sky
