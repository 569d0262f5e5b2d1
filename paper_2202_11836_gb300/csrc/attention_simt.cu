// Masked scaled dot-product attention on the CUDA cores, for every head dim up to 128
// and any strides: fp32 arithmetic on fp32 or bf16 storage, queries of one length over
// keys of another.  The fp32 path of self attention, and cross attention wherever the
// tensor-core kernels do not apply.
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "attention_simt.h"
#include "common.cuh"
#include "ptx.cuh"
#include "row4.cuh"

namespace sky {
namespace attn {

// delta[b, a, s] = sum_d dctx * ctx: one warp per (row, head), rows of ldo.  (fp32; bf16:
// attn_delta_keys)
template <typename T>
__global__ void attn_delta(const T* __restrict__ ctx, const T* __restrict__ dctx, int S, int64_t ldo,
                           int A, int D, int64_t rows, float* __restrict__ delta) {
  pdl_wait();
  pdl_trigger();
  const int64_t w = (blockIdx.x * (int64_t)blockDim.x + threadIdx.x) >> 5;
  const int l = threadIdx.x & 31;
  if (w >= rows * A) return;
  const int64_t row = w / A;
  const int a = (int)(w % A);
  const T* c = ctx + row * ldo + a * D;
  const T* dc = dctx + row * ldo + a * D;
  float acc = 0.f;
  for (int d = l; d < D; d += 32) acc += to_f32(c[d]) * to_f32(dc[d]);
  acc = warp_sum(acc);
  if (l == 0) {
    const int64_t b = row / S, s = row % S;
    delta[(b * A + a) * S + s] = acc;
  }
}

// A CTA of four warps owns 16 rows
// of one (sequence, head) and walks the other side in tiles of 64 rows staged in
// shared memory.  Half a warp owns two rows, so row maxima and sums are
// shuffles among 16 lanes and a row's probabilities go to shared memory and
// back within the half warp.  Score products: 2 rows x 4 columns a thread (six
// 16-byte shared loads for 32 FMAs); accumulating products: 2 rows x 4 dims.
// Short sequences and few heads make these latency-bound; a warp per row with
// scalar loads took 116 us forward and 182 us backward at 4 x 101 tokens, 12
// heads of 64.
constexpr int FR = 16, FC = 64, F_THR = 128;  // rows of a CTA, columns of a tile
constexpr int FP_LD = FC + 4;                 // row stride of the probability tiles
// (the backward of sequences up to 16 tokens: tiles of 16 columns, NC = 1 of 4)

// Rows are staged F_THR / G a pass, G threads a row (D <= 4 G), through registers, so
// that a tile's loads are all in flight before the first is stored.  Loading and
// storing in turn waited for each: 4 x 32 tokens, 2 heads of 64, forward 6.4 us,
// now 3.8, backward 10.7 and 7.3; 4 x 101, 12 heads 17.0 and 12.2, 39.9 and 29.4; 4 x
// 256, 24 heads of 32 52.6 and 48.7 (58.1 with 16 threads a row).
template <int G, int NC = FC / 16>
struct Stage {  // a tile's 16 NC rows: BATCHES of PASSES passes, R rows each
  static constexpr int ROWS = 16 * NC;
  static constexpr int PASSES = ROWS * G / F_THR < 8 ? ROWS * G / F_THR : 8;
  static constexpr int R = PASSES * F_THR / G, BATCHES = ROWS / R;
  static constexpr int OWN = FR * G / F_THR;  // passes of the CTA's FR rows
  static constexpr int CC = G > 16 ? G / 16 : 1;  // 64-value column groups of an output row
};
// Rows from `rows` on are zeros.  vec: D, ld and X allow load4.
template <int G, typename T, int N>
__device__ __forceinline__ void load_rows(const T* __restrict__ X, int64_t ld, int r0, int rows, int D, bool vec,
                                          float4 (&v)[N]) {
  const int c = (threadIdx.x % G) * 4;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int r = r0 + F_THR / G * i + threadIdx.x / G;
    v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r < rows && c < D) {
      const T* p = X + static_cast<int64_t>(r) * ld + c;
      if (vec) {
        v[i] = load4(p);
      } else {
        v[i].x = to_f32(p[0]);
        if (c + 1 < D) v[i].y = to_f32(p[1]);
        if (c + 2 < D) v[i].z = to_f32(p[2]);
        if (c + 3 < D) v[i].w = to_f32(p[3]);
      }
    }
  }
}
template <int G, int N>
__device__ __forceinline__ void put_rows(float* s, int LD, int D, const float4 (&v)[N]) {
  const int c = (threadIdx.x % G) * 4;
  if (c >= D) return;
#pragma unroll
  for (int i = 0; i < N; ++i)
    *reinterpret_cast<float4*>(s + (F_THR / G * i + threadIdx.x / G) * LD + c) = v[i];
}
// acc[i][c] = row (2 ty + i) . column row (tx + 16 c), over D (a multiple of 4 in shared memory)
template <int NC>
__device__ __forceinline__ void scores(const float* rows, const float* cols, int LD, int D, float (&acc)[2][NC]) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[i][c] = 0.f;
  for (int d = 0; d < D; d += 4) {
    float4 r[2], k[NC];
#pragma unroll
    for (int i = 0; i < 2; ++i) r[i] = *reinterpret_cast<const float4*>(rows + (2 * ty + i) * LD + d);
#pragma unroll
    for (int c = 0; c < NC; ++c) k[c] = *reinterpret_cast<const float4*>(cols + (tx + 16 * c) * LD + d);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int c = 0; c < NC; ++c)
        acc[i][c] = fmaf(r[i].w, k[c].w, fmaf(r[i].z, k[c].z, fmaf(r[i].y, k[c].y, fmaf(r[i].x, k[c].x, acc[i][c]))));
  }
}
// o[i][cc] += sum_j w[2 ty + i][j] cols[j][4 tx + 64 cc ..] over the tile's first n columns (n <= 64)
template <int CC, int W_LD = FP_LD>
__device__ __forceinline__ void accumulate(const float* w, const float* cols, int LD, int D, int n, float4 (&o)[2][CC]) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  for (int j = 0; j < n; j += 4) {
    float4 p[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) p[i] = *reinterpret_cast<const float4*>(w + (2 * ty + i) * W_LD + j);
#pragma unroll
    for (int cc = 0; cc < CC; ++cc) {
      const int d = 4 * tx + 64 * cc;
      if (d >= D) continue;
      float4 v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<const float4*>(cols + (j + e) * LD + d);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float pe[4] = {p[i].x, p[i].y, p[i].z, p[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          o[i][cc].x = fmaf(pe[e], v[e].x, o[i][cc].x);
          o[i][cc].y = fmaf(pe[e], v[e].y, o[i][cc].y);
          o[i][cc].z = fmaf(pe[e], v[e].z, o[i][cc].z);
          o[i][cc].w = fmaf(pe[e], v[e].w, o[i][cc].w);
        }
      }
    }
  }
}
template <typename T>
__device__ __forceinline__ void store_to(T* p, int d, int D, bool vec, const float4& v) {  // p: value d of a row
  if (vec) {
    store4(p, v);
  } else {
    p[0] = from_f32<T>(v.x);
    if (d + 1 < D) p[1] = from_f32<T>(v.y);
    if (d + 2 < D) p[2] = from_f32<T>(v.z);
    if (d + 3 < D) p[3] = from_f32<T>(v.w);
  }
}
template <int CC, typename T>
__device__ __forceinline__ void store_rows(T* X, int64_t ld, int r0, int rows, int D, bool vec, float scale0,
                                           float scale1, const float4 (&o)[2][CC]) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = r0 + 2 * ty + i;
    if (r >= rows) continue;
    const float sc = i ? scale1 : scale0;
#pragma unroll
    for (int cc = 0; cc < CC; ++cc) {
      const int d = 4 * tx + 64 * cc;
      if (d >= D) continue;
      const float4 v = make_float4(o[i][cc].x * sc, o[i][cc].y * sc, o[i][cc].z * sc, o[i][cc].w * sc);
      store_to(X + static_cast<int64_t>(r) * ld + d, d, D, vec, v);
    }
  }
}
__device__ __forceinline__ float half_warp_max(float v) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float half_warp_sum(float v) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// SELF: Q, K and V are blocks of the same rows, as many queries as keys, a key head each.
// Known to the compiler, it is worth 7% of a small forward (3.9 -> 3.5 us at 4 x 32 tokens, 2
// heads of 64).
template <bool SELF>
struct Strides {
  int H, Skv, group;
  int64_t q, k, v, o;
  __device__ explicit Strides(const Geometry& g)
      : H(static_cast<int>(g.ldo)), Skv(SELF ? g.Sq : g.Skv), group(SELF ? 1 : g.group), q(SELF ? 3 * static_cast<int64_t>(H) : g.ldq),
        k(SELF ? q : g.ldk), v(SELF ? q : g.ldv), o(SELF ? H : g.ldo) {}
};

// CTAs an SM that the registers are kept to: three of head dims above 64, whose shared memory
// lets no more fit, four up to 64; up to 32 the compiler's own choice (80 registers) for self
// attention and five for cross attention.  Three for all gave the compiler 141 to 154
// registers, and many CTAs waited for a place (us, three and these): 8 x 512 tokens, 2 heads
// of 64 88 and 56; 32 x 512, 8 of 32 615 and 506; 4 x 32, 2 of 64 3.6 and 3.7; 8 x 300 over
// 512, 8 on 4 of 64 109 and 91, of 32 80 and 69.
template <bool SELF, int G>
constexpr int kFwdCtas = G > 16 ? 3 : G > 8 ? 4 : SELF ? 0 : 5;

template <bool SELF, typename T, int G>
__global__ void __launch_bounds__(F_THR, kFwdCtas<SELF, G>) attn_fwd_simt(const Geometry g, const T* __restrict__ gq,
                                                          const T* __restrict__ gk, const T* __restrict__ gv,
                                                          const int32_t* __restrict__ lens, T* __restrict__ ctx,
                                                          float* __restrict__ lse) {
  using ST = Stage<G>;
  constexpr int CC = ST::CC;
  pdl_wait();
  extern __shared__ __align__(16) float sm[];
  const int LD = g.LD, D = g.D, Sq = g.Sq;
  const bool vec = g.vec;
  float *sq = sm, *sk = sq + FR * LD, *sv = sk + FC * LD, *sp = sv + FC * LD;
  const int tiles = (Sq + FR - 1) / FR;
  const int a = static_cast<int>(blockIdx.x) / tiles, q0 = (static_cast<int>(blockIdx.x) % tiles) * FR, b = blockIdx.y;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const Strides<SELF> ld(g);
  const int len = valid_keys(lens, b, SELF ? 1 : 0, ld.Skv, g.status), kv = a / ld.group;
  const T* q = gq + static_cast<int64_t>(b) * Sq * ld.q + a * D;
  const T* k = SELF ? q + ld.H : gk + static_cast<int64_t>(b) * ld.Skv * ld.k + kv * D;
  const T* v = SELF ? q + 2 * ld.H : gv + static_cast<int64_t>(b) * ld.Skv * ld.v + kv * D;
  const float sc = 1.f / sqrtf((float)D);
  float4 own[ST::OWN];
  load_rows<G>(q, ld.q, q0, Sq, D, vec, own);
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  float4 o[2][CC] = {};
  for (int k0 = 0; k0 < len; k0 += FC) {
    __syncthreads();
// (self attention batch by batch: 4 x 200 tokens, 6 heads of 128 52.9 us unrolled, 49.7 so)
#pragma unroll (SELF ? 1 : ST::BATCHES)
    for (int h = 0; h < ST::BATCHES; ++h) {
      constexpr int R = ST::R;
      float4 kx[ST::PASSES], vx[ST::PASSES];
      load_rows<G>(k, ld.k, k0 + R * h, len, D, vec, kx);
      load_rows<G>(v, ld.v, k0 + R * h, len, D, vec, vx);
      if (h == 0 && k0 == 0) put_rows<G>(sq, LD, D, own);
      put_rows<G>(sk + R * h * LD, LD, D, kx);
      put_rows<G>(sv + R * h * LD, LD, D, vx);
    }
    __syncthreads();
    float s[2][4];
    scores(sq, sk, LD, D, s);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float mx = -INFINITY;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        s[i][c] = k0 + tx + 16 * c < len ? s[i][c] * sc : -INFINITY;
        mx = fmaxf(mx, s[i][c]);
      }
      // (finite also while every score so far is -inf: those keys then add nothing)
      const float mn = fmaxf(fmaxf(m[i], half_warp_max(mx)), -FLT_MAX);
      const float al = expf(m[i] - mn);  // 0 in the first tile
      m[i] = mn;
      float sum = 0.f;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const float e = expf(s[i][c] - mn);  // masked: 0
        sp[(2 * ty + i) * FP_LD + tx + 16 * c] = e;
        sum += e;
      }
      l[i] = l[i] * al + half_warp_sum(sum);
#pragma unroll
      for (int cc = 0; cc < CC; ++cc) {
        o[i][cc].x *= al; o[i][cc].y *= al; o[i][cc].z *= al; o[i][cc].w *= al;
      }
    }
    __syncwarp();
    accumulate<CC>(sp, sv, LD, D, min(FC, len - k0), o);
    __syncwarp();
  }
  pdl_trigger();
  const bool any = SELF || len > 0;
  store_rows<CC>(ctx + static_cast<int64_t>(b) * Sq * ld.o + a * D, ld.o, q0, Sq, D, vec, any ? 1.f / l[0] : 0.f,
                 any ? 1.f / l[1] : 0.f, o);
  if (tx == 0 && (SELF || lse))
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (q0 + 2 * ty + i < Sq)  // (without a key: -inf)
        lse[(static_cast<int64_t>(b) * g.A + a) * Sq + q0 + 2 * ty + i] = (m[i] + logf(l[i])) * 1.4426950408889634f;  // base 2
}

// dQ: own rows are queries (Q, dO), columns keys (K, V).  dK, dV: own rows are keys (K,
// V), columns the queries (Q, dO) of every head of the group, head after head.  Blocks of
// the two kinds alternate, then come what is left of the more numerous.  Either way
//   P = exp2(s log2(e)/sqrt(D) - lse_q),  dS = P (dp - delta_q),
// s and dp the products of the first and second operands; dQ or dK = dS . first
// operand of the columns / sqrt(D), dV = P . dO.  Four CTAs an SM (128 registers) are
// faster up to a head dim of 64 (29.8 us against 34.7 at 4 x 101, 12 heads), above it
// the registers are (50.6 against 57.0 at 2 x 200, 6 heads of 128).
//
// Not SELF: where a block has many columns and there are few blocks, the CTAs of a cluster
// share its columns and add their parts.
struct Splits {
  int ks;           // CTAs of a cluster; 1: none, blocks of the two kinds alternate
  bool keys_first;  // the kind with the longer blocks comes first
  bool whole[2];    // whether the first kind's blocks, and the second's, are left whole
};
enum Kind { SELF_ATTENTION, CROSS, CROSS_SPLIT };
template <Kind KIND, typename T, int G, int NC>
__global__ void __launch_bounds__(F_THR, G > 16 ? 1 : 4) attn_bwd_simt(const Geometry g, const T* __restrict__ gq,
                                                      const T* __restrict__ gk, const T* __restrict__ gv,
                                                      const int32_t* __restrict__ lens, const T* __restrict__ dctx,
                                                      const float* __restrict__ lse, const float* __restrict__ delta,
                                                      T* __restrict__ dq, T* __restrict__ dk, T* __restrict__ dv,
                                                      const Splits sp) {
  constexpr bool SELF = KIND == SELF_ATTENTION, SPLIT = KIND == CROSS_SPLIT;
  using ST = Stage<G, NC>;
  constexpr int CC = ST::CC, TC = ST::ROWS, P_LD = TC + 4;
  pdl_wait();
  extern __shared__ __align__(16) float sm[];
  const Strides<SELF> ld(g);
  const int LD = g.LD, D = g.D, Sq = g.Sq, Skv = ld.Skv;
  const bool vec = g.vec;
  float *r0s = sm, *r1s = r0s + FR * LD, *c0s = r1s + FR * LD, *c1s = c0s + TC * LD;
  float *sds = c1s + TC * LD, *sps = sds + FR * P_LD, *sl = sps + FR * P_LD, *sd = sl + TC;
  const int qtiles = (Sq + FR - 1) / FR, ktiles = (Skv + FR - 1) / FR;
  const int qunits = qtiles * g.A, kunits = ktiles * (g.A / ld.group);
  // its place: kind, number within the kind, and part of the columns
  int x = blockIdx.x, split = 0, splits = 1;
  bool keys;  // own rows are keys
  if (SELF) {
    keys = x & 1;
    x >>= 1;
  } else if (!SPLIT) {
    const int both = min(qunits, kunits);
    keys = x < 2 * both ? x & 1 : qunits < kunits;
    x = x < 2 * both ? x >> 1 : x - both;
  } else {  // clusters of one kind, then of the other: a block each, or one of every CTA
    const int n = sp.keys_first ? kunits : qunits, first = sp.whole[0] ? (n + sp.ks - 1) / sp.ks * sp.ks : n * sp.ks;
    const bool second = x >= first;
    keys = second != sp.keys_first;
    if (second) x -= first;
    if (!sp.whole[second]) {
      splits = sp.ks;
      split = x % splits;
      x /= splits;
    } else if (x >= (keys ? kunits : qunits)) {
      return;
    }
  }
  const int tiles = keys ? ktiles : qtiles;
  const int head = x / tiles, r0 = (x % tiles) * FR, b = blockIdx.y;  // of its kind
  const int kv = keys ? head : head / ld.group, heads = keys ? ld.group : 1;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int len = valid_keys(lens, b, SELF ? 1 : 0, Skv, g.status);
  const T* self = gq + static_cast<int64_t>(b) * Sq * ld.q + head * D;  // (of queries)
  const T* k = SELF ? self + ld.H : gk + static_cast<int64_t>(b) * Skv * ld.k + kv * D;
  const T* v = SELF ? self + 2 * ld.H : gv + static_cast<int64_t>(b) * Skv * ld.v + kv * D;
  const float sc = 1.f / sqrtf((float)D), sl2 = sc * 1.4426950408889634f;
  float4 o0[2][CC] = {}, o1[2][CC] = {};
  const int rows = keys ? Skv : Sq, cols = keys ? Sq : len;
  float4 own0[ST::OWN], own1[ST::OWN];
  const int ctiles = (cols + TC - 1) / TC, all = keys && r0 >= len ? 0 : heads * ctiles;
  const int begin = SPLIT ? split * all / splits : 0, end = SPLIT ? (split + 1) * all / splits : all;
  float lr[2] = {}, dr[2] = {};
  if (begin < end) {
    const T* dO = dctx + static_cast<int64_t>(b) * Sq * ld.o + head * D;  // (of queries)
    load_rows<G>(keys ? k : self, keys ? ld.k : ld.q, r0, rows, D, vec, own0);
    load_rows<G>(keys ? v : dO, keys ? ld.v : ld.o, r0, rows, D, vec, own1);
    if (!keys)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int64_t r = (static_cast<int64_t>(b) * g.A + head) * Sq + min(r0 + 2 * ty + i, Sq - 1);
        lr[i] = lse[r];
        dr[i] = delta[r];
      }
  }
  int h = SPLIT && begin < end ? begin / ctiles : 0, from = SPLIT ? begin - h * ctiles : 0;
  for (int left = end - begin; left > 0; ++h, from = 0, left = SELF ? 0 : left) {  // a head's tiles
    const int a = !SELF && keys ? kv * ld.group + h : head, to = SPLIT ? min(ctiles, from + left) : ctiles;
    const T* q = SELF ? self : gq + static_cast<int64_t>(b) * Sq * ld.q + a * D;
    const T* dO = dctx + static_cast<int64_t>(b) * Sq * ld.o + a * D;
    const float *lse_b = lse + (static_cast<int64_t>(b) * g.A + a) * Sq, *del_b = delta + (static_cast<int64_t>(b) * g.A + a) * Sq;
    const bool first = SELF || left == end - begin;
    left -= to - from;
    for (int c0 = from * TC; c0 < to * TC; c0 += TC) {
      __syncthreads();
      // columns: queries (Q, dO; all S) or keys (K, V; the valid ones)
      const T *x0 = keys ? q : k, *x1 = keys ? dO : v;
      float lc = 0.f, dc = 0.f;
      if (keys && threadIdx.x < TC) {
        const int c = min(c0 + static_cast<int>(threadIdx.x), Sq - 1);
        lc = lse_b[c];
        dc = del_b[c];
      }
#pragma unroll
      for (int t = 0; t < ST::BATCHES; ++t) {
        constexpr int R = ST::R;
        float4 v0[ST::PASSES], v1[ST::PASSES];
        load_rows<G>(x0, keys ? ld.q : ld.k, c0 + R * t, cols, D, vec, v0);
        load_rows<G>(x1, keys ? ld.o : ld.v, c0 + R * t, cols, D, vec, v1);
        if (t == 0 && first && c0 == from * TC) {
          put_rows<G>(r0s, LD, D, own0);
          put_rows<G>(r1s, LD, D, own1);
        }
        put_rows<G>(c0s + R * t * LD, LD, D, v0);
        put_rows<G>(c1s + R * t * LD, LD, D, v1);
      }
      if (keys && threadIdx.x < TC) {
        sl[threadIdx.x] = lc;
        sd[threadIdx.x] = dc;
      }
      __syncthreads();
      float s[2][NC], dp[2][NC];
      scores(r0s, c0s, LD, D, s);
      scores(r1s, c1s, LD, D, dp);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const int cl = tx + 16 * c;
          const bool live = c0 + cl < cols && (!keys || r0 + 2 * ty + i < len);
          const float p = live ? exp2f(fmaf(s[i][c], sl2, -(keys ? sl[cl] : lr[i]))) : 0.f;
          sds[(2 * ty + i) * P_LD + cl] = live ? p * (dp[i][c] - (keys ? sd[cl] : dr[i])) : 0.f;
          if (keys) sps[(2 * ty + i) * P_LD + cl] = p;
        }
      __syncwarp();
      const int n = min(TC, cols - c0);
      accumulate<CC, P_LD>(sds, c0s, LD, D, n, o0);
      if (keys) accumulate<CC, P_LD>(sps, c1s, LD, D, n, o1);
      __syncwarp();
    }
  }
  pdl_trigger();
  T* out = dq + static_cast<int64_t>(b) * Sq * ld.q + head * D;
  T* out_k = SELF ? out + ld.H : dk + static_cast<int64_t>(b) * Skv * ld.k + kv * D;
  T* out_v = SELF ? out + 2 * ld.H : dv + static_cast<int64_t>(b) * Skv * ld.v + kv * D;
  if (!SPLIT || splits == 1) {
    store_rows<CC>(keys ? out_k : out, keys ? ld.k : ld.q, r0, rows, D, vec, sc, sc, o0);
    if (keys) store_rows<CC>(out_v, ld.v, r0, rows, D, vec, 1.f, 1.f, o1);
    return;
  }
  // the parts, over the columns' tiles, and FR / splits rows of their sum, in split order
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int cc = 0; cc < CC; ++cc) {
      const int d = 4 * tx + 64 * cc;
      if (d >= D) continue;
      *reinterpret_cast<float4*>(c0s + (2 * ty + i) * LD + d) = o0[i][cc];
      if (keys) *reinterpret_cast<float4*>(c1s + (2 * ty + i) * LD + d) = o1[i][cc];
    }
  ptx::cluster_sync();
  const int groups = (D + 3) / 4, mine = FR / splits;
  for (int e = threadIdx.x; e < mine * groups; e += F_THR) {
    const int lr_ = split * mine + e / groups, d = e % groups * 4, r = r0 + lr_;
    if (r >= rows) continue;
    for (int which = 0; which < (keys ? 2 : 1); ++which) {
      const uint32_t at = ptx::smem_u32((which ? c1s : c0s) + lr_ * LD + d);
      float4 u = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int c = 0; c < splits; ++c) {
        const float4 w = ptx::ld_cluster_f4(ptx::mapa_shared(at, c));
        u.x += w.x; u.y += w.y; u.z += w.z; u.w += w.w;
      }
      if (!which) u = make_float4(u.x * sc, u.y * sc, u.z * sc, u.w * sc);
      const int64_t ldr = !keys ? ld.q : which ? ld.v : ld.k;
      store_to((!keys ? out : which ? out_v : out_k) + r * ldr + d, d, D, vec, u);
    }
  }
  ptx::cluster_sync();  // the peers have read this CTA's part
}

// delta of bf16 storage: the sum over the keys of P dP.  dot(dctx, ctx) is the same sum, but of
// a rounded ctx it is off by up to 2^-8 sum |dctx ctx|, the same for every key of the row,
// which a mean of V makes larger than dS.  Own rows are queries, columns keys, as for dQ; the
// CTAs of a cluster share a block's columns.  Two of the backward's seven products once more
// (us, from the rounded ctx and this): 4 x 200 over 333, 8 heads on 2 of 128 210 and 264; 8 x
// 300 over 512, 8 on 4 of 32 265 and 320; 10 over 3000, 4 on 1 of 128 61 and 96.
template <typename T, int G>
__global__ void __launch_bounds__(F_THR, G > 16 ? 2 : 4) attn_delta_keys(const Geometry g, const T* __restrict__ gq,
                                                                         const T* __restrict__ gk, const T* __restrict__ gv,
                                                                         const int32_t* __restrict__ lens,
                                                                         const T* __restrict__ dctx,
                                                                         const float* __restrict__ lse,
                                                                         float* __restrict__ delta, int splits) {
  using ST = Stage<G>;
  pdl_wait();
  extern __shared__ __align__(16) float sm[];
  const int LD = g.LD, D = g.D, Sq = g.Sq;
  float *r0s = sm, *r1s = r0s + FR * LD, *c0s = r1s + FR * LD, *c1s = c0s + FC * LD, *part = c1s + FC * LD;
  const int tiles = (Sq + FR - 1) / FR, split = static_cast<int>(blockIdx.x) % splits, x = static_cast<int>(blockIdx.x) / splits;
  const int a = x / tiles, q0 = (x % tiles) * FR, b = blockIdx.y, kv = a / g.group;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int len = valid_keys(lens, b, 0, g.Skv, g.status);
  const T* q = gq + static_cast<int64_t>(b) * Sq * g.ldq + a * D;
  const T* dO = dctx + static_cast<int64_t>(b) * Sq * g.ldo + a * D;
  const T* k = gk + static_cast<int64_t>(b) * g.Skv * g.ldk + kv * D;
  const T* v = gv + static_cast<int64_t>(b) * g.Skv * g.ldv + kv * D;
  const int64_t at = (static_cast<int64_t>(b) * g.A + a) * Sq;
  const float sl2 = 1.f / sqrtf((float)D) * 1.4426950408889634f;
  const int all = (len + FC - 1) / FC, begin = split * all / splits, end = (split + 1) * all / splits;
  float lr[2], d[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 2; ++i) lr[i] = lse[at + min(q0 + 2 * ty + i, Sq - 1)];
  if (begin < end) {
    float4 own0[ST::OWN], own1[ST::OWN];
    load_rows<G>(q, g.ldq, q0, Sq, D, g.vec, own0);
    load_rows<G>(dO, g.ldo, q0, Sq, D, g.vec, own1);
    put_rows<G>(r0s, LD, D, own0);
    put_rows<G>(r1s, LD, D, own1);
  }
  for (int c0 = begin * FC; c0 < end * FC; c0 += FC) {
    __syncthreads();
#pragma unroll
    for (int t = 0; t < ST::BATCHES; ++t) {
      constexpr int R = ST::R;
      float4 v0[ST::PASSES], v1[ST::PASSES];
      load_rows<G>(k, g.ldk, c0 + R * t, len, D, g.vec, v0);
      load_rows<G>(v, g.ldv, c0 + R * t, len, D, g.vec, v1);
      put_rows<G>(c0s + R * t * LD, LD, D, v0);
      put_rows<G>(c1s + R * t * LD, LD, D, v1);
    }
    __syncthreads();
    float s[2][4], dp[2][4];
    scores(r0s, c0s, LD, D, s);
    scores(r1s, c1s, LD, D, dp);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (c0 + tx + 16 * c < len) d[i] = fmaf(exp2f(fmaf(s[i][c], sl2, -lr[i])), dp[i][c], d[i]);
  }
  pdl_trigger();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    d[i] = half_warp_sum(d[i]);
    if (tx == 0) part[2 * ty + i] = d[i];
  }
  if (splits > 1) ptx::cluster_sync();
  else __syncthreads();
  const int r = 2 * static_cast<int>(threadIdx.x);
  if (split == 0 && r < FR) {  // two rows a thread, in split order
    float2 sum = *reinterpret_cast<const float2*>(part + r);
    for (int c = 1; c < splits; ++c) {
      const float2 w = ptx::ld_cluster_f2(ptx::mapa_shared(ptx::smem_u32(part + r), c));
      sum.x += w.x;
      sum.y += w.y;
    }
    if (q0 + r < Sq) delta[at + q0 + r] = sum.x;
    if (q0 + r + 1 < Sq) delta[at + q0 + r + 1] = sum.y;
  }
  if (splits > 1) ptx::cluster_sync();  // the first CTA has read the sums
}

// Launch shape: the shared row stride (four floats past the head dim, so the 16 lanes of
// a score product read different banks) and the bytes it makes.
constexpr int row_stride(int D) { return (D + 3) / 4 * 4 + 4; }
constexpr int fwd_smem(int D) { return ((FR + 2 * FC) * row_stride(D) + FR * FP_LD) * 4; }
constexpr int delta_smem(int D) { return ((2 * FR + 2 * FC) * row_stride(D) + FR) * 4; }
constexpr int bwd_smem(int D, int NC) {
  return ((2 * FR + 32 * NC) * row_stride(D) + 2 * FR * (16 * NC + 4) + 32 * NC) * 4;
}
template <int G>
using Group = std::integral_constant<int, G>;
// Whether every head row allows 4-value accesses.
template <typename T>
bool rows_of_4(const Geometry& g, const void* ctx, const void* x = nullptr, const void* y = nullptr,
               const void* z = nullptr) {
  const auto on = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % (4 * sizeof(T)) == 0; };
  return g.D % 4 == 0 && (g.ldq | g.ldk | g.ldv | g.ldo) % 4 == 0 && on(g.q) && on(g.k) && on(g.v) && on(ctx) && on(x) &&
         on(y) && on(z);
}

template <bool SELF, typename T>
cudaError_t fwd_simt(Geometry g, int B, T* ctx, float* lse, cudaStream_t stream) {
  g.LD = row_stride(g.D);
  g.vec = rows_of_4<T>(g, ctx);
  const auto go = [&](auto group, auto kern) {  // `group` threads a row: head dims up to four times that
    static OncePerDevice once;
    const cudaError_t e = allow_smem(once, kern, fwd_smem(4 * decltype(group)::value));
    if (e != cudaSuccess) return e;
    return launch_pdl(kern, dim3((unsigned)ceil_div(g.Sq, FR) * g.A, B), dim3(F_THR), fwd_smem(g.D), stream, 1, g,
                      static_cast<const T*>(g.q), static_cast<const T*>(g.k), static_cast<const T*>(g.v), g.lens, ctx, lse);
  };
  count_launches(1);
  return g.D <= 32   ? go(Group<8>{}, attn_fwd_simt<SELF, T, 8>)
         : g.D <= 64 ? go(Group<16>{}, attn_fwd_simt<SELF, T, 16>)
                     : go(Group<32>{}, attn_fwd_simt<SELF, T, 32>);
}

// The columns of the kind that has more of them, and of the other where it has more than is
// then left to a CTA, are split while the longest block takes about as long as the SMs'
// share of all work: to a step each where the CTAs all fit at once, two where they take up
// to four rounds.  us, whole and split, heads of 64 unless stated: 6 queries of 6 heads of
// 128 on 2, 1650 keys 182 and 40; 9 x 468, 4 on 1, 6 keys 199 and 51; 2 x 182, 8 on 2, 38
// keys 105 and 28; 3 x 51, one of 128, 340 keys 41 and 19; 2 x 605, 6 of 128, 37 keys 124
// and 54.  Beyond these limits: 2 x 57, 12 of 128 on 6, 177 keys (a step each, more than a
// round) 34 and 43; 10 x 490, 6 of 32, 69 keys (eight rounds) 97 and 248; 116, 24 of 128 on
// 6, 1453 keys (balanced whole) 370 and 435.  Tiles of 16 columns are left whole.
Splits bwd_splits(const Geometry& g, int B, unsigned* blocks) {
  const int64_t units[2] = {static_cast<int64_t>(ceil_div(g.Sq, FR)) * g.A,
                            static_cast<int64_t>(ceil_div(g.Skv, FR)) * (g.A / g.group)};  // queries, keys
  const int steps[2] = {ceil_div(g.Skv, FC), ceil_div(g.Sq, FC) * g.group};
  const bool keys = steps[1] > steps[0];
  const int64_t room = static_cast<int64_t>(sm_count() > 0 ? sm_count() : 148) * (g.D > 64 ? 2 : 4);
  const int64_t all = (units[0] * steps[0] + units[1] * steps[1]) * B;
  Splits sp{1, keys, {true, true}};
  for (int ks = 2; ks <= 8 && steps[keys] >= ks && std::max(g.Sq, g.Skv) > 16; ks *= 2) {
    const bool whole = steps[!keys] <= ceil_div(steps[keys], ks);  // the shorter kind
    const int64_t n = ks * (units[keys] + (whole ? ceil_div(units[!keys], ks) : units[!keys]));
    if (n * B > 4 * room || (n * B > room && steps[keys] < 2 * ks)) break;
    if (9 * room * ceil_div(steps[keys], ks / 2) < 8 * all) break;
    sp = {ks, keys, {false, whole}};
    *blocks = static_cast<unsigned>(n);
  }
  return sp;
}

// A block's keys over a cluster while the CTAs all fit at once and each keeps two tiles (us,
// whole and split: 10 queries, 4 heads on 1 of 128, 3000 keys 316 and 96; 60, 4 heads of 32,
// 700 keys 45 and 25).
template <typename T>
cudaError_t delta_keys(const Geometry& g, int B, const T* dctx, const float* lse, float* delta, cudaStream_t stream) {
  const int64_t blocks = static_cast<int64_t>(ceil_div(g.Sq, FR)) * g.A;
  const int64_t room = static_cast<int64_t>(sm_count() > 0 ? sm_count() : 148) * (g.D > 64 ? 2 : 4);
  int ks = 1;
  while (ks < 8 && 2 * ks * blocks * B <= room && ceil_div(g.Skv, FC) >= 4 * ks) ks *= 2;
  const auto go = [&](auto group) {
    constexpr int G = decltype(group)::value;
    static OncePerDevice once;
    const cudaError_t e = allow_smem(once, attn_delta_keys<T, G>, delta_smem(4 * G));
    if (e != cudaSuccess) return e;
    return launch_pdl(attn_delta_keys<T, G>, dim3(static_cast<unsigned>(blocks * ks), B), dim3(F_THR), delta_smem(g.D),
                      stream, ks, g, static_cast<const T*>(g.q), static_cast<const T*>(g.k), static_cast<const T*>(g.v),
                      g.lens, dctx, lse, delta, ks);
  };
  return g.D <= 32 ? go(Group<8>{}) : g.D <= 64 ? go(Group<16>{}) : go(Group<32>{});
}

template <bool SELF, typename T>
cudaError_t bwd_simt(Geometry g, int B, const T* ctx, const T* dctx, const float* lse, float* delta, T* dq, T* dk,
                     T* dv, cudaStream_t stream) {
  g.LD = row_stride(g.D);
  g.vec = rows_of_4<T>(g, dctx, dq, dk, dv);
  cudaError_t le;
  if constexpr (std::is_same<T, float>::value) {
    const int64_t rows = static_cast<int64_t>(B) * g.Sq;
    le = launch_pdl(attn_delta<T>, dim3(ceil_div(rows * g.A * 32, 256)), dim3(256), 0, stream, 1, ctx, dctx, g.Sq, g.ldo,
                    g.A, g.D, rows, delta);
  } else {
    le = delta_keys(g, B, dctx, lse, delta, stream);
  }
  count_launches(2);
  if (le != cudaSuccess) return le;
  Splits sp{1, false, {true, true}};
  unsigned blocks = (unsigned)ceil_div(g.Sq, FR) * g.A + (unsigned)ceil_div(g.Skv, FR) * (g.A / g.group);
  if (!SELF) sp = bwd_splits(g, B, &blocks);
  const auto go = [&](auto group, auto nc, auto kern) {
    constexpr int G = decltype(group)::value, NC = decltype(nc)::value;
    static OncePerDevice once[2];  // (both cross kinds have the same type)
    const cudaError_t e = allow_smem(once[sp.ks > 1], kern, bwd_smem(4 * G, NC));
    if (e != cudaSuccess) return e;
    return launch_pdl(kern, dim3(blocks, B), dim3(F_THR), bwd_smem(g.D, NC), stream, sp.ks, g,
                      static_cast<const T*>(g.q), static_cast<const T*>(g.k), static_cast<const T*>(g.v), g.lens, dctx, lse,
                      static_cast<const float*>(delta), dq, dk, dv, sp);
  };
  // Up to 16 tokens a 64-column tile is mostly empty: 128 x 8 tokens, 6 heads of 128
  // 52.4 us with it, 27.8 with 16 columns (a warp a row 28.8); 12 of 64 45.2 and 25.5
  // (41.1); 64 x 16, 12 of 64 29.8 and 18.3 (70.4).
  const auto width = [&](auto group) {
    constexpr int G = decltype(group)::value;
    constexpr Kind WHOLE = SELF ? SELF_ATTENTION : CROSS;
    if constexpr (!SELF)
      if (sp.ks > 1) return go(group, std::integral_constant<int, 4>{}, attn_bwd_simt<CROSS_SPLIT, T, G, 4>);
    return std::max(g.Sq, g.Skv) <= 16 ? go(group, std::integral_constant<int, 1>{}, attn_bwd_simt<WHOLE, T, G, 1>)
                                       : go(group, std::integral_constant<int, 4>{}, attn_bwd_simt<WHOLE, T, G, 4>);
  };
  return g.D <= 32 ? width(Group<8>{}) : g.D <= 64 ? width(Group<16>{}) : width(Group<32>{});
}

template <typename T>
cudaError_t launch_fwd_simt(const Geometry& g, int B, T* ctx, float* lse, cudaStream_t stream) {
  return fwd_simt<false>(g, B, ctx, lse, stream);
}
template <typename T>
cudaError_t launch_bwd_simt(const Geometry& g, int B, const T* ctx, const T* dctx, const float* lse, float* delta, T* dq,
                            T* dk, T* dv, cudaStream_t stream) {
  return bwd_simt<false>(g, B, ctx, dctx, lse, delta, dq, dk, dv, stream);
}
template cudaError_t launch_fwd_simt(const Geometry&, int, float*, float*, cudaStream_t);
template cudaError_t launch_fwd_simt(const Geometry&, int, __nv_bfloat16*, float*, cudaStream_t);
template cudaError_t launch_bwd_simt(const Geometry&, int, const float*, const float*, const float*, float*, float*, float*,
                                     float*, cudaStream_t);
template cudaError_t launch_bwd_simt(const Geometry&, int, const __nv_bfloat16*, const __nv_bfloat16*, const float*, float*,
                                     __nv_bfloat16*, __nv_bfloat16*, __nv_bfloat16*, cudaStream_t);

// Packed QKV rows of H-wide blocks.
static Geometry packed(const float* q, const int32_t* lens, int S, int H, int A, int32_t* status) {
  const int64_t rs = 3 * static_cast<int64_t>(H);
  return {q, q + H, q + 2 * H, rs, rs, rs, H, S, S, A, 1, H / A, 0, false, lens, status};
}
cudaError_t launch_fwd_self(const float* qkv, const int32_t* lens, int B, int S, int H, int A, float* ctx, float* lse,
                            int32_t* status, cudaStream_t stream) {
  return fwd_simt<true>(packed(qkv, lens, S, H, A, status), B, ctx, lse, stream);
}
cudaError_t launch_bwd_self(const float* qkv, const float* ctx, const float* dctx, const float* lse, const int32_t* lens,
                            int B, int S, int H, int A, float* delta, float* dqkv, cudaStream_t stream) {
  return bwd_simt<true>(packed(qkv, lens, S, H, A, nullptr), B, ctx, dctx, lse, delta, dqkv, dqkv + H, dqkv + 2 * H, stream);
}

}  // namespace attn
}  // namespace sky
