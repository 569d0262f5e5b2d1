// Cross attention of few query rows: the step of a decoder that writes token by token.
// The rows of one key head, q_len * group of them (row r: query r / group, head r %
// group), are at most 16, or 32 over many keys, so a key or value is read for a handful of
// products and the kernels are bound by those reads.  Keys are split over the warps of a
// CTA and the CTAs of a cluster, in chunks of 32 dealt out in turn; each warp keeps m, l
// and O of its chunks (a softmax in one pass), and the parts are joined in the order of
// warps, then of CTAs: m the largest, l and O scaled to it.
//
// What lies behind the valid keys reaches nothing: scores there are replaced by -inf, and
// V's rows are cleared before a product takes them.
#include <cuda.h>

#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "attention_few.h"
#include "attention_tc.h"
#include "common.cuh"
#include "ptx.cuh"
#include "row4.cuh"

namespace sky {
namespace few {

constexpr int CHUNK = 32, NW = 4;  // keys; warps of a CTA
constexpr float LOG2E = 1.4426950408889634f;
constexpr uint64_t kTimeoutNs = 2000000000;  // of a wait, as in the other kernels

struct Params {
  attn::Geometry g;
  int all_rows;  // of a key head
  float scale;  // log2(e) / sqrt(D)
  void* ctx;
  float* lse;  // or null
};

// One part of a row: what a warp, or a CTA, has of it.
struct Part {
  float m = -FLT_MAX, l = 0.f;
  float4 o = {0.f, 0.f, 0.f, 0.f};
  __device__ void add(const float2& ml, const float4& x) {  // m is the largest already
    const float s = exp2f(ml.x - m);
    l += s * ml.y;
    o.x += s * x.x; o.y += s * x.y; o.z += s * x.z; o.w += s * x.w;
  }
};

// Joins the parts: O[w][ROWS][LD] and ml[w][ROWS] of this CTA's warps in shared memory,
// then one part of every CTA of the cluster, and writes ctx and lse of the rows from
// row0 on.  Both passes go over 4-value groups of a row.
template <typename T, int ROWS>
__device__ void join(const Params& p, float* O, float2* ml, int LD, int len, int b, int kv, int row0) {
  const attn::Geometry& g = p.g;
  const int groups = (g.D + 3) / 4, rank = blockIdx.x, ranks = gridDim.x, rows = min(ROWS, p.all_rows - row0);
  const auto finish = [&](const Part& x, int local, int d) {
    const int row = row0 + local, q = row / g.group, a = kv * g.group + row % g.group;
    const float inv = len > 0 ? 1.f / x.l : 0.f;
    T* out = static_cast<T*>(p.ctx) + (static_cast<int64_t>(b) * g.Sq + q) * g.ldo + a * g.D + d;
    const float v[4] = {x.o.x * inv, x.o.y * inv, x.o.z * inv, x.o.w * inv};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (d + i < g.D) out[i] = from_f32<T>(v[i]);
    // (without a key: log2 of 0)
    if (d == 0 && p.lse) p.lse[(static_cast<int64_t>(b) * g.A + a) * g.Sq + q] = x.m + log2f(x.l);
  };
  __syncthreads();
  for (int e = threadIdx.x; e < rows * groups; e += NW * 32) {
    const int row = e / groups, d = e % groups * 4;
    Part x;
#pragma unroll
    for (int w = 0; w < NW; ++w) x.m = fmaxf(x.m, ml[w * ROWS + row].x);
#pragma unroll
    for (int w = 0; w < NW; ++w)
      x.add(ml[w * ROWS + row], *reinterpret_cast<const float4*>(O + (w * ROWS + row) * LD + d));
    if (ranks == 1) {
      finish(x, row, d);
      continue;
    }
    *reinterpret_cast<float4*>(O + row * LD + d) = x.o;  // over what this thread has read
    if (d == 0) ml[NW * ROWS + row] = make_float2(x.m, x.l);
  }
  if (ranks == 1) return;
  ptx::cluster_sync();
  const uint32_t so = ptx::smem_u32(O), sml = ptx::smem_u32(ml + NW * ROWS);
  for (int e = rank * NW * 32 + threadIdx.x; e < rows * groups; e += ranks * NW * 32) {
    const int row = e / groups, d = e % groups * 4;
    Part x;
    for (int c = 0; c < ranks; ++c) x.m = fmaxf(x.m, ptx::ld_cluster_f2(ptx::mapa_shared(sml + row * 8, c)).x);
    for (int c = 0; c < ranks; ++c)
      x.add(ptx::ld_cluster_f2(ptx::mapa_shared(sml + row * 8, c)),
            ptx::ld_cluster_f4(ptx::mapa_shared(so + (row * LD + d) * 4, c)));
    finish(x, row, d);
  }
  ptx::cluster_sync();  // the peers have read this CTA's part
}

// ------------------------------------------------------ bf16, head dim 64
// mma.sync m16n8k16: 16 rows suffice, where the 128-row tiles of tcgen05 would be empty.
// Each warp has a ring of its own: one lane brings a chunk's K and V by TMA into
// 128-byte-swizzled rows, the warp reads the fragments with ldmatrix (K as it lies, V
// transposed), and the stage is free again when they are in registers.  No warp waits
// for another before the parts are joined.
//
// One token of 32 requests, 256..512 keys, 16 heads: 11.2 us, 50 MB at 4.5 TB/s; the
// reads alone would take 7.4, launch, first loads and joining are the rest (2.4 us with
// three keys).  Long sources pay for the longest: 4 of 5000..20000 keys, 4 key heads, 13.3
// (floor 7.6); a warp takes 0.45 us a chunk, whose latency two stages and three CTAs an SM
// cover (told to stay at three, the compiler takes 108 registers for 80: 11.6 and 13.6
// before).  Measured against that form (us, the two cases): fragments loaded by the lanes
// themselves with cp.async, 323 instructions a 16-key chunk, 14.9 and 21.0; three stages
// 15.4 and 18.1 (two CTAs an SM); chunks of 16 11.5 and 14.6; eight warps a CTA 17.4 and
// 22.2; copies issued under lane == 0 13.3 and 14.5 (their operands then go to uniform
// registers one by one).
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldmatrix4t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}

constexpr int STAGES = 2, TILE = CHUNK * 128;  // bytes of a chunk's K or V
constexpr int MMA_ROWS = 32, MMA_LD = 64 + 4;  // at most
constexpr int RINGS = NW * STAGES * 2 * TILE, PARTS = (NW * MMA_ROWS * MMA_LD) * 4 + (NW + 1) * MMA_ROWS * 8;
constexpr int BARS = RINGS > PARTS ? RINGS : PARTS;  // the parts go over the rings
constexpr int MMA_SMEM = BARS + NW * STAGES * 8 + 1024;

// H: blocks of eight rows that hold any, two to a 16-row operand
template <int H>
__global__ void __launch_bounds__(NW * 32, 3) attn_few_mma(const __grid_constant__ CUtensorMap tmK,
                                                        const __grid_constant__ CUtensorMap tmV, const Params p) {
  constexpr int M = (H + 1) / 2, ROWS = 16 * M;
  const auto used = [](int i, int h) { return 2 * i + h < H; };  // half h of operand i
  extern __shared__ uint8_t raw[];
  uint8_t* sm = raw + (((ptx::smem_u32(raw) + 1023u) & ~1023u) - ptx::smem_u32(raw));
  const attn::Geometry& geo = p.g;
  // (the warp's number from one lane, so that what the copies take is known to be uniform)
  const int kv = blockIdx.y, b = blockIdx.z, warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
  const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const bool issuer = ptx::elect_one();
  uint64_t* full = reinterpret_cast<uint64_t*>(sm + BARS) + warp * STAGES;
  uint8_t* ring = sm + warp * STAGES * 2 * TILE;
  const int step = gridDim.x * NW, first = blockIdx.x * NW + warp;
  const auto fetch = [&](int n) {  // the warp's chunk n
    const int st = n % STAGES, k0 = (first + n * step) * CHUNK;
    if (!issuer) return;
    ptx::mbar_arrive_expect_tx(&full[st], 2 * TILE);
    ptx::tma_load_4d(ring + st * 2 * TILE, &tmK, &full[st], 0, kv, k0, b);
    ptx::tma_load_4d(ring + st * 2 * TILE + TILE, &tmV, &full[st], 0, kv, k0, b);
  };
  if (issuer) {
    for (int i = 0; i < STAGES; ++i) ptx::mbar_init(&full[i], 1);
    ptx::fence_mbar_init();
    ptx::fence_proxy_async_smem();
  }
  pdl_wait();
  // the first chunks are on their way before the length is known: those that the tensors
  // have room for
  const int room = (geo.Skv + CHUNK - 1) / CHUNK;
  int fetched = min(STAGES, room > first ? (room - first + step - 1) / step : 0);
  for (int n = 0; n < fetched; ++n) fetch(n);
  const int len = attn::valid_keys(geo.lens, b, 0, geo.Skv, geo.status);
  const int chunks = (len + CHUNK - 1) / CHUNK;
  const int mine = chunks > first ? (chunks - first + step - 1) / step : 0;
  uint32_t qa[M][4][4];
  float o[M][8][4] = {}, m[M][2], l[M][2];
#pragma unroll
  for (int i = 0; i < M; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = g + 8 * (2 * i + h), q = row / geo.group, a = kv * geo.group + row % geo.group;
      const __nv_bfloat16* s = static_cast<const __nv_bfloat16*>(geo.q) +
                               (static_cast<int64_t>(b) * geo.Sq + q) * geo.ldq + a * 64 + 2 * c;
#pragma unroll
      for (int k = 0; k < 8; ++k)
        qa[i][k >> 1][h + 2 * (k & 1)] =
            used(i, h) && row < p.all_rows ? *reinterpret_cast<const uint32_t*>(s + 8 * k) : 0u;
      m[i][h] = -INFINITY;
      l[i][h] = 0.f;
    }
  __syncwarp();  // the barriers are ready
  // ldmatrix rows of the lane (16-byte piece i of row r is at i ^ (r & 7)): K: key lane %
  // 8 of an 8-key tile, piece lane / 8 (+ 4); V: key lane % 16 of a 16-key step, piece
  // lane / 16 (+ 2 d)
  const uint32_t base = ptx::smem_u32(ring);
  const uint32_t krow = (lane & 7) * 128, vrow = TILE + (lane & 15) * 128;
  bool ok = true;
  for (int n = 0; n < mine; ++n) {
    const int st = n % STAGES, left = len - (first + n * step) * CHUNK;
    const uint32_t src = base + st * 2 * TILE;
    if (!__all_sync(0xffffffffu, ptx::mbar_wait(&full[st], (n / STAGES) & 1, kTimeoutNs, geo.status))) {
      ok = false;
      break;
    }
    if (left < CHUNK) {  // P is 0 there, and V anything
      for (int i = left * 8 + lane; i < CHUNK * 8; i += 32) ptx::st_shared_v4(src + TILE + i * 16, 0, 0, 0, 0);
      __syncwarp();
    }
    float s[M][CHUNK / 8][4] = {};
#pragma unroll
    for (int t = 0; t < CHUNK / 8; ++t) {
      uint32_t x[4], y[4];
      ldmatrix4(src + t * 1024 + krow + (((lane >> 3) ^ (lane & 7)) << 4), x);
      ldmatrix4(src + t * 1024 + krow + (((4 + (lane >> 3)) ^ (lane & 7)) << 4), y);
#pragma unroll
      for (int i = 0; i < M; ++i) {
        mma16816(s[i][t], qa[i][0], x[0], x[1]);
        mma16816(s[i][t], qa[i][1], x[2], x[3]);
        mma16816(s[i][t], qa[i][2], y[0], y[1]);
        mma16816(s[i][t], qa[i][3], y[2], y[3]);
      }
    }
    if (left < CHUNK) {
#pragma unroll
      for (int i = 0; i < M; ++i)
#pragma unroll
        for (int t = 0; t < CHUNK / 8; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (8 * t + 2 * c + (e & 1) >= left) s[i][t][e] = -INFINITY;
    }
    float nm[M][2], alpha[M][2];
    bool raised = false;
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (!used(i, h)) continue;
        float mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < CHUNK / 8; ++t) mx = fmaxf(mx, fmaxf(s[i][t][2 * h], s[i][t][2 * h + 1]));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        const float mn = fmaxf(fmaxf(m[i][h], mx * p.scale), -FLT_MAX);
        raised |= mn > m[i][h];
        alpha[i][h] = exp2f(m[i][h] - mn);
        m[i][h] = mn;
        nm[i][h] = -mn;
      }
    if (__any_sync(0xffffffffu, raised)) {
#pragma unroll
      for (int i = 0; i < M; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (!used(i, h)) continue;
          l[i][h] *= alpha[i][h];
#pragma unroll
          for (int d = 0; d < 8; ++d) {
            o[i][d][2 * h] *= alpha[i][h];
            o[i][d][2 * h + 1] *= alpha[i][h];
          }
        }
    }
#pragma unroll
    for (int u = 0; u < CHUNK / 16; ++u) {
      uint32_t pa[M][4] = {};
#pragma unroll
      for (int i = 0; i < M; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (!used(i, h)) continue;
            const float e0 = ptx::ex2_ftz(fmaf(s[i][2 * u + t][2 * h], p.scale, nm[i][h]));
            const float e1 = ptx::ex2_ftz(fmaf(s[i][2 * u + t][2 * h + 1], p.scale, nm[i][h]));
            l[i][h] += e0 + e1;
            pa[i][2 * t + h] = ptx::pack_bf16(e0, e1);  // rounded as the tensor cores take it
          }
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        uint32_t v[4];
        ldmatrix4t(src + u * 2048 + vrow + (((2 * d + (lane >> 4)) ^ (lane & 7)) << 4), v);
#pragma unroll
        for (int i = 0; i < M; ++i) {
          mma16816(o[i][2 * d], pa[i], v[0], v[1]);
          mma16816(o[i][2 * d + 1], pa[i], v[2], v[3]);
        }
      }
    }
    __syncwarp();  // the stage is read
    if (n + STAGES < mine) {
      fetch(n + STAGES);
      fetched = n + STAGES + 1;
    }
  }
  // copies behind the length, or behind a wait that ran out
  for (int n = ok ? mine : max(0, fetched - STAGES); n < fetched; ++n)
    ptx::mbar_wait(&full[n % STAGES], (n / STAGES) & 1, kTimeoutNs, geo.status);
  pdl_trigger();
  __syncthreads();  // every warp's ring is read: the parts go over it
  float* O = reinterpret_cast<float*>(sm);
  float2* ml = reinterpret_cast<float2*>(O + NW * ROWS * MMA_LD);
#pragma unroll
  for (int i = 0; i < M; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (!used(i, h)) continue;
      l[i][h] += __shfl_xor_sync(0xffffffffu, l[i][h], 1);
      l[i][h] += __shfl_xor_sync(0xffffffffu, l[i][h], 2);
      const int row = warp * ROWS + g + 8 * (2 * i + h);
#pragma unroll
      for (int d = 0; d < 8; ++d)
        *reinterpret_cast<float2*>(O + row * MMA_LD + 8 * d + 2 * c) = make_float2(o[i][d][2 * h], o[i][d][2 * h + 1]);
      if (c == 0) ml[row] = make_float2(m[i][h], l[i][h]);
    }
  join<__nv_bfloat16, ROWS>(p, O, ml, MMA_LD, len, b, kv, 0);
}

// ------------------------------------------- any type, head dim and alignment
// fp32 arithmetic.  LK lanes of four dims hold a key (LK a power of two, 4 LK >= D), KP =
// 32 / LK keys a pass, LK passes a chunk.  Lane l of key group `sub` ends up with the
// score of pass l, key l KP + sub, so the softmax of a row is a warp's reduction; its
// values are handed back by shuffles as V's rows are read.  A CTA takes up to RB rows.
template <typename T>
__device__ __forceinline__ float4 row4(const T* p, int d, int D, bool vec) {
  if (vec) return d < D ? load4(p + d) : make_float4(0.f, 0.f, 0.f, 0.f);
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = d + i < D ? to_f32(p[d + i]) : 0.f;
  return make_float4(v[0], v[1], v[2], v[3]);
}

// v[i] of the LK lanes of a key group -> in lane l the group's sum of v[l % 8]: three
// steps in which each lane keeps half of its values and hands on the others, then plain
// ones, 7 + log2(LK / 8) shuffles instead of 8 log2(LK).
template <int LK>
__device__ __forceinline__ float sum_of_8(float (&v)[8], int lane) {
#pragma unroll
  for (int k = 4; k >= 1; k >>= 1) {
    const bool upper = (lane & k) != 0;
#pragma unroll
    for (int j = 0; j < k; ++j)
      v[j] = (upper ? v[j + k] : v[j]) + __shfl_xor_sync(0xffffffffu, upper ? v[j] : v[j + k], k);
  }
#pragma unroll
  for (int o = 8; o < LK; o <<= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
  return v[0];
}

template <typename T, int LK, int RB>
__global__ void __launch_bounds__(NW * 32) attn_few_simt(const Params p) {
  constexpr int KP = 32 / LK, PASSES = LK, LD = 4 * LK, BATCH = 8;
  static_assert(CHUNK == 32 && LK >= BATCH, "a pass for every lane of a key");
  __shared__ __align__(16) float O[NW * RB * LD];
  __shared__ float2 ml[(NW + 1) * RB];
  const attn::Geometry& geo = p.g;
  const int blocks = (p.all_rows + RB - 1) / RB;
  const int kv = blockIdx.y / blocks, r0 = blockIdx.y % blocks * RB, b = blockIdx.z;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane / LK, d = lane % LK * 4;
  pdl_wait();
  const int len = attn::valid_keys(geo.lens, b, 0, geo.Skv, geo.status);
  float4 q[RB], o[RB];
  float m[RB], l[RB];
#pragma unroll
  for (int r = 0; r < RB; ++r) {
    const int row = r0 + r, qi = row / geo.group, a = kv * geo.group + row % geo.group;
    q[r] = o[r] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (row < p.all_rows)
      q[r] = row4(static_cast<const T*>(geo.q) + (static_cast<int64_t>(b) * geo.Sq + qi) * geo.ldq + a * geo.D, d, geo.D, geo.vec);
    m[r] = -INFINITY;
    l[r] = 0.f;
  }
  const T* kb = static_cast<const T*>(geo.k) + static_cast<int64_t>(b) * geo.Skv * geo.ldk + kv * geo.D;
  const T* vb = static_cast<const T*>(geo.v) + static_cast<int64_t>(b) * geo.Skv * geo.ldv + kv * geo.D;
  const auto load = [&](const T* base, int64_t ld, int key) {
    return key < len ? row4(base + key * ld, d, geo.D, geo.vec) : make_float4(0.f, 0.f, 0.f, 0.f);
  };
  const int chunks = (len + CHUNK - 1) / CHUNK, step = gridDim.x * NW;
  for (int j = blockIdx.x * NW + warp; j < chunks; j += step) {
    const int k0 = j * CHUNK + sub;  // the lane's key of pass i: k0 + i KP
    float s[RB] = {};
#pragma unroll
    for (int i0 = 0; i0 < PASSES; i0 += BATCH) {
      float4 x[BATCH];
#pragma unroll
      for (int i = 0; i < BATCH; ++i) x[i] = load(kb, geo.ldk, k0 + (i0 + i) * KP);
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        float v[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i)
          v[i] = fmaf(q[r].w, x[i].w, fmaf(q[r].z, x[i].z, fmaf(q[r].y, x[i].y, q[r].x * x[i].x)));
        const float sum = sum_of_8<LK>(v, lane);
        if (lane % LK / BATCH == i0 / BATCH) s[r] = sum;
      }
    }
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      const float x = k0 + lane % LK * KP < len ? s[r] * p.scale : -INFINITY;
      const float mn = fmaxf(fmaxf(m[r], warp_max(x)), -FLT_MAX), alpha = exp2f(m[r] - mn);
      m[r] = mn;
      s[r] = exp2f(x - mn);
      l[r] = l[r] * alpha + s[r];
      o[r].x *= alpha; o[r].y *= alpha; o[r].z *= alpha; o[r].w *= alpha;
    }
#pragma unroll
    for (int i0 = 0; i0 < PASSES; i0 += BATCH) {
      float4 x[BATCH];
#pragma unroll
      for (int i = 0; i < BATCH; ++i) x[i] = load(vb, geo.ldv, k0 + (i0 + i) * KP);
#pragma unroll
      for (int i = 0; i < BATCH; ++i)
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          const float e = __shfl_sync(0xffffffffu, s[r], sub * LK + i0 + i);
          o[r].x = fmaf(e, x[i].x, o[r].x);
          o[r].y = fmaf(e, x[i].y, o[r].y);
          o[r].z = fmaf(e, x[i].z, o[r].z);
          o[r].w = fmaf(e, x[i].w, o[r].w);
        }
    }
  }
  pdl_trigger();
#pragma unroll
  for (int r = 0; r < RB; ++r) {
    l[r] = warp_sum(l[r]);
#pragma unroll
    for (int off = LK; off < 32; off <<= 1) {
      o[r].x += __shfl_xor_sync(0xffffffffu, o[r].x, off);
      o[r].y += __shfl_xor_sync(0xffffffffu, o[r].y, off);
      o[r].z += __shfl_xor_sync(0xffffffffu, o[r].z, off);
      o[r].w += __shfl_xor_sync(0xffffffffu, o[r].w, off);
    }
    if (sub == 0) *reinterpret_cast<float4*>(O + (warp * RB + r) * LD + d) = o[r];
    if (lane == 0) ml[warp * RB + r] = make_float2(m[r], l[r]);
  }
  join<T, RB>(p, O, ml, LD, len, b, kv, r0);
}

}  // namespace few

namespace few {
// The keys of a head over the CTAs of a cluster: doubled up to `most` fourths of a CTA an
// SM, each left more than `keys` of them.  Twice 5/4 CTAs an SM are what still fits at once
// with three an SM.  us: 512 heads of 256..512 keys unsplit 11.2, in two 18; 256 heads of 512
// (16 rows) 6.9 and 13.7, 78 of 10300 13.6 and 18.5 (in two and four); 50 of 2300 in four 6.8,
// in eight 16.4.  A cluster costs 1 to 3 us to start and join, so it is left alone for short
// keys: 48 heads of 442 unsplit 3.8, in two 4.3; 8 of 1167 8.8 in two, four.  The CUDA cores
// take 3 us for a chunk that takes the others 0.5, so shorter shares pay there: 12 heads of
// 300 in two 5.0, unsplit 7.9; 192 of 512 in two 12.6, unsplit 17.5; 32 of 600 13.7 and 30.
int split(int64_t heads, int Skv, int keys, int most) {
  const int sms = sm_count() > 0 ? sm_count() : 148;
  int ctas = 1;
  while (ctas < 16 && 4 * ctas * heads < most * sms && Skv > keys * ctas) ctas *= 2;
  return ctas;
}

// Clusters of more than eight CTAs have to be asked for.
template <typename... KArgs, typename... Args>
cudaError_t launch(OncePerDevice& wide, void (*kern)(KArgs...), dim3 grid, size_t smem, cudaStream_t stream,
                   const Args&... args) {
  if (grid.x > 8) {
    int device = -1;
    cudaError_t e = cudaGetDevice(&device);
    if (e == cudaSuccess)
      e = wide(device, [&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1); });
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(kern, grid, dim3(NW * 32), smem, stream, static_cast<int>(grid.x), args...);
}

float scale(int D) { return LOG2E / sqrtf(static_cast<float>(D)); }

template <typename T>
cudaError_t few_simt(const attn::Geometry& g, int B, T* ctx, float* lse, cudaStream_t stream) {
  const int rows = g.Sq * g.group, Akv = g.A / g.group;
  const Params p{g, rows, scale(g.D), ctx, lse};
  const auto go = [&](auto lanes, auto rb) {
    constexpr int RB = decltype(rb)::value;
    const int heads = Akv * ((rows + RB - 1) / RB);
    static OncePerDevice wide;
    return launch(wide, attn_few_simt<T, decltype(lanes)::value, RB>,
                  dim3(split(static_cast<int64_t>(heads) * B, g.Skv, 128, 8), heads, B), 0, stream, p);
  };
  const auto block = [&](auto lanes) {
    return rows == 1 ? go(lanes, std::integral_constant<int, 1>{}) : go(lanes, std::integral_constant<int, 4>{});
  };
  return g.D <= 32   ? block(std::integral_constant<int, 8>{})
         : g.D <= 64 ? block(std::integral_constant<int, 16>{})
                     : block(std::integral_constant<int, 32>{});
}
}  // namespace few

// Up to 32 rows where the keys are many: the tiles' kernel splits them over four CTAs at
// most.  us, 32 rows, 128-row tiles and this: 4 heads of 20000 keys 42 and 12.6, 24 of 3000
// 10.3 and 9.1, 128 of 3000 22.8 and 22.4; of 1100 keys 7.1 and 7.0, 12.7 and 13.2; 128 of
// 700 8.2 and 11.2.
bool cross_attention_few_fits(const attn::Geometry& g) {
  const int64_t rows = static_cast<int64_t>(g.Sq) * g.group;
  return rows <= few::MMA_ROWS / 2 || (rows <= few::MMA_ROWS && g.Skv >= 2048);
}

sky_status cross_attention_few(const attn::Geometry& g, int B, void* ctx, float* lse, cudaStream_t stream) {
  using namespace few;
  const int Akv = g.A / g.group, ctas = split(static_cast<int64_t>(Akv) * B, g.Skv, 512, 5);
  const Params p{g, g.Sq * g.group, scale(g.D), ctx, lse};
  CUtensorMap tk, tv;
  SKY_CHECK(attn_tc::cross_map(&tk, g.k, Akv, g.Skv, B, g.ldk, 1, CHUNK) &&
                attn_tc::cross_map(&tv, g.v, Akv, g.Skv, B, g.ldv, 1, CHUNK),
            SKY_ERR_CUDA, "cuTensorMapEncodeTiled failed for the cross attention operands");
  const auto go = [&](auto halves) {
    auto kern = attn_few_mma<decltype(halves)::value>;
    static OncePerDevice once, wide;
    const cudaError_t e = allow_smem(once, kern, MMA_SMEM);
    return e != cudaSuccess ? e : launch(wide, kern, dim3(ctas, Akv, B), MMA_SMEM, stream, tk, tv, p);
  };
  const cudaError_t e = p.all_rows <= 8    ? go(std::integral_constant<int, 1>{})
                        : p.all_rows <= 16 ? go(std::integral_constant<int, 2>{})
                                           : go(std::integral_constant<int, 4>{});
  count_launches(1);
  return e == cudaSuccess ? SKY_OK : cuda_fail(e, "few-row cross attention launch");
}

// Against the tiled kernel, 16 rows a CTA and a head's keys in one (fp32, us): one row, 16
// heads of 128, 2 x 1659 keys 15 and 136; 64 x 8 rows, 16 heads of 64, 512 keys 78 and
// 105; 16 rows 131 and 104.  More rows where the tiles leave SMs idle: 32 rows, 4 heads,
// 2000 keys 10.6 and 104; 2 x 64 rows, 16 heads, 600 keys 23 and 33; 64 rows, 8 heads, 64
// keys 5.5 and 5.0, 200 keys 8.1 and 13.3; 32 x 12 rows, 8 heads of 128 38 and 32.
bool cross_attention_few_simt_pays(const attn::Geometry& g, int B) {
  const int64_t tiles = static_cast<int64_t>(ceil_div(g.Sq, 16)) * g.A * B;
  return g.Sq <= 8 || (tiles <= (sm_count() > 0 ? sm_count() : 148) && g.Skv > 96);
}

template <typename T>
sky_status cross_attention_few_simt(const attn::Geometry& geo, int B, T* ctx, float* lse, cudaStream_t stream) {
  attn::Geometry g = geo;
  const auto on = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % (4 * sizeof(T)) == 0; };
  g.vec = g.D % 4 == 0 && (g.ldq | g.ldk | g.ldv) % 4 == 0 && on(g.q) && on(g.k) && on(g.v);
  const cudaError_t e = few::few_simt(g, B, ctx, lse, stream);
  count_launches(1);
  return e == cudaSuccess ? SKY_OK : cuda_fail(e, "few-row cross attention launch");
}
template sky_status cross_attention_few_simt(const attn::Geometry&, int, float*, float*, cudaStream_t);
template sky_status cross_attention_few_simt(const attn::Geometry&, int, __nv_bfloat16*, float*, cudaStream_t);

}  // namespace sky
