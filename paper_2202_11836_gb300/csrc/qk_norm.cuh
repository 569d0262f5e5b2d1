// Root-mean-square norm of every query and key head with the rotation by position in
// the same pass, forward and backward.  Per head x of D values with gain g:
//   r = 1 / sqrt(mean(x^2) + eps),  xhat = r x,  z = g xhat,  y = R(pos) z,
// R turning each pair (z_a, z_b) by the angle pos * theta^(-2 i / D).  Backward, the
// turn being its own transpose's inverse:
//   dz = R(-pos) dy,  dg = sum over tokens and heads of dz xhat,
//   h = dz g,  dx = r (h - xhat mean(h xhat)).
//
// HBM-bound: forward reads and writes every head once, backward reads x and dy and
// writes dx; r is formed again, which costs no bytes.  The arithmetic, in packed pairs, is
// a third to a half of the time that the bytes take, so both have to overlap.
//
// Layout: D / 16 lanes hold a head, each 8 values of its low half and the 8 values D / 2
// behind them, two 16-byte accesses of bf16 and, whichever way pairs are formed, both
// values of every pair.  A warp takes 32 / lanes heads a pass and NP passes a token.  It
// keeps its set of heads and walks over the tokens, so gains and gain gradients stay in
// registers.  Every lane copies its own 16-byte pieces of the tokens ahead to shared
// memory with cp.async and reads them back itself: STAGES - 1 tokens a warp are on their
// way without a register held or a barrier passed.
//
// 8192 tokens x 32 heads of 64, bf16: forward 12.3 us, 67 MB at 5.5 TB/s (the copy rate
// would take 9.9); backward 21.4, of which the two gains' sums over CTAs 1.9, 101 MB at 4.7
// TB/s (14.9).  What is left is the first loads and the last stores of a launch.  With
// loads into registers, fp32 arithmetic one by one and addresses formed anew for every
// token: 15.2 and 27.9.
//
// Angles.  pos * frequency in fp32 is off by whole turns' fractions at far positions
// (2^-24 of 10^6 radians is 0.06).  So the host gives each frequency as a fraction of a
// turn in 64-bit fixed point, and pos * F modulo 2^64 is the turned fraction exactly, up
// to |pos| 2^-65 of a turn and what the doubles on the host lost, a few 2^-53 of the
// frequency: 2^-50 |pos| radians in all.  Its top 32 bits, as a
// signed fraction, go to sincospif.  Lane i computes angles i, i + 32, ... of the token
// once for all heads of the warp, and they are shared through shared memory.
#pragma once
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "common.cuh"
#include "ptx.cuh"
#include "rowwise.h"

namespace sky {
namespace qkn {

constexpr int WARPS = 8, THR = WARPS * 32, STAGES = 3;
constexpr int MAX_D = 256, MAX_ANGLES = MAX_D / 2;
enum Rotation { NONE = 0, HALVES = 1, PAIRS = 2 };

struct Params {
  const void* x;    // rows of ldx values, q_heads + k_heads heads of D at the front
  const void* dy;   // backward: rows of ldy
  void* out;        // forward: y, rows of ldy; backward: dx, rows of ldx
  const void* gain[2];  // of queries and keys, or null: ones
  const int32_t* pos;
  float* part;      // backward: [2][gridDim.x][D] partial gain gradients, or
  float* dgain[2];  // in one cluster the gradients themselves (or null)
  int64_t ldx, ldy;
  int rows, D, heads[2];
  int chunks[2];    // sets of heads of a warp
  float eps;
  uint64_t turn[MAX_ANGLES];  // frequency i in 2^-64 turns
};

// Eight values as four pairs, from the 16-byte pieces they are copied in and to memory.
using Pairs = uint64_t[4];
template <typename T>
constexpr int kPieces = sizeof(T) / 2;  // of eight values
__device__ __forceinline__ void pairs_of(const uint32_t (&w)[4], Pairs& v) {  // bf16
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
__device__ __forceinline__ void read8(const __nv_bfloat16*, uint32_t slot, Pairs& v) {
  uint32_t w[4];
  ptx::ld_shared_v4(slot, w);
  pairs_of(w, v);
}
__device__ __forceinline__ void read8(const float*, uint32_t slot, Pairs& v) {
  const float4 a = ptx::ld_shared_f4(slot), b = ptx::ld_shared_f4(slot + 512);
  v[0] = pack2(a.x, a.y); v[1] = pack2(a.z, a.w); v[2] = pack2(b.x, b.y); v[3] = pack2(b.z, b.w);
}
__device__ __forceinline__ void write8(__nv_bfloat16* p, const Pairs& v) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 x = unpack2(v[i]);
    w[i] = ptx::pack_bf16(x.x, x.y);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void write8(float* p, const Pairs& v) {
  const float2 a = unpack2(v[0]), b = unpack2(v[1]), c = unpack2(v[2]), d = unpack2(v[3]);
  reinterpret_cast<float4*>(p)[0] = make_float4(a.x, a.y, b.x, b.y);
  reinterpret_cast<float4*>(p)[1] = make_float4(c.x, c.y, d.x, d.y);
}
__device__ __forceinline__ uint64_t both(float v) { return pack2(v, v); }
__device__ __forceinline__ float sum2(uint64_t a, uint64_t b) {
  const float2 x = unpack2(add2(a, b));
  return x.x + x.y;
}

template <int LP>
__device__ __forceinline__ float head_sum(float v) {  // over the LP lanes of a head
#pragma unroll
  for (int o = LP / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// What a warp works on: the lane's place in its heads and the warp's in the grid.  DIM: the
// head dim where its lanes fill it, 16 LP, else 0 (known at run time).
template <typename T, int LP, int NP, int DIM>
struct Place {
  int kind, head0;        // queries or keys; the lane's head of pass 0 (pass p: + p HPW)
  int heads;              // of the kind
  int token0, step, n;    // the warp's tokens: token0, token0 + step, ..., n of them
  int D, lo;              // head dim; offset of the lane's low values in a head, the high ones D / 2 behind
  bool lane_live;         // (LP lanes are a power of two, D / 16 of them hold values)
  static constexpr int HPW = 32 / LP;
  __device__ explicit Place(const Params& p) {
    const int lane = threadIdx.x & 31, sets = p.chunks[0] + p.chunks[1];
    const int w = blockIdx.x * WARPS + (threadIdx.x >> 5), warps = gridDim.x * WARPS / sets * sets;
    int c = w % sets;
    kind = c >= p.chunks[0];
    if (kind) c -= p.chunks[0];
    heads = p.heads[kind];
    head0 = c * HPW * NP + lane / LP;
    token0 = w / sets;
    step = warps / sets;
    n = w < warps && token0 < p.rows ? (p.rows - 1 - token0) / step + 1 : 0;
    D = DIM ? DIM : p.D;
    lane_live = DIM || lane % LP < D / 16;
    lo = lane % LP * 8;
  }
  // whether any lane has a head in the pass (the same for the whole warp)
  __device__ bool any(int pass) const { return head0 - static_cast<int>(threadIdx.x & 31) / LP + pass * HPW < heads; }
  __device__ bool live(int pass) const { return lane_live && head0 + pass * HPW < heads; }
  // The lane's low values of pass 0 in token0's row, and what a step, a pass and the high
  // values are away, in values
  __device__ int64_t first(const Params& p, int64_t ld) const {
    return token0 * ld + (static_cast<int64_t>(kind ? p.heads[0] : 0) + head0) * D + lo;
  }
  __device__ int pass_at(int pass) const { return pass * HPW * D; }
  __device__ void gains(const Params& p, Pairs& glo, Pairs& ghi) const {
    const T* g = static_cast<const T*>(p.gain[kind]);
    const auto at = [&](int d) { return !lane_live ? 0.f : g ? to_f32(g[d]) : 1.f; };
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      glo[i] = pack2(at(lo + 2 * i), at(lo + 2 * i + 1));
      ghi[i] = pack2(at(D / 2 + lo + 2 * i), at(D / 2 + lo + 2 * i + 1));
    }
  }
};

// The warp's ring: its tokens' pieces of one or two tensors, each lane's own.  Lanes
// without a head copy nothing and read the zeros that they start with.
template <typename T, int LP, int NP, int DIM, int TENSORS, int STAGES>
struct Ring {
  static constexpr int PIECES = kPieces<T>, SLOTS = TENSORS * NP * 2 * PIECES, BYTES = STAGES * SLOTS * 512;
  const Place<T, LP, NP, DIM>& at;
  uint32_t base, put, got;  // the lane's slots; stages to copy to and to read, as offsets
  int ahead;                // tokens sent for
  const T* src[TENSORS];
  int64_t stride[TENSORS];
  __device__ Ring(const Params& p, const Place<T, LP, NP, DIM>& place, uint8_t* shared)
      : at(place), base(ptx::smem_u32(shared) + (threadIdx.x >> 5) * BYTES + (threadIdx.x & 31) * 16), put(0), got(0), ahead(0) {
    src[0] = static_cast<const T*>(p.x) + at.first(p, p.ldx);
    stride[0] = at.step * p.ldx;
    if (TENSORS > 1) {
      src[TENSORS - 1] = static_cast<const T*>(p.dy) + at.first(p, p.ldy);
      stride[TENSORS - 1] = at.step * p.ldy;
    }
#pragma unroll
    for (int i = 0; i < NP; ++i)
      if (!at.live(i))
        for (int st = 0; st < STAGES; ++st)
          for (int k = 0; k < TENSORS; ++k)
            for (int c = 0; c < 2 * PIECES; ++c) ptx::st_shared_v4(base + st * SLOTS * 512 + slot(k, i, c), 0, 0, 0, 0);
  }
  static __device__ constexpr uint32_t slot(int tensor, int pass, int piece) {
    return ((tensor * NP + pass) * 2 * PIECES + piece) * 512;
  }
  static __device__ uint32_t next(uint32_t stage) { return stage == (STAGES - 1) * SLOTS * 512 ? 0 : stage + SLOTS * 512; }
  __device__ void fetch() {  // the warp's next token, if there is one
    if (ahead < at.n) {
#pragma unroll
      for (int k = 0; k < TENSORS; ++k) {
#pragma unroll
        for (int i = 0; i < NP; ++i)
          if (at.live(i)) {
#pragma unroll
            for (int c = 0; c < 2 * PIECES; ++c) {
              const T* x = src[k] + at.pass_at(i) + (c < PIECES ? 0 : at.D / 2) + c % PIECES * (16 / static_cast<int>(sizeof(T)));
              asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(base + put + slot(k, i, c)), "l"(x) : "memory");
            }
          }
        src[k] += stride[k];
      }
      ++ahead;
      put = next(put);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  __device__ void start() {
#pragma unroll
    for (int n = 0; n < STAGES - 1; ++n) fetch();
  }
  // sends for one token more (to the stage that was read last) and waits for the oldest
  __device__ void wait() {
    fetch();
    asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
  }
  __device__ void read(int tensor, int pass, Pairs& lo, Pairs& hi) const {
    read8(static_cast<const T*>(nullptr), base + got + slot(tensor, pass, 0), lo);
    read8(static_cast<const T*>(nullptr), base + got + slot(tensor, pass, PIECES), hi);
  }
  __device__ void done() { got = next(got); }
};

// Cosines and sines of a token's angles, and the lane's turning of its pairs by them.
// HALVES: pair i of (lo[i], hi[i]); PAIRS: pairs i < 4 of (lo[2 i], lo[2 i + 1]), then of
// hi.
template <int ROT, int LP>
struct Angles {
  static constexpr int N = (LP * 8 + 31) / 32;  // angles a lane computes
  static constexpr int TAB = ROT == NONE ? 1 : 2 * LP * 8;  // floats of a warp: cosines, sines
  uint64_t turn[N];
  int pos;     // of the warp's tokens 32 by 32, one a lane
  float* tab;  // the warp's
  uint64_t c[ROT == PAIRS ? 8 : 4], s[ROT == PAIRS ? 8 : 4];  // HALVES: two pairs each; PAIRS: (cos, cos), (-sin, sin)
  __device__ Angles(const Params& p, float* shared) {
    if (ROT == NONE) return;
    const int lane = threadIdx.x & 31;
    tab = shared + (threadIdx.x >> 5) * TAB;
#pragma unroll
    for (int i = 0; i < N; ++i) turn[i] = lane + 32 * i < p.D / 2 ? p.turn[lane + 32 * i] : 0;
  }
  // of the warp's token n; sign -1 turns back
  __device__ void get(const Params& p, int token0, int step, int n, float sign) {
    if (ROT == NONE) return;
    const int lane = threadIdx.x & 31;
    if (n % 32 == 0) {
      const int64_t t = token0 + static_cast<int64_t>(n + lane) * step;
      pos = t < p.rows ? p.pos[t] : 0;
    }
    const int64_t at = __shfl_sync(0xffffffffu, pos, n % 32);
    __syncwarp();  // the token before has been read
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint64_t f = turn[i] * static_cast<uint64_t>(at);
      float sn, cs;
      sincospif(static_cast<float>(static_cast<int32_t>(f >> 32)) * 0x1p-31f, &sn, &cs);
      if (N * 32 == LP * 8 || lane + 32 * i < LP * 8) {
        tab[lane + 32 * i] = cs;
        tab[LP * 8 + lane + 32 * i] = sn * sign;
      }
    }
    __syncwarp();
    const int l = lane % LP;
    if (ROT == HALVES) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float4 x = *reinterpret_cast<const float4*>(tab + l * 8 + 4 * k);
        const float4 y = *reinterpret_cast<const float4*>(tab + LP * 8 + l * 8 + 4 * k);
        c[2 * k] = pack2(x.x, x.y); c[2 * k + 1] = pack2(x.z, x.w);
        s[2 * k] = pack2(y.x, y.y); s[2 * k + 1] = pack2(y.z, y.w);
      }
    } else {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        // (idle lanes of a head read inside the table)
        const int a = (k ? p.D / 4 : 0) + l * 4, q = a < LP * 8 ? a : 0;
        const float4 x = *reinterpret_cast<const float4*>(tab + q), y = *reinterpret_cast<const float4*>(tab + LP * 8 + q);
        const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          c[(4 * k + i) % (ROT == PAIRS ? 8 : 4)] = both(xs[i]);
          s[(4 * k + i) % (ROT == PAIRS ? 8 : 4)] = pack2(-ys[i], ys[i]);
        }
      }
    }
  }
  __device__ void apply(Pairs& lo, Pairs& hi) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (ROT == HALVES) {
        const uint64_t a = lo[i], b = hi[i];
        lo[i] = fma2(mul2(b, both(-1.f)), s[i], mul2(a, c[i]));
        hi[i] = fma2(a, s[i], mul2(b, c[i]));
      }
      if (ROT == PAIRS) {
        const float2 a = unpack2(lo[i]), b = unpack2(hi[i]);
        lo[i] = fma2(pack2(a.y, a.x), s[i], mul2(lo[i], c[i]));
        hi[i] = fma2(pack2(b.y, b.x), s[(4 + i) % (ROT == PAIRS ? 8 : 4)], mul2(hi[i], c[(4 + i) % (ROT == PAIRS ? 8 : 4)]));
      }
    }
  }
};

template <typename T, int LP, int ROT, int NP, int DIM>
__global__ void __launch_bounds__(THR) qk_norm_fwd(const __grid_constant__ Params p) {
  extern __shared__ __align__(16) uint8_t ring_mem[];
  __shared__ __align__(16) float tab[WARPS * Angles<ROT, LP>::TAB];
  const Place<T, LP, NP, DIM> at(p);
  Angles<ROT, LP> ang(p, tab);
  const float inv = 1.f / static_cast<float>(at.D);
  Ring<T, LP, NP, DIM, 1, STAGES> ring(p, at, ring_mem);
  T* y = static_cast<T*>(p.out) + at.first(p, p.ldy);
  const int64_t to_next = at.step * p.ldy;
  pdl_wait();
  pdl_trigger();
  ring.start();
  Pairs glo, ghi;
  at.gains(p, glo, ghi);
  for (int n = 0; n < at.n; ++n) {
    ang.get(p, at.token0, at.step, n, 1.f);
    ring.wait();
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if (!at.any(i)) continue;
      Pairs lo, hi;
      ring.read(0, i, lo, hi);
      uint64_t a = 0, b = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        a = fma2(lo[e], lo[e], a);
        b = fma2(hi[e], hi[e], b);
      }
      const uint64_t r = both(rsqrtf(head_sum<LP>(sum2(a, b)) * inv + p.eps));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        lo[e] = mul2(mul2(lo[e], r), glo[e]);
        hi[e] = mul2(mul2(hi[e], r), ghi[e]);
      }
      ang.apply(lo, hi);
      if (at.live(i)) {
        write8(y + at.pass_at(i), lo);
        write8(y + at.pass_at(i) + at.D / 2, hi);
      }
    }
    ring.done();
    y += to_next;
  }
}

// ONE: the grid is one cluster, which adds up the gain gradients itself.
template <typename T, int LP, int ROT, int NP, int DIM, bool ONE>
__global__ void __launch_bounds__(THR) qk_norm_bwd(const __grid_constant__ Params p) {
  extern __shared__ __align__(16) uint8_t ring_mem[];
  __shared__ __align__(16) float tab[WARPS * Angles<ROT, LP>::TAB];
  __shared__ float red[WARPS][LP * 16];
  __shared__ __align__(8) float sums[ONE ? 2 : 1][ONE ? LP * 16 : 1];
  __shared__ int kind_of[WARPS];
  const Place<T, LP, NP, DIM> at(p);
  Angles<ROT, LP> ang(p, tab);
  const float inv = 1.f / static_cast<float>(at.D);
  Ring<T, LP, NP, DIM, 2, STAGES> ring(p, at, ring_mem);
  T* dx = static_cast<T*>(p.out) + at.first(p, p.ldx);
  const int64_t to_next = at.step * p.ldx;
  pdl_wait();
  pdl_trigger();
  ring.start();
  Pairs glo, ghi, alo = {}, ahi = {};
  at.gains(p, glo, ghi);
  for (int n = 0; n < at.n; ++n) {
    ang.get(p, at.token0, at.step, n, -1.f);
    ring.wait();
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if (!at.any(i)) continue;
      Pairs lo, hi, zl, zh;
      ring.read(0, i, lo, hi);
      ring.read(1, i, zl, zh);
      ang.apply(zl, zh);
      uint64_t a = 0, b = 0, c = 0, d = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        a = fma2(lo[e], lo[e], a);
        b = fma2(hi[e], hi[e], b);
        c = fma2(mul2(zl[e], glo[e]), lo[e], c);
        d = fma2(mul2(zh[e], ghi[e]), hi[e], d);
      }
      const float ss = head_sum<LP>(sum2(a, b)), sh = head_sum<LP>(sum2(c, d));
      // (lanes without a head: zeros, whose norm without an eps would be NaN in the gains' sums)
      const float rs = rsqrtf(ss * inv + (at.live(i) ? p.eps : 1.f));
      const uint64_t r = both(rs), m = both(-(sh * rs * inv));  // - mean of h xhat
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        lo[e] = mul2(lo[e], r);
        hi[e] = mul2(hi[e], r);
        alo[e] = fma2(zl[e], lo[e], alo[e]);
        ahi[e] = fma2(zh[e], hi[e], ahi[e]);
        lo[e] = mul2(r, fma2(lo[e], m, mul2(zl[e], glo[e])));
        hi[e] = mul2(r, fma2(hi[e], m, mul2(zh[e], ghi[e])));
      }
      if (at.live(i)) {
        write8(dx + at.pass_at(i), lo);
        write8(dx + at.pass_at(i) + at.D / 2, hi);
      }
    }
    ring.done();
    dx += to_next;
  }
  // gain gradients: the warp's heads, then the CTA's warps in order, into one row of
  // partial sums for each kind
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float2 u = unpack2(alo[e]), v = unpack2(ahi[e]);
#pragma unroll
    for (int o = LP; o < 32; o <<= 1) {
      u.x += __shfl_xor_sync(0xffffffffu, u.x, o);
      u.y += __shfl_xor_sync(0xffffffffu, u.y, o);
      v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
      v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
    }
    if (lane < LP && at.lane_live) {
      *reinterpret_cast<float2*>(&red[w][at.lo + 2 * e]) = u;
      *reinterpret_cast<float2*>(&red[w][at.D / 2 + at.lo + 2 * e]) = v;
    }
  }
  if (lane == 0) kind_of[w] = at.kind;
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * p.D; i += THR) {
    const int kind = i >= p.D, d = i - kind * p.D;
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < WARPS; ++v)
      if (kind_of[v] == kind) s += red[v][d];
    if (ONE) sums[kind][d] = s;
    else p.part[(static_cast<int64_t>(kind) * gridDim.x + blockIdx.x) * p.D + d] = s;
  }
  if constexpr (ONE) {  // in the order of the CTAs
    ptx::cluster_sync();
    for (int i = threadIdx.x; blockIdx.x == 0 && i < p.D; i += THR) {  // pairs
      const int kind = i >= p.D / 2, d = 2 * (i - kind * (p.D / 2));
      const uint32_t at = ptx::smem_u32(&sums[kind][d]);
      float2 s = make_float2(0.f, 0.f);
      for (int c = 0; c < static_cast<int>(gridDim.x); ++c) {
        const float2 x = ptx::ld_cluster_f2(ptx::mapa_shared(at, c));
        s.x += x.x;
        s.y += x.y;
      }
      if (p.dgain[kind]) {
        p.dgain[kind][d] = s.x;
        p.dgain[kind][d + 1] = s.y;
      }
    }
    ptx::cluster_sync();  // the first CTA has read the sums
  }
}

// ------------------------------------------------------------------- host
// Calls f with the lanes of a head (a power of two), the rotation, the passes of a warp and
// the head dim, where the lanes of the usual ones fill it, as constants.  Two passes where
// both kinds then come out in whole warps' sets.
template <typename F>
auto pick(const sky_qk_norm_shape& s, F&& f) {
  using std::integral_constant;
  const auto turn = [&](auto lp, auto np, auto dim) {
    return s.rotation == SKY_ROTATE_HALVES  ? f(lp, integral_constant<int, HALVES>{}, np, dim)
           : s.rotation == SKY_ROTATE_PAIRS ? f(lp, integral_constant<int, PAIRS>{}, np, dim)
                                            : f(lp, integral_constant<int, NONE>{}, np, dim);
  };
  const auto passes = [&](auto lp, auto dim) {
    constexpr int SET = 2 * 32 / decltype(lp)::value;
    return s.q_heads % SET || s.k_heads % SET ? turn(lp, integral_constant<int, 1>{}, dim)
                                              : turn(lp, integral_constant<int, 2>{}, dim);
  };
  const auto any = [&](auto lp) { return turn(lp, integral_constant<int, 1>{}, integral_constant<int, 0>{}); };
  const auto full = [&](auto lp) {
    constexpr int D = 16 * decltype(lp)::value;
    return s.head_dim == D ? passes(lp, integral_constant<int, D>{}) : any(lp);
  };
  const int lanes = s.head_dim / 16;
  return lanes <= 1   ? any(integral_constant<int, 1>{})
         : lanes <= 2 ? full(integral_constant<int, 2>{})
         : lanes <= 4 ? full(integral_constant<int, 4>{})
         : lanes <= 8 ? full(integral_constant<int, 8>{})
                      : any(integral_constant<int, 16>{});
}

// CTAs an SM.  8192 tokens of 32 heads of 64, us: forward 12.3 with three, 14.7 with two
// (and four stages); backward 22 with one, 26 with two of 128 registers, whose main loop
// is as fast (19.6 and 19.8) but leaves twice the partial rows to add.  (Three is what that
// forward's 78 registers let fit.  Forms of more, such as pairs and head dims from 80 on, and
// fp32 in two passes, whose rings take 96 KiB, fit two, and run the plan in two rounds.)
inline int max_ctas(bool bwd) {
  const int sms = sm_count() > 0 ? sm_count() : 148;
  return sms * (bwd ? 1 : 3);
}

// Sets of heads for warps of `hpw` heads a pass and `np` passes, and the CTAs: as many as
// give every warp its last token in the same round, up to `most`.
inline int plan(const sky_qk_norm_shape& s, int hpw, int np, int most, Params* p) {
  p->chunks[0] = ceil_div(s.q_heads, hpw * np);
  p->chunks[1] = ceil_div(s.k_heads, hpw * np);
  const int sets = p->chunks[0] + p->chunks[1];
  const int widest = std::max(1, most * WARPS / sets);                 // tokens at a time
  const int rounds = ceil_div(s.rows, widest), step = ceil_div(s.rows, rounds);
  return ceil_div(static_cast<int64_t>(step) * sets, WARPS);
}

template <typename T>
sky_status forward(const sky_qk_norm_shape& s, Params& p, cudaStream_t st) {
  return pick(s, [&](auto lp, auto rot, auto np, auto dim) {
    constexpr int LP = decltype(lp)::value, ROT = decltype(rot)::value, NP = decltype(np)::value, DIM = decltype(dim)::value;
    const int ctas = plan(s, 32 / LP, NP, max_ctas(false), &p);
    auto kern = qk_norm_fwd<T, LP, ROT, NP, DIM>;
    constexpr int SMEM = WARPS * Ring<T, LP, NP, DIM, 1, STAGES>::BYTES;
    static OncePerDevice once;
    cudaError_t e = allow_smem(once, kern, SMEM);
    if (e == cudaSuccess) e = launch_pdl(kern, dim3(ctas), dim3(THR), SMEM, st, 1, p);
    count_launches(1);
    return e == cudaSuccess ? SKY_OK : cuda_fail(e, "head norm forward launch");
  });
}

template <typename T>
sky_status backward(const sky_qk_norm_shape& s, Params& p, float* dq_gain, float* dk_gain, cudaStream_t st) {
  int ctas = 0;
  bool one = false;
  const sky_status done = pick(s, [&](auto lp, auto rot, auto np, auto dim) {
    constexpr int LP = decltype(lp)::value, ROT = decltype(rot)::value, NP = decltype(np)::value, DIM = decltype(dim)::value;
    // Few tokens: one cluster of up to eight CTAs, four tokens a warp at most, in place of
    // a second launch (64 tokens of 16 heads, from the host: 17.5 -> 15.4 us)
    ctas = plan(s, 32 / LP, 1, max_ctas(true), &p);
    const int64_t work = static_cast<int64_t>(s.rows) * (p.chunks[0] + p.chunks[1]);
    one = work <= 4 * 8 * WARPS && p.chunks[0] + p.chunks[1] <= 8 * WARPS;
    if (one) ctas = std::min(8, ceil_div(work, WARPS));
    else ctas = plan(s, 32 / LP, NP, max_ctas(true), &p);
    const auto go = [&](auto kern, int cluster) {
      constexpr int SMEM = WARPS * Ring<T, LP, NP, DIM, 2, STAGES>::BYTES;  // (enough for one pass too)
      static OncePerDevice once[2];
      const cudaError_t e = allow_smem(once[cluster > 0], kern, SMEM);
      return e != cudaSuccess ? e : launch_pdl(kern, dim3(ctas), dim3(THR), SMEM, st, std::max(1, cluster), p);
    };
    p.dgain[0] = dq_gain;
    p.dgain[1] = dk_gain;
    const cudaError_t e = one ? go(qk_norm_bwd<T, LP, ROT, 1, DIM, true>, ctas) : go(qk_norm_bwd<T, LP, ROT, NP, DIM, false>, 0);
    count_launches(1);
    return e == cudaSuccess ? SKY_OK : cuda_fail(e, "head norm backward launch");
  });
  if (done != SKY_OK || one) return done;
  ColSegments segs = {};
  if (dq_gain) segs.seg[segs.n++] = {p.part, dq_gain, ctas, s.head_dim};
  if (dk_gain) segs.seg[segs.n++] = {p.part + static_cast<int64_t>(ctas) * s.head_dim, dk_gain, ctas, s.head_dim};
  return reduce_column_segments(segs, st);
}

}  // namespace qkn
}  // namespace sky
