// One AdamW step over many tensors, moments in 32 bits or in 8 (sky_optim.h).
//
// A stream bound by HBM: a value with fp32 moments, fp32 gradients and a bf16 copy moves 30
// bytes, with moments in 8 bits 18.  A warp takes 256 consecutive values of one tensor, the
// block that shares a scale in 8 bits: a lane holds values 4 lane .. and 128 + 4 lane .., so
// every access of a warp is contiguous, and the block's largest values are two warp
// reductions.  Those go over the bits of |x| as integers, which are ordered as the numbers
// are and put NaN above all: a moment that is not finite stays visible.
//
// The tensors' table travels in the kernel's parameters: nothing to allocate or to copy, and
// a captured call keeps its own.  A CTA's chunks of 2048 values come in ascending order, so
// its tensor is found by walking on from the one before.  Blocks that are whole and aligned take
// one access a lane for four values, and with moments in 8 bits, whose arithmetic takes nearly
// as long as the bytes, the blocks ahead are on their way into shared memory meanwhile (cp.async;
// a warp's own, so nothing waits for another); others go value by value.
//
// Products and sums of the moments are rounded one by one (no fused multiply-add): what a
// byte holds then does not depend on which of them a compiler contracts.  The root of v goes by the
// hardware's approximation (2^-23 of it) in the update.  For r's byte it has to be the rounded root:
// where the approximation leaves open which of two codes is nearer (eight steps of its last place
// or less from the border between them), or a value is below the least code, the warp takes exact
// roots for its block, and ties and small values in full.
//
// us for 67M values with moments in 8 bits and fp32 gradients, where HBM takes 179 at copy rate:
// exact roots and quotients for every value and a choice of access at each load (91 instructions a
// value) 221, now (66) 215; without any arithmetic 211, so what is left is HBM with eleven streams:
// three or four CTAs an SM in the place of two take 229 to 303, runs of four blocks a warp 247.  With
// bf16 gradients 33.6M values take 96 of 80.  Moments in 32 bits: 33.6M values 158 of 148.
#include <cuda_fp8.h>

#include <cfloat>
#include <cmath>

#include "../../include/sky_optim.h"
#include "abi.h"
#include "common.cuh"
#include "ptx.cuh"

namespace sky {
namespace adamw {
namespace {

constexpr int THREADS = 256, CHUNK = SKY_STATE_BLOCK * (THREADS / 32);
constexpr float TINY = 1e-30f;  // the largest value of a block that counts as zeros
constexpr int FEW = 32, MANY = 400;  // tensors of a launch: its parameters are 2.4 or 29 KiB

struct Tensor {
  float* w;
  const void* g;
  void* m;
  void* v;
  float* ms;
  float* vs;
  __nv_bfloat16* p;
  int64_t n;
  int32_t decay, vec;  // vec: every pointer allows a lane's four values in one access
};

template <int N>
struct Args {
  float lr, b1, b2, eps, wd, c1, c2;
  int tensors;
  int64_t chunks;
  const sky_adamw_now* now;
  int32_t first[N + 1];  // first chunk of every tensor
  Tensor t[N];
};

__device__ __forceinline__ void load4(const float* x, float (&v)[4]) {
  const float4 f = __ldcs(reinterpret_cast<const float4*>(x));
  v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
}
__device__ __forceinline__ void store4(float* x, const float (&v)[4]) {
  *reinterpret_cast<float4*>(x) = make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store4(__nv_bfloat16* x, const float (&v)[4]) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
  *reinterpret_cast<uint2*>(x) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

// Gradients as they lie: four values in 16 or 8 bytes.
template <typename G> struct Raw;
template <> struct Raw<float> { using type = float4; };
template <> struct Raw<__nv_bfloat16> { using type = uint2; };
__device__ __forceinline__ void gradients(const float4& u, float (&g)[4]) {
  g[0] = u.x; g[1] = u.y; g[2] = u.z; g[3] = u.w;
}
__device__ __forceinline__ void gradients(const uint2& u, float (&g)[4]) {
  g[0] = __uint_as_float(u.x << 16);
  g[1] = __uint_as_float(u.x & 0xffff0000u);
  g[2] = __uint_as_float(u.y << 16);
  g[3] = __uint_as_float(u.y & 0xffff0000u);
}

// e4m3 bytes, two by two.
__device__ __forceinline__ void m_values(uint32_t codes, float scale, float (&m)[4]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const __half2_raw raw =
        __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>((codes >> (16 * h)) & 0xffffu), __NV_E4M3);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&raw));
    m[2 * h] = __fmul_rn(f.x, scale);
    m[2 * h + 1] = __fmul_rn(f.y, scale);
  }
}
__device__ __forceinline__ uint32_t m_codes(const float (&m)[4], float inv) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(__fmul_rn(m[0], inv), __fmul_rn(m[1], inv)), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(__fmul_rn(m[2], inv), __fmul_rn(m[3], inv)), __NV_SATFINITE, __NV_E4M3);
  return lo | hi << 16;
}
// A byte of r holds the low four bits of the exponent (2^-16 .. 2^-1, which fp32 holds as
// 111 .. 126) above the first four of the fraction: the fp32 number's own bits, shifted.
constexpr uint32_t LEAST = 111u << 23;  // what code 0 would be
__device__ __forceinline__ float r_value(uint32_t c) { return c ? __uint_as_float((c << 19) + LEAST) : 0.f; }
// To nearest, ties to even, and no code 0 for what is not 0.  (Above 255: NaN only.)
__device__ __forceinline__ uint32_t r_code(float y) {
  const uint32_t b = __float_as_uint(y);
  const int c = static_cast<int>(b + 0x3ffffu + ((b >> 19) & 1u) - LEAST) >> 19;
  return static_cast<uint32_t>(min(max(c, y == 0.f ? 0 : 1), 255));
}
// The same where `nearest` and `least` allow it: y's bits from half a code below, 8 more to see on
// which side of a border it is near; the code is what is above the low 19 of them.
__device__ __forceinline__ int r_bits(float y) { return static_cast<int>(__float_as_uint(y) + 0x40008u - LEAST); }

__device__ __forceinline__ float root(float x) {  // (2^-23 of it; 0 for subnormals)
  float y;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float inverse(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The scale of a block whose largest |x| has these bits, and its inverse.
__device__ __forceinline__ void block_scale(uint32_t top_bits, float unit, float& scale, float& inv) {
  const float top = __uint_as_float(top_bits);
  const bool zero = top < TINY;
  scale = zero ? 0.f : __fmul_rn(top, unit);
  inv = zero ? 0.f : __frcp_rn(scale);
}

// The settings of a step, as the values need them.
struct Rule {
  float b1, b2, d1, d2, eps, gs, root2, rate, lr_wd;
};

template <int N>
__device__ __forceinline__ Rule rule_of(const Args<N>& a) {
  float lr = a.lr, c1 = a.c1, c2 = a.c2, gs = 1.f;
  if (a.now) {
    lr = a.now->lr;
    c1 = a.now->correction1;
    c2 = a.now->correction2;
    gs = a.now->grad_scale;
  }
  return {a.b1, a.b2, __fsub_rn(1.f, a.b1), __fsub_rn(1.f, a.b2), a.eps, gs, __fsqrt_rn(__frcp_rn(c2)),
          __fdiv_rn(lr, c1), __fmul_rn(lr, a.wd)};
}

// A lane's values of a block: 4 lane .. and 128 + 4 lane ...
template <bool SMALL>
struct Values {
  float w[2][4], m[2][4], v[2][4];
  uint32_t mc[2], rc[2];  // SMALL: bytes, before and after
  float ms, vs;           // scales, before and after
};

// The step of a block's values, by a whole warp; g: raw gradients.
template <bool SMALL, typename R>
__device__ __forceinline__ void step(const Rule& a, const R (&g)[2], float wd, Values<SMALL>& x) {
  float r[2][4], m_top = 0.f;
  uint32_t v_top = 0;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float gg[4];
    gradients(g[h], gg);
    if constexpr (SMALL) {
      m_values(x.mc[h], x.ms, x.m[h]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float y = __fmul_rn(r_value((x.rc[h] >> (8 * e)) & 255u), x.vs);
        x.v[h][e] = __fmul_rn(y, y);
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float y = __fmul_rn(gg[e], a.gs);
      float &m = x.m[h][e], &v = x.v[h][e];
      m = __fadd_rn(__fmul_rn(m, a.b1), __fmul_rn(y, a.d1));
      v = __fadd_rn(__fmul_rn(v, a.b2), __fmul_rn(__fmul_rn(y, y), a.d2));
      r[h][e] = root(v);
      m_top = fmaxf(m_top, fabsf(m));
      v_top = max(v_top, __float_as_uint(v));  // (never negative; NaN is above all)
    }
  }
  if constexpr (SMALL) {
    float m_inv, r_inv;
    v_top = __reduce_max_sync(0xffffffffu, v_top);
    // (m is finite where v is)
    const uint32_t mt = __reduce_max_sync(0xffffffffu, __float_as_uint(m_top));
    block_scale(v_top >= 0x7f800000u ? v_top : mt, 1.f / 448.f, x.ms, m_inv);
    block_scale(__float_as_uint(__fsqrt_rn(__uint_as_float(v_top))), 1.f / 0.96875f, x.vs, r_inv);
    uint32_t nearest = 0x7ffffu;
    int least = 0x7fffffff;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      int c[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        c[e] = r_bits(__fmul_rn(r[h][e], r_inv));
        nearest = min(nearest, static_cast<uint32_t>(c[e]) & 0x7ffffu);
        least = min(least, c[e]);
        c[e] >>= 19;
      }
      x.mc[h] = m_codes(x.m[h], m_inv);
      x.rc[h] = __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
    }
    if (__any_sync(0xffffffffu, nearest < 16 || least < (1 << 19))) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        x.rc[h] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          r[h][e] = __fsqrt_rn(x.v[h][e]);
          x.rc[h] |= r_code(__fmul_rn(r[h][e], r_inv)) << (8 * e);
        }
      }
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float& w = x.w[h][e];
      // (a subnormal v's root: 8-bit blocks have it from above)
      const float rr = SMALL || x.v[h][e] >= 1.17549435e-38f ? r[h][e] : __fsqrt_rn(x.v[h][e]);
      w = fmaf(-wd, w, w);
      w = fmaf(-a.rate * x.m[h][e], inverse(fmaf(rr, a.root2, a.eps)), w);
    }
}

// Where a block lies.
struct Place {
  int at;      // tensor
  int64_t i0;  // first value; -1: there is none
  bool whole;  // four values a lane in one access
};
template <int N>
__device__ __forceinline__ Place place_of(const Args<N>& a, int64_t c, int& at, int warp) {
  if (c >= a.chunks) return {0, -1, false};
  while (c >= a.first[at + 1]) ++at;
  const int64_t i0 = ((c - a.first[at]) * (THREADS / 32) + warp) * SKY_STATE_BLOCK, n = a.t[at].n;
  return {at, i0 < n ? i0 : -1, a.t[at].vec && i0 + SKY_STATE_BLOCK <= n};
}

template <typename G>
__device__ __forceinline__ void load_whole(const Tensor& t, int64_t i, typename Raw<G>::type (&g)[2], Values<false>& x) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    g[h] = __ldcs(reinterpret_cast<const typename Raw<G>::type*>(static_cast<const G*>(t.g) + i + 128 * h));
    load4(t.w + i + 128 * h, x.w[h]);
    load4(static_cast<const float*>(t.m) + i + 128 * h, x.m[h]);
    load4(static_cast<const float*>(t.v) + i + 128 * h, x.v[h]);
  }
}

// A block on its way: gradients, weights, the bytes of m and r, the scales.
template <typename G>
struct Ahead {
  static constexpr int STAGES = 3, W = SKY_STATE_BLOCK * sizeof(G), CODES = W + 4 * SKY_STATE_BLOCK;
  static constexpr int SCALES = CODES + 2 * SKY_STATE_BLOCK, BYTES = SCALES + 16;
  static constexpr int SMEM = STAGES * BYTES * (THREADS / 32);
};
__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
template <typename G>
__device__ __forceinline__ void send(const Tensor& t, int64_t i0, uint32_t to, int lane) {
  const char* g = static_cast<const char*>(t.g) + i0 * static_cast<int>(sizeof(G)) + 16 * lane;
  const char* w = reinterpret_cast<const char*>(t.w + i0) + 16 * lane;
#pragma unroll
  for (int k = 0; k < static_cast<int>(sizeof(G)) / 2; ++k) copy16(to + 512 * k + 16 * lane, g + 512 * k);
#pragma unroll
  for (int k = 0; k < 2; ++k) copy16(to + Ahead<G>::W + 512 * k + 16 * lane, w + 512 * k);
  const uint8_t* code = static_cast<const uint8_t*>(lane < 16 ? t.m : t.v) + i0 + 16 * (lane & 15);
  copy16(to + Ahead<G>::CODES + 16 * lane, code);
  if (lane < 2)
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to + Ahead<G>::SCALES + 4 * lane),
                 "l"((lane ? t.vs : t.ms) + i0 / SKY_STATE_BLOCK)
                 : "memory");
}
template <typename G>
__device__ __forceinline__ void receive(uint32_t from, int lane, typename Raw<G>::type (&g)[2], Values<true>& x) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t at = 128 * h + 4 * lane;
    if constexpr (sizeof(G) == 4) {
      g[h] = ptx::ld_shared_f4(from + 4 * at);
    } else {
      asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(g[h].x), "=r"(g[h].y) : "r"(from + 2 * at) : "memory");
    }
    const float4 w = ptx::ld_shared_f4(from + Ahead<G>::W + 4 * at);
    x.w[h][0] = w.x; x.w[h][1] = w.y; x.w[h][2] = w.z; x.w[h][3] = w.w;
    x.mc[h] = ptx::ld_shared_u32(from + Ahead<G>::CODES + at);
    x.rc[h] = ptx::ld_shared_u32(from + Ahead<G>::CODES + SKY_STATE_BLOCK + at);
  }
  x.ms = __uint_as_float(ptx::ld_shared_u32(from + Ahead<G>::SCALES));
  x.vs = __uint_as_float(ptx::ld_shared_u32(from + Ahead<G>::SCALES + 4));
}

template <bool SMALL>
__device__ __forceinline__ void store_whole(const Tensor& t, int64_t i, const Values<SMALL>& x) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    store4(t.w + i + 128 * h, x.w[h]);
    if constexpr (SMALL) {
      *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(t.m) + i + 128 * h) = x.mc[h];
      *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(t.v) + i + 128 * h) = x.rc[h];
    } else {
      store4(static_cast<float*>(t.m) + i + 128 * h, x.m[h]);
      store4(static_cast<float*>(t.v) + i + 128 * h, x.v[h]);
    }
  }
  if (t.p) {
#pragma unroll
    for (int h = 0; h < 2; ++h) store4(t.p + i + 128 * h, x.w[h]);
  }
}

// A block that ends early or lies off the grid, value by value; what is behind the end counts as 0.
// (A call, to keep its registers out of the way of the others; it takes the settings anew, because
// what is handed over by reference lies in local memory for everybody: 435 us for 67M values.)
template <typename G, bool SMALL, int N>
__device__ __noinline__ void ragged(const Args<N>& args, int at, int64_t i0) {
  const Rule a = rule_of(args);
  const Tensor& t = args.t[at];
  const int lane = threadIdx.x & 31;
  const float wd = t.decay ? a.lr_wd : 0.f;
  Values<SMALL> x;
  float4 g[2];
  const int64_t n = t.n;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float gg[4];
    x.mc[h] = x.rc[h] = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t i = i0 + 128 * h + 4 * lane + e;
      const bool in = i < n;
      gg[e] = in ? to_f32<G>(static_cast<const G*>(t.g)[i]) : 0.f;
      x.w[h][e] = in ? t.w[i] : 0.f;
      if constexpr (SMALL) {
        if (in) {
          x.mc[h] |= static_cast<uint32_t>(static_cast<const uint8_t*>(t.m)[i]) << (8 * e);
          x.rc[h] |= static_cast<uint32_t>(static_cast<const uint8_t*>(t.v)[i]) << (8 * e);
        }
      } else {
        x.m[h][e] = in ? static_cast<const float*>(t.m)[i] : 0.f;
        x.v[h][e] = in ? static_cast<const float*>(t.v)[i] : 0.f;
      }
    }
    g[h] = make_float4(gg[0], gg[1], gg[2], gg[3]);
  }
  const int64_t blk = i0 / SKY_STATE_BLOCK;
  if constexpr (SMALL) {
    x.ms = t.ms[blk];
    x.vs = t.vs[blk];
  }
  step<SMALL>(a, g, wd, x);
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t i = i0 + 128 * h + 4 * lane + e;
      if (i >= n) continue;
      t.w[i] = x.w[h][e];
      if (t.p) t.p[i] = __float2bfloat16_rn(x.w[h][e]);
      if constexpr (SMALL) {
        static_cast<uint8_t*>(t.m)[i] = static_cast<uint8_t>(x.mc[h] >> (8 * e));
        static_cast<uint8_t*>(t.v)[i] = static_cast<uint8_t>(x.rc[h] >> (8 * e));
      } else {
        static_cast<float*>(t.m)[i] = x.m[h][e];
        static_cast<float*>(t.v)[i] = x.v[h][e];
      }
    }
  if (SMALL && lane == 0) {
    t.ms[blk] = x.ms;
    t.vs[blk] = x.vs;
  }
}

template <typename G, bool SMALL, int N>
__global__ void __launch_bounds__(THREADS, SMALL ? 2 : 4) adamw_many(const __grid_constant__ Args<N> a) {
  pdl_wait();
  pdl_trigger();
  const Rule rule = rule_of(a);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  typename Raw<G>::type g[2];
  Values<SMALL> x;
  if constexpr (SMALL) {
    extern __shared__ __align__(16) uint8_t stages[];
    constexpr int STAGES = Ahead<G>::STAGES;
    const uint32_t mine = ptx::smem_u32(stages) + warp * STAGES * Ahead<G>::BYTES;
    int at = 0, put = 0, get = 0;  // tensor, stages
    int64_t ahead = blockIdx.x;
    Place places[STAGES];  // (indexed by constants only)
    const auto look = [&]() {  // the next block, on its way
      const Place p = place_of(a, ahead, at, warp);
      ahead += gridDim.x;
      if (p.whole && p.i0 >= 0) send<G>(a.t[p.at], p.i0, mine + put * Ahead<G>::BYTES, lane);
      asm volatile("cp.async.commit_group;" ::: "memory");
      if (++put == STAGES) put = 0;
      return p;
    };
#pragma unroll
    for (int k = 0; k + 1 < STAGES; ++k) places[k] = look();
    for (int64_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {  // (everything here is warp-uniform)
      places[STAGES - 1] = look();
      const Place here = places[0];
#pragma unroll
      for (int k = 0; k + 1 < STAGES; ++k) places[k] = places[k + 1];
      asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
      __syncwarp();  // every lane's copies are here
      if (here.i0 >= 0) {  // (else: a tensor's last chunk)
        const Tensor& t = a.t[here.at];
        const float wd = t.decay ? rule.lr_wd : 0.f;
        if (here.whole) {
          receive<G>(mine + get * Ahead<G>::BYTES, lane, g, x);
          step<SMALL>(rule, g, wd, x);
          store_whole<SMALL>(t, here.i0 + 4 * lane, x);
          if (lane == 0) {
            t.ms[here.i0 / SKY_STATE_BLOCK] = x.ms;
            t.vs[here.i0 / SKY_STATE_BLOCK] = x.vs;
          }
        } else {
          ragged<G, SMALL>(a, here.at, here.i0);
        }
      }
      __syncwarp();  // every lane has read the stage
      if (++get == STAGES) get = 0;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
  } else {
    int at = 0;
    for (int64_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
      const Place here = place_of(a, c, at, warp);
      if (here.i0 < 0) continue;
      const Tensor& t = a.t[here.at];
      const float wd = t.decay ? rule.lr_wd : 0.f;
      if (here.whole) {
        load_whole<G>(t, here.i0 + 4 * lane, g, x);
        step<SMALL>(rule, g, wd, x);
        store_whole<SMALL>(t, here.i0 + 4 * lane, x);
      } else {
        ragged<G, SMALL>(a, here.at, here.i0);
      }
    }
  }
}

bool on(const void* p, size_t grid) { return reinterpret_cast<uintptr_t>(p) % grid == 0; }

sky_status check(const sky_adamw_config* c, const sky_adamw_tensor* t, int32_t n, const sky_adamw_now* now) {
  SKY_CHECK(c && t, SKY_ERR_INVALID_ARG, "null argument");
  SKY_CHECK(n > 0, SKY_ERR_INVALID_ARG, "no tensors");
  SKY_CHECK(c->grad_dtype == SKY_DTYPE_BF16 || c->grad_dtype == SKY_DTYPE_FP32, SKY_ERR_INVALID_ARG,
            "unknown gradient dtype");
  SKY_CHECK(c->states == SKY_STATE_FP32 || c->states == SKY_STATE_8BIT, SKY_ERR_INVALID_ARG, "unknown kind of states");
  SKY_CHECK(std::isfinite(c->lr) && c->lr >= 0.f && c->beta1 >= 0.f && c->beta1 < 1.f && c->beta2 >= 0.f &&
                c->beta2 < 1.f && std::isfinite(c->eps) && c->eps >= FLT_MIN && std::isfinite(c->weight_decay) &&
                c->weight_decay >= 0.f && c->step >= 1,
            SKY_ERR_INVALID_ARG, "a setting out of its range");
  SKY_CHECK(on(now, 4), SKY_ERR_INVALID_ARG, "d_now off the 4-byte grid");
  const bool small = c->states == SKY_STATE_8BIT;
  const size_t g = c->grad_dtype == SKY_DTYPE_BF16 ? 2 : 4, s = small ? 1 : 4;
  int64_t all = 0;
  for (int i = 0; i < n; ++i) {
    SKY_CHECK(t[i].w && t[i].g && t[i].m && t[i].v && (!small || (t[i].m_scale && t[i].v_scale)), SKY_ERR_INVALID_ARG,
              "null pointer in tensor %d", i);
    SKY_CHECK(t[i].n > 0 && (t[i].decay == 0 || t[i].decay == 1), SKY_ERR_INVALID_ARG, "bad size or decay in tensor %d", i);
    SKY_CHECK(t[i].n <= (int64_t{1} << 40), SKY_ERR_UNSUPPORTED, "tensor %d has more than 2^40 values", i);
    SKY_CHECK(on(t[i].w, 4) && on(t[i].g, g) && on(t[i].m, s) && on(t[i].v, s) && on(t[i].p, 2) &&
                  (!small || (on(t[i].m_scale, 4) && on(t[i].v_scale, 4))),
              SKY_ERR_INVALID_ARG, "a pointer of tensor %d off its type's grid", i);
    all += t[i].n + CHUNK;
    SKY_CHECK(all <= (int64_t{1} << 41), SKY_ERR_UNSUPPORTED, "more than 2^41 values");
  }
  return SKY_OK;
}

template <typename G, bool SMALL, int N>
sky_status launch(const sky_adamw_config& c, const sky_adamw_tensor* ts, int n, const sky_adamw_now* now, cudaStream_t st) {
  Args<N> a{};
  a.lr = c.lr; a.b1 = c.beta1; a.b2 = c.beta2; a.eps = c.eps; a.wd = c.weight_decay;
  a.c1 = static_cast<float>(1.0 - std::pow(static_cast<double>(c.beta1), static_cast<double>(c.step)));
  a.c2 = static_cast<float>(1.0 - std::pow(static_cast<double>(c.beta2), static_cast<double>(c.step)));
  a.tensors = n;
  a.now = now;
  const size_t g16 = SMALL ? 16 : 4 * sizeof(G);
  for (int i = 0; i < n; ++i) {
    const sky_adamw_tensor& t = ts[i];
    const bool vec = on(t.w, 16) && on(t.g, g16) && on(t.m, 16) && on(t.v, 16) && on(t.p, 8);
    a.t[i] = {t.w, t.g, t.m, t.v, t.m_scale, t.v_scale, static_cast<__nv_bfloat16*>(t.p), t.n, t.decay, vec};
    a.first[i] = static_cast<int32_t>(a.chunks);
    a.chunks += (t.n + CHUNK - 1) / CHUNK;
  }
  a.first[n] = static_cast<int32_t>(a.chunks);
  const int sms = sm_count();
  SKY_CHECK(sms > 0, SKY_ERR_CUDA, "no CUDA device");
  const int grid = static_cast<int>(std::min<int64_t>(a.chunks, (SMALL ? 2 : 8) * sms));
  const size_t smem = SMALL ? Ahead<G>::SMEM : 0;
  static OncePerDevice once;
  cudaError_t e = allow_smem(once, adamw_many<G, SMALL, N>, smem);
  if (e != cudaSuccess) return cuda_fail(e, "AdamW shared memory");
  e = launch_pdl(adamw_many<G, SMALL, N>, dim3(grid), dim3(THREADS), smem, st, 1, a);
  count_launches(1);
  return e == cudaSuccess ? SKY_OK : cuda_fail(e, "AdamW launch");
}

template <typename G, bool SMALL>
sky_status all(const sky_adamw_config& c, const sky_adamw_tensor* ts, int n, const sky_adamw_now* now, cudaStream_t st) {
  for (int i = 0; i < n; i += MANY) {
    const int part = std::min(MANY, n - i);
    const sky_status s = part <= FEW ? launch<G, SMALL, FEW>(c, ts + i, part, now, st)
                                     : launch<G, SMALL, MANY>(c, ts + i, part, now, st);
    if (s != SKY_OK) return s;
  }
  return SKY_OK;
}

}  // namespace
}  // namespace adamw
}  // namespace sky

using namespace sky;

extern "C" sky_status sky_adamw_step(const sky_adamw_config* config, const sky_adamw_tensor* tensors, int32_t n_tensors,
                                     const sky_adamw_now* d_now, void* stream) {
  ABI_GUARD_BEGIN
  const sky_status ok = adamw::check(config, tensors, n_tensors, d_now);
  if (ok != SKY_OK) return ok;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool small = config->states == SKY_STATE_8BIT;
  if (config->grad_dtype == SKY_DTYPE_BF16)
    return small ? adamw::all<__nv_bfloat16, true>(*config, tensors, n_tensors, d_now, st)
                 : adamw::all<__nv_bfloat16, false>(*config, tensors, n_tensors, d_now, st);
  return small ? adamw::all<float, true>(*config, tensors, n_tensors, d_now, st)
               : adamw::all<float, false>(*config, tensors, n_tensors, d_now, st);
  ABI_GUARD_END
}
