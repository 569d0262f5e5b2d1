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
// its tensor is found by walking on from the one before.
//
// Products and sums of the moments are rounded one by one (no fused multiply-add): what a
// byte holds then does not depend on which of them a compiler contracts.
#include <cuda_fp8.h>

#include <cmath>

#include "../../include/sky_optim.h"
#include "abi.h"
#include "common.cuh"

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

// Four values at i; those from n on are 0.
template <typename T>
__device__ __forceinline__ float4 load4(const T* x, int64_t i, int64_t n, bool vec) {
  if (vec) {
    if constexpr (sizeof(T) == 4) {
      return __ldcs(reinterpret_cast<const float4*>(x + i));
    } else {
      const uint2 u = __ldcs(reinterpret_cast<const uint2*>(x + i));
      return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                         __uint_as_float(u.y & 0xffff0000u));
    }
  }
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = i + e < n ? to_f32<T>(x[i + e]) : 0.f;
  return make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ uint32_t load4(const uint8_t* x, int64_t i, int64_t n, bool vec) {
  if (vec) return __ldcs(reinterpret_cast<const uint32_t*>(x + i));
  uint32_t v = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (i + e < n) v |= static_cast<uint32_t>(x[i + e]) << (8 * e);
  return v;
}
__device__ __forceinline__ void store4(float* x, int64_t i, int64_t n, bool vec, const float (&v)[4]) {
  if (vec) {
    __stcs(reinterpret_cast<float4*>(x + i), make_float4(v[0], v[1], v[2], v[3]));
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (i + e < n) x[i + e] = v[e];
}
__device__ __forceinline__ void store4(__nv_bfloat16* x, int64_t i, int64_t n, bool vec, const float (&v)[4]) {
  if (vec) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
    __stcs(reinterpret_cast<uint2*>(x + i),
           make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b)));
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (i + e < n) x[i + e] = __float2bfloat16_rn(v[e]);
}
__device__ __forceinline__ void store4(uint8_t* x, int64_t i, int64_t n, bool vec, uint32_t v) {
  if (vec) {
    __stcs(reinterpret_cast<uint32_t*>(x + i), v);
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (i + e < n) x[i + e] = static_cast<uint8_t>(v >> (8 * e));
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
__device__ __forceinline__ float r_value(uint32_t c) {
  return c ? __uint_as_float((c + (111u << 4)) << 19) : 0.f;
}
__device__ __forceinline__ uint32_t r_code(float y) {
  const uint32_t b = __float_as_uint(y);
  const int c = static_cast<int>((b + 0x3ffffu + ((b >> 19) & 1u)) >> 19) - (111 << 4);
  return y == 0.f ? 0u : static_cast<uint32_t>(min(max(c, 1), 255));
}

// The scale of a block whose largest |x| has these bits, and its inverse.
__device__ __forceinline__ void block_scale(uint32_t top_bits, float unit, float& scale, float& inv) {
  const float top = __uint_as_float(top_bits);
  const bool zero = top < TINY;
  scale = zero ? 0.f : __fmul_rn(top, unit);
  inv = zero ? 0.f : __frcp_rn(scale);
}

template <typename G, bool SMALL, int N>
__global__ void __launch_bounds__(THREADS) adamw_many(const __grid_constant__ Args<N> a) {
  pdl_wait();
  pdl_trigger();
  float lr = a.lr, c1 = a.c1, c2 = a.c2, gs = 1.f;
  if (a.now) {
    lr = a.now->lr;
    c1 = a.now->correction1;
    c2 = a.now->correction2;
    gs = a.now->grad_scale;
  }
  const float i1 = __frcp_rn(c1), i2 = __frcp_rn(c2), root2 = __fsqrt_rn(i2);
  const float d1 = __fsub_rn(1.f, a.b1), d2 = __fsub_rn(1.f, a.b2);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int at = 0;
  for (int64_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
    while (c >= a.first[at + 1]) ++at;
    const Tensor& t = a.t[at];
    const int64_t blk = (c - a.first[at]) * (THREADS / 32) + warp, i0 = blk * SKY_STATE_BLOCK, n = t.n;
    if (i0 >= n) continue;  // warp-uniform: a tensor's last chunk
    const bool whole = t.vec && i0 + SKY_STATE_BLOCK <= n;
    float w[2][4], m[2][4], r[2][4];
    float4 g4[2], w4[2], m4[2], v4[2];
    uint32_t mc[2], vc[2];
    float ms = 0.f, vs = 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t i = i0 + 128 * h + 4 * lane;
      g4[h] = load4(static_cast<const G*>(t.g), i, n, whole);
      w4[h] = load4(static_cast<const float*>(t.w), i, n, whole);
      if constexpr (SMALL) {
        mc[h] = load4(static_cast<const uint8_t*>(t.m), i, n, whole);
        vc[h] = load4(static_cast<const uint8_t*>(t.v), i, n, whole);
      } else {
        m4[h] = load4(static_cast<const float*>(t.m), i, n, whole);
        v4[h] = load4(static_cast<const float*>(t.v), i, n, whole);
      }
    }
    if constexpr (SMALL) {
      ms = t.ms[blk];
      vs = t.vs[blk];
    }
    const float wd = t.decay ? __fmul_rn(lr, a.wd) : 0.f;
    uint32_t m_top = 0, r_top = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float g[4] = {g4[h].x, g4[h].y, g4[h].z, g4[h].w};
      float v[4];
      w[h][0] = w4[h].x; w[h][1] = w4[h].y; w[h][2] = w4[h].z; w[h][3] = w4[h].w;
      if constexpr (SMALL) {
        m_values(mc[h], ms, m[h]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = __fmul_rn(r_value((vc[h] >> (8 * e)) & 255u), vs);
          v[e] = __fmul_rn(x, x);
        }
      } else {
        m[h][0] = m4[h].x; m[h][1] = m4[h].y; m[h][2] = m4[h].z; m[h][3] = m4[h].w;
        v[0] = v4[h].x; v[1] = v4[h].y; v[2] = v4[h].z; v[3] = v4[h].w;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = __fmul_rn(g[e], gs);
        m[h][e] = __fadd_rn(__fmul_rn(m[h][e], a.b1), __fmul_rn(x, d1));
        v[e] = __fadd_rn(__fmul_rn(v[e], a.b2), __fmul_rn(__fmul_rn(x, x), d2));
        r[h][e] = __fsqrt_rn(v[e]);
        const float step = (m[h][e] * i1) / (r[h][e] * root2 + a.eps);
        w[h][e] = w[h][e] - wd * w[h][e];
        w[h][e] = w[h][e] - lr * step;
        if constexpr (SMALL) {
          m_top = max(m_top, __float_as_uint(m[h][e]) & 0x7fffffffu);
          r_top = max(r_top, __float_as_uint(r[h][e]) & 0x7fffffffu);
        } else {
          r[h][e] = v[e];  // what is stored
        }
      }
    }
    float m_inv = 0.f, r_inv = 0.f;
    if constexpr (SMALL) {
      block_scale(__reduce_max_sync(0xffffffffu, m_top), 1.f / 448.f, ms, m_inv);
      block_scale(__reduce_max_sync(0xffffffffu, r_top), 1.f / 0.96875f, vs, r_inv);
      if (lane == 0) {
        t.ms[blk] = ms;
        t.vs[blk] = vs;
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t i = i0 + 128 * h + 4 * lane;
      store4(t.w, i, n, whole, w[h]);
      if constexpr (SMALL) {
        store4(static_cast<uint8_t*>(t.m), i, n, whole, m_codes(m[h], m_inv));
        uint32_t codes = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) codes |= r_code(__fmul_rn(r[h][e], r_inv)) << (8 * e);
        store4(static_cast<uint8_t*>(t.v), i, n, whole, codes);
      } else {
        store4(static_cast<float*>(t.m), i, n, whole, m[h]);
        store4(static_cast<float*>(t.v), i, n, whole, r[h]);
      }
      if (t.p) store4(t.p, i, n, whole, w[h]);
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
                c->beta2 < 1.f && std::isfinite(c->eps) && c->eps > 0.f && std::isfinite(c->weight_decay) &&
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
  const size_t g16 = 4 * sizeof(G), s16 = SMALL ? 4 : 16;
  for (int i = 0; i < n; ++i) {
    const sky_adamw_tensor& t = ts[i];
    const bool vec = on(t.w, 16) && on(t.g, g16) && on(t.m, s16) && on(t.v, s16) && on(t.p, 8);
    a.t[i] = {t.w, t.g, t.m, t.v, t.m_scale, t.v_scale, static_cast<__nv_bfloat16*>(t.p), t.n, t.decay, vec};
    a.first[i] = static_cast<int32_t>(a.chunks);
    a.chunks += (t.n + CHUNK - 1) / CHUNK;
  }
  a.first[n] = static_cast<int32_t>(a.chunks);
  const int sms = sm_count();
  SKY_CHECK(sms > 0, SKY_ERR_CUDA, "no CUDA device");
  const int grid = static_cast<int>(std::min<int64_t>(a.chunks, 8 * sms));
  const cudaError_t e = launch_pdl(adamw_many<G, SMALL, N>, dim3(grid), dim3(THREADS), 0, st, 1, a);
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
