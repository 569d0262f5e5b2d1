// Root-mean-square norm of every query and key head with the rotation by position in
// the same pass, forward and backward.  Per head x of D values with gain g:
//   r = 1 / sqrt(mean(x^2) + eps),  xhat = r x,  z = g xhat,  y = R(pos) z,
// R turning each pair (z_a, z_b) by the angle pos * theta^(-2 i / D).  Backward, the
// turn being its own transpose's inverse:
//   dz = R(-pos) dy,  dg = sum over tokens and heads of dz xhat,
//   h = dz g,  dx = r (h - xhat mean(h xhat)).
//
// HBM-bound: forward reads and writes every head once, backward reads x and dy and
// writes dx; r is formed again, which costs no bytes.
//
// Layout: D / 16 lanes hold a head, each 8 values of its low half and the 8 values D / 2
// behind them, two 16-byte accesses of bf16 and, whichever way pairs are formed, both
// values of every pair.  A warp takes 32 / lanes heads a pass and NP passes a token, all
// loads of a token before the first use.  It keeps its set of heads and walks over the
// tokens, so gains and gain gradients stay in registers.
//
// Angles.  pos * frequency in fp32 is off by whole turns' fractions at far positions
// (2^-24 of 10^6 radians is 0.06).  So the host gives each frequency as a fraction of a
// turn in 64-bit fixed point, and pos * F modulo 2^64 is the turned fraction exactly, up
// to |pos| 2^-65 of a turn and what the double on the host lost.  Its top 32 bits, as a
// signed fraction, go to sincospif.  Lane i computes angles i, i + 32, ... of the token
// once for all heads of the warp, and they are shared through shared memory.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "abi.h"
#include "common.cuh"
#include "rowwise.h"

namespace sky {
namespace qkn {

constexpr int WARPS = 8, THR = WARPS * 32;
constexpr int MAX_D = 256, MAX_ANGLES = MAX_D / 2;
enum Rotation { NONE = 0, HALVES = 1, PAIRS = 2 };

struct Params {
  const void* x;    // rows of ldx values, q_heads + k_heads heads of D at the front
  const void* dy;   // backward: rows of ldy
  void* out;        // forward: y, rows of ldy; backward: dx, rows of ldx
  const void* gain[2];  // of queries and keys, or null: ones
  const int32_t* pos;
  float* part;      // backward: [2][gridDim.x][D] partial gain gradients
  int64_t ldx, ldy;
  int rows, D, heads[2];
  int chunks[2];    // sets of heads of a warp
  float eps;
  uint64_t turn[MAX_ANGLES];  // frequency i in 2^-64 turns
};

// 8 consecutive values as loaded, and as fp32
template <typename T>
struct Raw8;
template <>
struct Raw8<__nv_bfloat16> {
  uint4 u;
  __device__ void load(const __nv_bfloat16* p) { u = *reinterpret_cast<const uint4*>(p); }
  __device__ void zero() { u = make_uint4(0, 0, 0, 0); }
  __device__ void get(float (&v)[8]) const {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ void store(__nv_bfloat16* p, const float (&v)[8]) {
    __nv_bfloat162 w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<uint4*>(p) = *reinterpret_cast<uint4*>(w);
  }
};
template <>
struct Raw8<float> {
  float4 a, b;
  __device__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ void get(float (&v)[8]) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
  static __device__ void store(float* p, const float (&v)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
};

template <int LP>
__device__ __forceinline__ float head_sum(float v) {  // over the LP lanes of a head
#pragma unroll
  for (int o = LP / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// What a warp works on: the lane's place in its heads and the warp's in the grid.
template <typename T, int LP, int NP>
struct Place {
  int kind, head0;        // queries or keys; the lane's head of pass 0 (pass p: + p HPW)
  int heads;              // of the kind
  int token0, step;       // the warp's tokens
  int lo, hi;             // the lane's value offsets in a head
  bool lane_live;         // (LP lanes are a power of two, D / 16 of them hold values)
  static constexpr int HPW = 32 / LP;
  __device__ explicit Place(const Params& p) {
    const int lane = threadIdx.x & 31, n = p.chunks[0] + p.chunks[1];
    const int w = blockIdx.x * WARPS + (threadIdx.x >> 5), warps = gridDim.x * WARPS / n * n;
    int c = w % n;
    kind = c >= p.chunks[0];
    if (kind) c -= p.chunks[0];
    heads = p.heads[kind];
    head0 = c * HPW * NP + lane / LP;
    token0 = w < warps ? w / n : p.rows;
    step = warps / n;
    const int l = lane % LP;
    lane_live = l < p.D / 16;
    lo = l * 8;
    hi = p.D / 2 + l * 8;
  }
  // whether any lane has a head in the pass (the same for the whole warp)
  __device__ bool any(int pass) const { return head0 - static_cast<int>(threadIdx.x & 31) / LP + pass * HPW < heads; }
  __device__ bool live(int pass) const { return lane_live && head0 + pass * HPW < heads; }
  __device__ int64_t column(const Params& p, int pass) const {
    return static_cast<int64_t>((kind ? p.heads[0] : 0) + head0 + pass * HPW) * p.D;
  }
  __device__ void gains(const Params& p, float (&glo)[8], float (&ghi)[8]) const {
    const T* g = static_cast<const T*>(p.gain[kind]);
    if (g && lane_live) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        glo[i] = to_f32(g[lo + i]);
        ghi[i] = to_f32(g[hi + i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) glo[i] = ghi[i] = lane_live ? 1.f : 0.f;
    }
  }
};

// (cos, sin) of the lane's pairs: HALVES: pair i of (lo[i], hi[i]); PAIRS: pairs i < 4 of
// (lo[2 i], lo[2 i + 1]), then of hi.
template <int ROT, int LP>
struct Angles {
  static constexpr int N = (LP * 8 + 31) / 32;  // angles a lane computes
  uint64_t turn[N];
  float2* tab;  // the warp's
  __device__ Angles(const Params& p, float2* shared) {
    if (ROT == NONE) return;
    const int lane = threadIdx.x & 31;
    tab = shared + (threadIdx.x >> 5) * LP * 8;
#pragma unroll
    for (int i = 0; i < N; ++i) turn[i] = lane + 32 * i < p.D / 2 ? p.turn[lane + 32 * i] : 0;
  }
  __device__ void get(int pos, int D, float2 (&cs)[8]) {
    if (ROT == NONE) return;
    const int lane = threadIdx.x & 31;
    __syncwarp();  // the token before has been read
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint64_t f = turn[i] * static_cast<uint64_t>(static_cast<int64_t>(pos));
      float s, c;
      sincospif(static_cast<float>(static_cast<int32_t>(f >> 32)) * 0x1p-31f, &s, &c);
      if (N * 32 == LP * 8 || lane + 32 * i < LP * 8) tab[lane + 32 * i] = make_float2(c, s);
    }
    __syncwarp();
    const int l = lane % LP;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // (idle lanes of a head read inside the table: 8 LP entries)
      const int a = ROT == HALVES ? l * 8 + i : i < 4 ? l * 4 + i : (D / 4 + l * 4 + i - 4) % (LP * 8);
      cs[i] = tab[a];
    }
  }
};

// Turns by the angles (sign 1) or back (-1).
template <int ROT>
__device__ __forceinline__ void turn_pairs(const float2 (&cs)[8], float sign, float (&lo)[8], float (&hi)[8]) {
  auto one = [&](const float2& t, float& a, float& b) {
    const float s = sign * t.y, x = a;
    a = x * t.x - b * s;
    b = x * s + b * t.x;
  };
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (ROT == HALVES) one(cs[i], lo[i], hi[i]);
    if (ROT == PAIRS) {
      if (i < 4) one(cs[i], lo[2 * i], lo[2 * i + 1]);
      else one(cs[i], hi[2 * i - 8], hi[2 * i - 7]);
    }
  }
}

template <typename T, int LP, int ROT, int NP>
__global__ void __launch_bounds__(THR) qk_norm_fwd(const __grid_constant__ Params p) {
  __shared__ float2 tab[ROT == NONE ? 1 : WARPS * LP * 8];
  const Place<T, LP, NP> at(p);
  Angles<ROT, LP> ang(p, tab);
  const float inv = 1.f / static_cast<float>(p.D);
  pdl_wait();
  pdl_trigger();
  float glo[8], ghi[8];
  at.gains(p, glo, ghi);
  for (int t = at.token0; t < p.rows; t += at.step) {
    const T* x = static_cast<const T*>(p.x) + t * p.ldx;
    T* y = static_cast<T*>(p.out) + t * p.ldy;
    Raw8<T> rl[NP], rh[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if (at.live(i)) {
        rl[i].load(x + at.column(p, i) + at.lo);
        rh[i].load(x + at.column(p, i) + at.hi);
      } else {
        rl[i].zero();
        rh[i].zero();
      }
    }
    float2 cs[8];
    ang.get(ROT == NONE ? 0 : p.pos[t], p.D, cs);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if (!at.any(i)) continue;
      float lo[8], hi[8], ss = 0.f;
      rl[i].get(lo);
      rh[i].get(hi);
#pragma unroll
      for (int e = 0; e < 8; ++e) ss += lo[e] * lo[e] + hi[e] * hi[e];
      const float r = rsqrtf(head_sum<LP>(ss) * inv + p.eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        lo[e] = lo[e] * r * glo[e];
        hi[e] = hi[e] * r * ghi[e];
      }
      turn_pairs<ROT>(cs, 1.f, lo, hi);
      if (at.live(i)) {
        Raw8<T>::store(y + at.column(p, i) + at.lo, lo);
        Raw8<T>::store(y + at.column(p, i) + at.hi, hi);
      }
    }
  }
}

template <typename T, int LP, int ROT, int NP>
__global__ void __launch_bounds__(THR) qk_norm_bwd(const __grid_constant__ Params p) {
  __shared__ float2 tab[ROT == NONE ? 1 : WARPS * LP * 8];
  __shared__ float red[WARPS][LP * 16];
  __shared__ int kind_of[WARPS];
  const Place<T, LP, NP> at(p);
  Angles<ROT, LP> ang(p, tab);
  const float inv = 1.f / static_cast<float>(p.D);
  pdl_wait();
  pdl_trigger();
  float glo[8], ghi[8], alo[8] = {}, ahi[8] = {};
  at.gains(p, glo, ghi);
  for (int t = at.token0; t < p.rows; t += at.step) {
    const T* x = static_cast<const T*>(p.x) + t * p.ldx;
    const T* dy = static_cast<const T*>(p.dy) + t * p.ldy;
    T* dx = static_cast<T*>(p.out) + t * p.ldx;
    Raw8<T> xl[NP], xh[NP], dl[NP], dh[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if (at.live(i)) {
        xl[i].load(x + at.column(p, i) + at.lo);
        xh[i].load(x + at.column(p, i) + at.hi);
        dl[i].load(dy + at.column(p, i) + at.lo);
        dh[i].load(dy + at.column(p, i) + at.hi);
      } else {
        xl[i].zero();
        xh[i].zero();
        dl[i].zero();
        dh[i].zero();
      }
    }
    float2 cs[8];
    ang.get(ROT == NONE ? 0 : p.pos[t], p.D, cs);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if (!at.any(i)) continue;
      float lo[8], hi[8], zl[8], zh[8], ss = 0.f, sh = 0.f;
      xl[i].get(lo);
      xh[i].get(hi);
      dl[i].get(zl);
      dh[i].get(zh);
      turn_pairs<ROT>(cs, -1.f, zl, zh);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        ss += lo[e] * lo[e] + hi[e] * hi[e];
        sh += zl[e] * glo[e] * lo[e] + zh[e] * ghi[e] * hi[e];
      }
      const float r = rsqrtf(head_sum<LP>(ss) * inv + p.eps);
      const float m = head_sum<LP>(sh) * r * inv;  // mean of h xhat
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        lo[e] *= r;
        hi[e] *= r;
        alo[e] += zl[e] * lo[e];
        ahi[e] += zh[e] * hi[e];
        lo[e] = r * (zl[e] * glo[e] - lo[e] * m);
        hi[e] = r * (zh[e] * ghi[e] - hi[e] * m);
      }
      if (at.live(i)) {
        Raw8<T>::store(dx + at.column(p, i) + at.lo, lo);
        Raw8<T>::store(dx + at.column(p, i) + at.hi, hi);
      }
    }
  }
  // gain gradients: the warp's heads, then the CTA's warps in order, into one row of
  // partial sums for each kind
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
#pragma unroll
  for (int o = LP; o < 32; o <<= 1)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      alo[e] += __shfl_xor_sync(0xffffffffu, alo[e], o);
      ahi[e] += __shfl_xor_sync(0xffffffffu, ahi[e], o);
    }
  if (lane < LP && at.lane_live) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      red[w][at.lo + e] = alo[e];
      red[w][at.hi + e] = ahi[e];
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
    p.part[(static_cast<int64_t>(kind) * gridDim.x + blockIdx.x) * p.D + d] = s;
  }
}

// ------------------------------------------------------------------- host
// Calls f with the lanes of a head (a power of two), the rotation and the passes of a
// warp as constants.
template <typename F>
auto pick(const sky_qk_norm_shape& s, F&& f) {
  using std::integral_constant;
  const int lanes = s.head_dim / 16;
  const auto turn = [&](auto lp) {
    constexpr integral_constant<int, (decltype(lp)::value >= 4 ? 2 : 1)> np{};
    return s.rotation == SKY_ROTATE_HALVES  ? f(lp, integral_constant<int, HALVES>{}, np)
           : s.rotation == SKY_ROTATE_PAIRS ? f(lp, integral_constant<int, PAIRS>{}, np)
                                            : f(lp, integral_constant<int, NONE>{}, np);
  };
  return lanes <= 1   ? turn(integral_constant<int, 1>{})
         : lanes <= 2 ? turn(integral_constant<int, 2>{})
         : lanes <= 4 ? turn(integral_constant<int, 4>{})
         : lanes <= 8 ? turn(integral_constant<int, 8>{})
                      : turn(integral_constant<int, 16>{});
}

int max_ctas(bool bwd) {
  const int sms = sm_count() > 0 ? sm_count() : 148;
  return sms * (bwd ? 2 : 4);
}

sky_status check(const sky_qk_norm_shape* s) {
  SKY_CHECK(s, SKY_ERR_INVALID_ARG, "null shape");
  SKY_CHECK(s->rows > 0 && s->q_heads >= 0 && s->k_heads >= 0 && s->head_dim > 0 &&
                static_cast<int64_t>(s->q_heads) + s->k_heads > 0,
            SKY_ERR_INVALID_ARG, "bad sizes");
  SKY_CHECK(s->dtype == SKY_DTYPE_BF16 || s->dtype == SKY_DTYPE_FP32, SKY_ERR_INVALID_ARG, "unknown dtype");
  SKY_CHECK(s->rotation >= SKY_ROTATE_NONE && s->rotation <= SKY_ROTATE_PAIRS, SKY_ERR_INVALID_ARG,
            "unknown rotation");
  SKY_CHECK(s->eps >= 0.f && std::isfinite(s->eps), SKY_ERR_INVALID_ARG, "eps must be finite and not negative");
  SKY_CHECK(s->rotation == SKY_ROTATE_NONE || (s->theta > 0. && std::isfinite(s->theta)), SKY_ERR_INVALID_ARG,
            "theta must be finite and positive");
  const int64_t width = (static_cast<int64_t>(s->q_heads) + s->k_heads) * s->head_dim;
  SKY_CHECK(s->ldx >= width && s->ldy >= width, SKY_ERR_INVALID_ARG, "rows shorter than their heads");
  SKY_CHECK(s->head_dim % 16 == 0 && s->head_dim <= MAX_D, SKY_ERR_UNSUPPORTED,
            "head norms need a head dim that is a multiple of 16, up to %d (got %d)", MAX_D, s->head_dim);
  const int vec = s->dtype == SKY_DTYPE_BF16 ? 8 : 4;
  SKY_CHECK(s->ldx % vec == 0 && s->ldy % vec == 0, SKY_ERR_UNSUPPORTED,
            "head norms need rows that are multiples of 16 bytes apart");
  SKY_CHECK(width <= (1 << 24), SKY_ERR_UNSUPPORTED, "rows of more than 2^24 values");
  return SKY_OK;
}

Params params(const sky_qk_norm_shape& s, const void* q_gain, const void* k_gain, const int32_t* pos) {
  Params p = {};
  p.gain[0] = q_gain;
  p.gain[1] = k_gain;
  p.pos = pos;
  p.ldx = s.ldx;
  p.ldy = s.ldy;
  p.rows = s.rows;
  p.D = s.head_dim;
  p.heads[0] = s.q_heads;
  p.heads[1] = s.k_heads;
  p.eps = s.eps;
  if (s.rotation != SKY_ROTATE_NONE)
    for (int i = 0; i < s.head_dim / 2; ++i) {
      const double f = std::pow(s.theta, -2.0 * i / s.head_dim) / 6.283185307179586476925;
      double whole;  // (whole turns a position change nothing; they arise for theta < 1)
      p.turn[i] = static_cast<uint64_t>(std::modf(f, &whole) * 18446744073709551616.0);
    }
  return p;
}

bool a16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Chunks of heads for warps of `hpw` heads a pass and `np` passes, and the CTAs that
// give every warp a token, up to `most`.
int plan(const sky_qk_norm_shape& s, int hpw, int np, int most, Params* p) {
  p->chunks[0] = ceil_div(s.q_heads, hpw * np);
  p->chunks[1] = ceil_div(s.k_heads, hpw * np);
  const int64_t warps = static_cast<int64_t>(s.rows) * (p->chunks[0] + p->chunks[1]);
  const int least = ceil_div(p->chunks[0] + p->chunks[1], WARPS);  // a warp for every chunk
  return std::max<int64_t>(least, std::min<int64_t>(most, (warps + WARPS - 1) / WARPS));
}

template <typename T>
sky_status forward(const sky_qk_norm_shape& s, Params& p, cudaStream_t st) {
  return pick(s, [&](auto lp, auto rot, auto np) {
    constexpr int LP = decltype(lp)::value, ROT = decltype(rot)::value, NP = decltype(np)::value;
    const int ctas = plan(s, 32 / LP, NP, max_ctas(false), &p);
    const cudaError_t e = launch_pdl(qk_norm_fwd<T, LP, ROT, NP>, dim3(ctas), dim3(THR), 0, st, 1, p);
    count_launches(1);
    return e == cudaSuccess ? SKY_OK : cuda_fail(e, "head norm forward launch");
  });
}

template <typename T>
sky_status backward(const sky_qk_norm_shape& s, Params& p, float* dq_gain, float* dk_gain, cudaStream_t st) {
  int ctas = 0;
  const sky_status done = pick(s, [&](auto lp, auto rot, auto np) {
    constexpr int LP = decltype(lp)::value, ROT = decltype(rot)::value, NP = decltype(np)::value;
    ctas = plan(s, 32 / LP, NP, max_ctas(true), &p);
    const cudaError_t e = launch_pdl(qk_norm_bwd<T, LP, ROT, NP>, dim3(ctas), dim3(THR), 0, st, 1, p);
    count_launches(1);
    return e == cudaSuccess ? SKY_OK : cuda_fail(e, "head norm backward launch");
  });
  if (done != SKY_OK) return done;
  ColSegments segs = {};
  if (dq_gain) segs.seg[segs.n++] = {p.part, dq_gain, ctas, s.head_dim};
  if (dk_gain) segs.seg[segs.n++] = {p.part + static_cast<int64_t>(ctas) * s.head_dim, dk_gain, ctas, s.head_dim};
  return reduce_column_segments(segs, st);
}

size_t workspace(const sky_qk_norm_shape& s) {  // 2 rows a CTA, of as many as any plan makes
  const int most = std::max(max_ctas(true), ceil_div(static_cast<int64_t>(s.q_heads) + s.k_heads + 2, WARPS));
  return static_cast<size_t>(2) * most * s.head_dim * sizeof(float);
}

}  // namespace qkn
}  // namespace sky

using namespace sky;

extern "C" {

sky_status sky_qk_norm_fwd(const sky_qk_norm_shape* shape, const void* x, const void* q_gain, const void* k_gain,
                           const int32_t* d_pos, void* y, void* stream) {
  ABI_GUARD_BEGIN
  const sky_status ok = qkn::check(shape);
  if (ok != SKY_OK) return ok;
  SKY_CHECK(x && y, SKY_ERR_INVALID_ARG, "null argument");
  SKY_CHECK(d_pos || shape->rotation == SKY_ROTATE_NONE, SKY_ERR_INVALID_ARG, "a rotation needs positions");
  SKY_CHECK(x != y || shape->ldx == shape->ldy, SKY_ERR_INVALID_ARG, "in place needs ldx == ldy");
  SKY_CHECK(qkn::a16(x) && qkn::a16(y), SKY_ERR_UNSUPPORTED, "head norm tensors must be 16-byte aligned");
  qkn::Params p = qkn::params(*shape, q_gain, k_gain, d_pos);
  p.x = x;
  p.out = y;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return shape->dtype == SKY_DTYPE_BF16 ? qkn::forward<__nv_bfloat16>(*shape, p, st) : qkn::forward<float>(*shape, p, st);
  ABI_GUARD_END
}

size_t sky_qk_norm_bwd_workspace_bytes(const sky_qk_norm_shape* shape) {
  return shape && qkn::check(shape) == SKY_OK ? qkn::workspace(*shape) : 0;
}

sky_status sky_qk_norm_bwd(const sky_qk_norm_shape* shape, const void* x, const void* dy, const void* q_gain,
                           const void* k_gain, const int32_t* d_pos, void* dx, float* dq_gain, float* dk_gain,
                           void* workspace, size_t workspace_bytes, void* stream) {
  ABI_GUARD_BEGIN
  const sky_status ok = qkn::check(shape);
  if (ok != SKY_OK) return ok;
  SKY_CHECK(x && dy && dx && workspace, SKY_ERR_INVALID_ARG, "null argument");
  SKY_CHECK(d_pos || shape->rotation == SKY_ROTATE_NONE, SKY_ERR_INVALID_ARG, "a rotation needs positions");
  SKY_CHECK(dx != dy || shape->ldx == shape->ldy, SKY_ERR_INVALID_ARG, "in place needs ldx == ldy");
  SKY_CHECK(qkn::a16(x) && qkn::a16(dy) && qkn::a16(dx), SKY_ERR_UNSUPPORTED,
            "head norm tensors must be 16-byte aligned");
  SKY_CHECK((reinterpret_cast<uintptr_t>(workspace) & 3) == 0, SKY_ERR_INVALID_ARG,
            "workspace must be 4-byte aligned");
  SKY_CHECK(workspace_bytes >= qkn::workspace(*shape), SKY_ERR_INVALID_ARG, "workspace too small");
  qkn::Params p = qkn::params(*shape, q_gain, k_gain, d_pos);
  p.x = x;
  p.dy = dy;
  p.out = dx;
  p.part = static_cast<float*>(workspace);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return shape->dtype == SKY_DTYPE_BF16 ? qkn::backward<__nv_bfloat16>(*shape, p, dq_gain, dk_gain, st)
                                        : qkn::backward<float>(*shape, p, dq_gain, dk_gain, st);
  ABI_GUARD_END
}

}  // extern "C"
