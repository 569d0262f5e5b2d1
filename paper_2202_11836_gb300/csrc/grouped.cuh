// Which group a tile of a ragged matrix belongs to, and GELU for the grouped products (device code).
#pragma once
#include "common.cuh"

namespace sky {
namespace grouped {

// The rows of group g, inside [0, rows] whatever the offsets hold.
__device__ __forceinline__ int2 group_rows(const int32_t* offset, int g, int rows) {
  const int lo = min(max(offset[g], 0), rows);
  return make_int2(lo, min(max(offset[g + 1], lo), rows));
}

struct Found {
  int group;   // -1: there are no so many tiles
  int lo, hi;  // its rows
  int tile;    // of the group's tiles
};

// The tile-th of all groups' tiles, tiles_of(n) of a group of n rows: a whole warp, 32 groups
// at a time.
template <typename F>
__device__ __forceinline__ Found find_tile(const int32_t* offset, int groups, int rows, int tile, F&& tiles_of) {
  const int lane = threadIdx.x & 31;
  for (int g0 = 0; g0 < groups; g0 += 32) {
    int2 r = make_int2(0, 0);
    if (g0 + lane < groups) r = group_rows(offset, g0 + lane, rows);
    const int n = tiles_of(r.y - r.x);
    int upto = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += up;
    }
    const uint32_t past = __ballot_sync(0xffffffffu, tile < upto);
    if (past) {
      const int at = __ffs(past) - 1;
      return {g0 + at, __shfl_sync(0xffffffffu, r.x, at), __shfl_sync(0xffffffffu, r.y, at),
              tile - __shfl_sync(0xffffffffu, upto - n, at)};
    }
    tile -= __shfl_sync(0xffffffffu, upto, 31);
  }
  return {-1, 0, 0, 0};
}

// Sets the bad-length bit where the offsets decrease or leave [0, rows]: by one thread block.
__device__ __forceinline__ void check_offsets(const int32_t* offset, int groups, int rows, int32_t* status) {
  if (!status) return;
  for (int g = threadIdx.x; g < groups; g += blockDim.x)
    if (offset[g] < 0 || offset[g + 1] < offset[g] || offset[g + 1] > rows) atomicOr(status, kStatusBadLength);
}

// GELU(h) = h Phi(h) and GELU'(h) = Phi(h) + h phi(h) of two values, in packed arithmetic where it
// pairs up.  With a = |h|, t = 1 / (1 + c a) and E = exp(-a^2 / 2), Phi(-a) = E t P(t): P is the
// polynomial of degree 6 whose largest relative error over a <= 13.5 is least (a linear program over
// 2400 points; c by search), 6.2e-7.  In fp32, with the hardware's reciprocal and exponential, Phi(-a) is
// off by at most 2^-18 + 1.5 a^2 2^-24 of itself, the second part being the exponent's roundings: the
// outputs are what bf16 and fp16 make of the exact values but for a few borders, in the tail too.  The
// three terms of the dense epilogues (gelu_and_grad_as2) are off by 2.2e-5 of 1, 0.4% of GELU(-3) and 2% of
// GELU(-5).  16384 rows, 8 groups of 4096 x 1024: 100.2 us with those, 100.7 with these; with one more
// term 102, and with the sign by arithmetic in the place of selects 5 more.
__device__ __forceinline__ void gelu_and_grad2(float h0, float h1, float2& g, float2& gp) {
  const auto both = [](float v) { return pack2(v, v); };
  constexpr float c = 0.265f;
  constexpr float P[7] = {0.105599828f, 0.107836783f, 0.0829465427f, 0.142493453f,
                          -0.0663631036f, 0.195273253f, -0.0677870684f};
  float t0, t1, e0, e1;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t0) : "f"(fmaf(fabsf(h0), c, 1.f)));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t1) : "f"(fmaf(fabsf(h1), c, 1.f)));
  const uint64_t h = pack2(h0, h1), t = pack2(t0, t1);
  const float2 x = unpack2(mul2(mul2(h, both(-0.72134752044448170f)), h));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(x.x));  // exp(-h^2/2)
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(x.y));
  const uint64_t E = pack2(e0, e1);
  uint64_t poly = both(P[6]);
#pragma unroll
  for (int i = 5; i >= 0; --i) poly = fma2(t, poly, both(P[i]));
  const uint64_t q = mul2(mul2(t, poly), E);
  const float2 lower = unpack2(q), upper = unpack2(fma2(q, both(-1.f), both(1.f)));
  const uint64_t Phi = pack2(h0 < 0.f ? lower.x : upper.x, h1 < 0.f ? lower.y : upper.y);
  g = unpack2(mul2(h, Phi));
  gp = unpack2(fma2(mul2(h, both(0.3989422804014327f)), E, Phi));
}

}  // namespace grouped
}  // namespace sky
