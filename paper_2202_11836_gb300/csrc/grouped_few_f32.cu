// fp32 products y = x W^T grouped by expert for few rows (a decoder's new tokens): as in
// grouped_few.cu the weights of every group that has a row are read once, for a handful of tokens
// each, so HBM bounds them, not the FMA pipe that the tiles of grouped_f32.cu are made for.
//
// A unit is up to four tokens of one group by the features of one block: four features a warp,
// whose lanes go along the inner dimension with 16-byte loads, and 4 x 4 sums a lane.  The sum over
// a warp halves the values that a lane holds at each step, so that 16 sums cost 16 exchanges and
// every value ends in a lane of its own.  Units of eight tokens read weights less often, but their
// code, fetched once a launch, is longer than the work of a small call (64 rows of 64 x 64 over 4
// groups 3.1 us with four, 6.0 with eight; 64 rows of 768 x 768 over 8 groups 10.8 and 13.9).
// Tiles of the same group are neighbours, which finds their weights in the L2 cache.  Where there
// are few units the warps of a block split the inner dimension and add in order.
//
// Bound by HBM with a row a group (8 rows, 8 groups of 4096 x 1024 22.3 us, 6.0 TB/s; 768 x 768 4.1),
// by the loads from the first-level cache with eight (64 rows 51).
#include <algorithm>

#include "common.cuh"
#include "grouped.cuh"
#include "grouped.h"
#include "ptx.cuh"

namespace sky {
namespace grouped {
namespace {

constexpr int ROWS = 4, FEATURES = 4, WARPS = 4, STEP = 128;

struct Params {
  Call c;
  int tiles, kw;  // tiles of tokens that the rows may make; warps along the inner dimension
};

// Sums N values a lane over the warp; a lane returns the sum of value lane / (32 / N).
template <int N>
__device__ __forceinline__ float warp_sums(float (&v)[N]) {
  const int lane = threadIdx.x & 31;
  int n = N;
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) {
    if (n > 1) {
      n /= 2;
      const bool up = lane & s;
#pragma unroll
      for (int i = 0; i < n; ++i) {
        const float keep = up ? v[i + n] : v[i], send = up ? v[i] : v[i + n];
        v[i] = keep + __shfl_xor_sync(0xffffffffu, send, s);
      }
    } else {
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], s);
    }
  }
  return v[0];
}

// Four elements of a lane, of the 128 from p: zeros behind the k-th.
template <bool VEC>
__device__ __forceinline__ float4 four(const float* p, int k) {
  const int lane = threadIdx.x & 31;
  if constexpr (VEC) {
    return lane * 4 < k ? __ldg(reinterpret_cast<const float4*>(p) + lane) : make_float4(0.f, 0.f, 0.f, 0.f);
  } else {
    return make_float4(lane < k ? __ldg(p + lane) : 0.f, lane + 32 < k ? __ldg(p + lane + 32) : 0.f,
                       lane + 64 < k ? __ldg(p + lane + 64) : 0.f, lane + 96 < k ? __ldg(p + lane + 96) : 0.f);
  }
}

// The sums over [k0, k1) of four features and R rows; those behind the last are the last's.
template <bool VEC, int R>
__device__ __forceinline__ float dots(const float* __restrict__ x, const float* __restrict__ w, int count, int features,
                                      int K, int k0, int k1) {
  float acc[FEATURES * R] = {};
#pragma unroll 2
  for (int k = k0; k < k1; k += STEP) {
    float4 a[FEATURES];
#pragma unroll
    for (int j = 0; j < FEATURES; ++j) a[j] = four<VEC>(w + static_cast<int64_t>(min(j, features - 1)) * K + k, k1 - k);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float4 b = four<VEC>(x + static_cast<int64_t>(min(r, count - 1)) * K + k, k1 - k);
#pragma unroll
      for (int j = 0; j < FEATURES; ++j) {
        float& s = acc[j * R + r];
        s = fmaf(a[j].x, b.x, s);
        s = fmaf(a[j].y, b.y, s);
        s = fmaf(a[j].z, b.z, s);
        s = fmaf(a[j].w, b.w, s);
      }
    }
  }
  return warp_sums(acc);
}

template <bool VEC>
__global__ void __launch_bounds__(32 * WARPS, 4) grouped_few_f32(const __grid_constant__ Params p) {
  __shared__ float part[WARPS][32];
  const Call& c = p.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();
  if (blockIdx.x == 0) check_offsets(c.offset, c.groups, c.rows, c.status);
  const Found at = find_tile(c.offset, c.groups, c.rows, static_cast<int>(blockIdx.x) % p.tiles,
                             [](int n) { return (n + ROWS - 1) / ROWS; });
  pdl_trigger();
  if (at.group < 0) return;
  const int row = at.lo + at.tile * ROWS, count = min(ROWS, at.hi - row);
  const int f = (static_cast<int>(blockIdx.x) / p.tiles * (WARPS / p.kw) + warp / p.kw) * FEATURES;
  const int features = min(FEATURES, c.out - f);  // (none, for the last warps)
  const int steps = (c.in + STEP - 1) / STEP, mine = warp % p.kw;
  const int k0 = mine * steps / p.kw * STEP, k1 = min((mine + 1) * steps / p.kw * STEP, c.in);
  const float* x = static_cast<const float*>(c.A) + static_cast<int64_t>(row) * c.in;
  const float* w = static_cast<const float*>(c.B) + (static_cast<int64_t>(at.group) * c.out + f) * c.in;
  const int R = count > 2 ? 4 : count;
  float v = 0.f;
  if (features > 0)
    v = R == 4   ? dots<VEC, 4>(x, w, count, features, c.in, k0, k1)
        : R == 2 ? dots<VEC, 2>(x, w, count, features, c.in, k0, k1)
                 : dots<VEC, 1>(x, w, count, features, c.in, k0, k1);
  if (p.kw > 1) {
    part[warp][lane] = v;
    __syncthreads();
    if (mine != 0) return;
    for (int i = 1; i < p.kw; ++i) v += part[warp + i][lane];
  }
  const int same = 8 / R, value = lane / same, j = value / R, r = value % R;  // lanes of the same value
  if (lane % same != 0 || j >= features || r >= count) return;
  const int64_t off = static_cast<int64_t>(row + r) * c.out + f + j;
  if (c.bias) v += static_cast<const float*>(c.bias)[static_cast<int64_t>(at.group) * c.out + f + j];
  if (c.epi == SKY_EPI_BIAS_GELU) {
    static_cast<float*>(c.aux_out)[off] = gelu_grad_f(v);
    v = gelu_f(v);
  }
  static_cast<float*>(c.C)[off] = v;
}

}  // namespace

// us of the tiles of grouped_f32.cu and here: 8 groups of 768 x 768, 8 rows 18.8 4.1, 64 rows 20.3
// 10.1; one group of it, 8 rows 7.9 4.4, 32 rows 7.9 6.0, 64 rows 8.1 9.8; 64 groups of 512 x 128, 64
// rows 13.1 8.9, 256 rows 16.1 16.1, 512 rows 16.5 25.8.
bool few_f32_pays(const Call& c) { return c.form == SKY_GEMM_XWT && c.rows <= 64 && c.rows <= 32 * c.groups; }

sky_status launch_few_f32(const Call& c, cudaStream_t st) {
  const int sms = sm_count();
  SKY_CHECK(sms > 0, SKY_ERR_CUDA, "no CUDA device");
  Params p{};
  p.c = c;
  const int64_t tiles = c.rows / ROWS + static_cast<int64_t>(std::min(c.groups, c.rows));
  const auto a16 = [](const void* q) { return (reinterpret_cast<uintptr_t>(q) & 15) == 0; };
  const bool vec = c.in % 4 == 0 && a16(c.A) && a16(c.B);
  const int steps = ceil_div(c.in, STEP);
  // Warps along the inner dimension: as many as make no more than four blocks an SM and have 1.5
  // steps each.  us at 1 / 2 / 4: 8 rows of 512 x 2048 over 4 groups (192 blocks at 1) 6.8 6.0 5.4, a row
  // of it (32) 4.5 3.6 3.1; 768 x 768, one group, a row (48) 3.1 3.0 2.8, 16 rows (240) 5.2 5.2 7.1, 32
  // rows (432) 6.0 8.2 10.3.
  p.kw = 1;
  while (p.kw < 4 && tiles * ceil_div(c.out, FEATURES * WARPS) * p.kw * 2 <= 4 * sms && steps >= 3 * p.kw) p.kw *= 2;
  const int f_blocks = ceil_div(c.out, FEATURES * (WARPS / p.kw));
  p.tiles = static_cast<int>(tiles);
  SKY_CHECK(tiles * f_blocks <= 0x7fffffff, SKY_ERR_UNSUPPORTED, "grouped product too large");
  const dim3 grid(static_cast<unsigned>(tiles * f_blocks));
  const cudaError_t e = vec ? launch_pdl(grouped_few_f32<true>, grid, dim3(32 * WARPS), 0, st, 1, p)
                            : launch_pdl(grouped_few_f32<false>, grid, dim3(32 * WARPS), 0, st, 1, p);
  count_launches(1);
  return e == cudaSuccess ? SKY_OK : cuda_fail(e, "grouped product of few rows launch");
}

}  // namespace grouped
}  // namespace sky
