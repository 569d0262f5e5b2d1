// Tokens' rows to the experts' order and back (sky_experts.h).
//
// Streams bound by HBM: (1 + top_k) rows of a token are read or written once (the gradient
// of the weighted sum: 1 + 2 top_k).  A warp takes a token's row, or a piece of it, 16
// bytes a lane; lane c holds where choice c lies.  The loads of two or four choices are
// issued before the first is used.  Which rows a token names decides nothing but addresses,
// so there are no atomics, and a sum's order is that of the choices.
#include <algorithm>

#include "../../include/sky_experts.h"
#include "abi.h"
#include "common.cuh"

namespace sky {
namespace erows {
namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int U = 2;               // 16-byte pieces of a lane
constexpr int SEG = 32 * U;        // pieces of a warp
constexpr int WIDE = 128;          // pieces that a warp of combine_backward takes, at most, while there are more warps
constexpr int MAX_TOP_K = 32;

struct Params {
  int tokens, top_k, pieces, segs;  // 16-byte pieces of a row, and groups of SEG of them
  const uint4* in;
  const uint4* in2;
  const int32_t* row;
  const float* weight;
  uint4* out;
  float* dweight;
};

template <typename T> struct Piece;
template <> struct Piece<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(const uint4& u, float (&v)[4]) {
    v[0] = __uint_as_float(u.x); v[1] = __uint_as_float(u.y); v[2] = __uint_as_float(u.z); v[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 put(const float (&v)[4]) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  }
};
template <> struct Piece<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(const uint4& u, float (&v)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 put(const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// Lane c: the place of the token's choice c, -1 if it has no row.
__device__ __forceinline__ int place_of(const Params& p, int t, int lane) {
  if (lane >= p.top_k) return -1;
  const int r = p.row[static_cast<int64_t>(t) * p.top_k + lane];
  return static_cast<int64_t>(r) < static_cast<int64_t>(p.tokens) * p.top_k ? r : -1;
}
__device__ __forceinline__ float weight_of(const Params& p, int t, int lane) {
  return lane < p.top_k ? p.weight[static_cast<int64_t>(t) * p.top_k + lane] : 0.f;
}

__global__ void __launch_bounds__(THREADS) dispatch_rows(const Params p) {
  pdl_wait();
  pdl_trigger();
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * WARPS + (threadIdx.x >> 5);
  const int t = static_cast<int>(unit / p.segs), seg = static_cast<int>(unit % p.segs), lane = threadIdx.x & 31;
  if (t >= p.tokens) return;
  const int place = place_of(p, t, lane);
  uint4 v[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = seg * SEG + u * 32 + lane;
    if (i < p.pieces) v[u] = p.in[static_cast<int64_t>(t) * p.pieces + i];
  }
  for (int c = 0; c < p.top_k; ++c) {
    const int r = __shfl_sync(0xffffffffu, place, c);
    if (r < 0) continue;  // warp-uniform
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = seg * SEG + u * 32 + lane;
      if (i < p.pieces) p.out[static_cast<int64_t>(r) * p.pieces + i] = v[u];
    }
  }
}

// Sums of rows.  N choices' loads are in flight together: two for up to two choices, whose smaller
// registers leave room for more warps, else four.
template <typename T, bool WEIGHTED, int N>
__global__ void __launch_bounds__(THREADS) add_rows(const Params p) {
  using P = Piece<T>;
  pdl_wait();
  pdl_trigger();
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * WARPS + (threadIdx.x >> 5);
  const int t = static_cast<int>(unit / p.segs), seg = static_cast<int>(unit % p.segs), lane = threadIdx.x & 31;
  if (t >= p.tokens) return;
  const int place = place_of(p, t, lane);
  const float weight = WEIGHTED ? weight_of(p, t, lane) : 1.f;
  float sum[U][P::N] = {};
  for (int c0 = 0; c0 < p.top_k; c0 += N) {
    uint4 v[N][U];
    int r[N];
#pragma unroll
    for (int c = 0; c < N; ++c) {
      r[c] = c0 + c < p.top_k ? __shfl_sync(0xffffffffu, place, c0 + c) : -1;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = seg * SEG + u * 32 + lane;
        if (r[c] >= 0 && i < p.pieces) v[c][u] = p.in[static_cast<int64_t>(r[c]) * p.pieces + i];
      }
    }
#pragma unroll
    for (int c = 0; c < N; ++c) {
      if (r[c] < 0) continue;
      const float w = WEIGHTED ? __shfl_sync(0xffffffffu, weight, c0 + c) : 1.f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float x[P::N];
        P::get(v[c][u], x);
#pragma unroll
        for (int e = 0; e < P::N; ++e) sum[u][e] = WEIGHTED ? fmaf(w, x[e], sum[u][e]) : sum[u][e] + x[e];
      }
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = seg * SEG + u * 32 + lane;
    if (i < p.pieces) p.out[static_cast<int64_t>(t) * p.pieces + i] = P::put(sum[u]);
  }
}

// in: rows, in2: dy.  W warps take a row, all of it at once where it has up to 64 W pieces, and
// add up their parts of the dot products in order.
template <typename T, int W, int N>
__global__ void __launch_bounds__(THREADS) combine_backward(const Params p) {
  using P = Piece<T>;
  constexpr int TOKENS = WARPS / W;
  __shared__ float parts[TOKENS][W][MAX_TOP_K];
  pdl_wait();
  pdl_trigger();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, local = warp / W, w = warp % W;
  const int t = blockIdx.x * TOKENS + local;
  if (t < p.tokens) {
    const int place = place_of(p, t, lane);
    const float weight = weight_of(p, t, lane);
    float mine = 0.f;  // lane c: its choice's dot product
    for (int c0 = 0; c0 < p.top_k; c0 += N) {
      int r[N];
      float wt[N], dot[N] = {};
#pragma unroll
      for (int c = 0; c < N; ++c) {
        r[c] = c0 + c < p.top_k ? __shfl_sync(0xffffffffu, place, c0 + c) : -1;
        wt[c] = __shfl_sync(0xffffffffu, weight, (c0 + c) & 31);
      }
      for (int i0 = w * 32 + lane; i0 < p.pieces; i0 += U * 32 * W) {
        uint4 d4[U], v[N][U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = i0 + 32 * W * u;
          if (i >= p.pieces) continue;
          d4[u] = p.in2[static_cast<int64_t>(t) * p.pieces + i];
#pragma unroll
          for (int c = 0; c < N; ++c)
            if (r[c] >= 0) v[c][u] = p.in[static_cast<int64_t>(r[c]) * p.pieces + i];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = i0 + 32 * W * u;
          if (i >= p.pieces) continue;
          float d[P::N];
          P::get(d4[u], d);
#pragma unroll
          for (int c = 0; c < N; ++c) {
            if (r[c] < 0) continue;
            float x[P::N];
            P::get(v[c][u], x);
#pragma unroll
            for (int e = 0; e < P::N; ++e) {
              dot[c] = fmaf(x[e], d[e], dot[c]);
              x[e] = wt[c] * d[e];
            }
            p.out[static_cast<int64_t>(r[c]) * p.pieces + i] = P::put(x);
          }
        }
      }
#pragma unroll
      for (int c = 0; c < N; ++c) {
        const float s = warp_sum(dot[c]);
        if (lane == c0 + c) mine = s;
      }
    }
    parts[local][w][lane] = mine;
  }
  __syncthreads();
  if (t < p.tokens && w == 0 && lane < p.top_k) {
    float s = parts[local][0][lane];
#pragma unroll
    for (int i = 1; i < W; ++i) s += parts[local][i][lane];
    p.dweight[static_cast<int64_t>(t) * p.top_k + lane] = s;
  }
}

sky_status check(const sky_rows_shape* s) {
  SKY_CHECK(s, SKY_ERR_INVALID_ARG, "null shape");
  SKY_CHECK(s->tokens > 0 && s->top_k > 0 && s->width > 0, SKY_ERR_INVALID_ARG, "bad sizes");
  SKY_CHECK(s->dtype == SKY_DTYPE_BF16 || s->dtype == SKY_DTYPE_FP32, SKY_ERR_INVALID_ARG, "unknown dtype");
  SKY_CHECK(s->width % (s->dtype == SKY_DTYPE_BF16 ? 8 : 4) == 0 && s->width <= (1 << 20), SKY_ERR_UNSUPPORTED,
            "experts' rows need a width of 16-byte pieces, up to 2^20 values (got %d)", s->width);
  SKY_CHECK(s->top_k <= MAX_TOP_K && static_cast<int64_t>(s->tokens) * s->top_k < (int64_t{1} << 31),
            SKY_ERR_UNSUPPORTED, "more than %d choices a token, or 2^31 or more in all", MAX_TOP_K);
  return SKY_OK;
}

bool on(const void* p, size_t grid) { return reinterpret_cast<uintptr_t>(p) % grid == 0; }

using Kernel = void (*)(Params);

// Warps for a row of combine_backward, up to eight: four pieces a lane of each.
int warps_of(int pieces) {
  int w = 1;
  while (w < WARPS && pieces > WIDE * w) w *= 2;
  return w;
}
template <typename T, int N>
Kernel backward_of(int warps) {
  switch (warps) {
    case 1: return combine_backward<T, 1, N>;
    case 2: return combine_backward<T, 2, N>;
    case 4: return combine_backward<T, 4, N>;
    default: return combine_backward<T, 8, N>;
  }
}
template <typename T>
Kernel backward_of(int warps, int top_k) {
  return top_k <= 2 ? backward_of<T, 2>(warps) : backward_of<T, 4>(warps);
}

enum Kind { DISPATCH, ADD, ADD_WEIGHTED, BACKWARD };

template <bool WEIGHTED>
Kernel add_of(const sky_rows_shape& s) {
  if (s.dtype == SKY_DTYPE_BF16)
    return s.top_k <= 2 ? add_rows<__nv_bfloat16, WEIGHTED, 2> : add_rows<__nv_bfloat16, WEIGHTED, 4>;
  return s.top_k <= 2 ? add_rows<float, WEIGHTED, 2> : add_rows<float, WEIGHTED, 4>;
}

sky_status launch(const sky_rows_shape& s, Params& p, Kind kind, cudaStream_t st) {
  p.tokens = s.tokens;
  p.top_k = s.top_k;
  p.pieces = s.width / (s.dtype == SKY_DTYPE_BF16 ? 8 : 4);
  p.segs = ceil_div(p.pieces, SEG);
  int64_t warps = static_cast<int64_t>(p.tokens) * p.segs;
  Kernel kern = kind == DISPATCH ? dispatch_rows : kind == ADD ? add_of<false>(s) : add_of<true>(s);
  if (kind == BACKWARD) {
    const int w = warps_of(p.pieces);
    kern = s.dtype == SKY_DTYPE_BF16 ? backward_of<__nv_bfloat16>(w, s.top_k) : backward_of<float>(w, s.top_k);
    warps = static_cast<int64_t>(p.tokens) * w;
  }
  const int64_t ctas = (warps + WARPS - 1) / WARPS;
  SKY_CHECK(ctas <= 0x7fffffff, SKY_ERR_UNSUPPORTED, "too many rows");
  const cudaError_t e = launch_pdl(kern, dim3(static_cast<unsigned>(ctas)), dim3(THREADS), 0, st, 1, p);
  count_launches(1);
  return e == cudaSuccess ? SKY_OK : cuda_fail(e, "experts' rows launch");
}

// One of the two kinds of calls of a matrix, an index and a matrix.
sky_status run(const sky_rows_shape* s, const void* in, const void* in2, const int32_t* row, const float* weight,
               void* out, float* dweight, Kind kind, void* stream) {
  const sky_status ok = check(s);
  if (ok != SKY_OK) return ok;
  SKY_CHECK(in && row && out && (kind < ADD_WEIGHTED || weight) && (kind != BACKWARD || (in2 && dweight)), SKY_ERR_INVALID_ARG, "null argument");
  SKY_CHECK(on(row, 4) && on(weight, 4) && on(dweight, 4), SKY_ERR_INVALID_ARG, "row or weights off the 4-byte grid");
  SKY_CHECK(on(in, 16) && on(in2, 16) && on(out, 16), SKY_ERR_UNSUPPORTED, "matrices must be 16-byte aligned");
  Params p{};
  p.in = static_cast<const uint4*>(in);
  p.in2 = static_cast<const uint4*>(in2);
  p.row = row;
  p.weight = weight;
  p.out = static_cast<uint4*>(out);
  p.dweight = dweight;
  return launch(*s, p, kind, static_cast<cudaStream_t>(stream));
}

}  // namespace
}  // namespace erows
}  // namespace sky

using namespace sky;

extern "C" {

sky_status sky_dispatch_fwd(const sky_rows_shape* shape, const void* x, const int32_t* row, void* rows, void* stream) {
  ABI_GUARD_BEGIN
  return erows::run(shape, x, nullptr, row, nullptr, rows, nullptr, erows::DISPATCH, stream);
  ABI_GUARD_END
}

sky_status sky_dispatch_bwd(const sky_rows_shape* shape, const void* drows, const int32_t* row, void* dx, void* stream) {
  ABI_GUARD_BEGIN
  return erows::run(shape, drows, nullptr, row, nullptr, dx, nullptr, erows::ADD, stream);
  ABI_GUARD_END
}

sky_status sky_combine_fwd(const sky_rows_shape* shape, const void* rows, const int32_t* row, const float* weight, void* y,
                           void* stream) {
  ABI_GUARD_BEGIN
  return erows::run(shape, rows, nullptr, row, weight, y, nullptr, erows::ADD_WEIGHTED, stream);
  ABI_GUARD_END
}

sky_status sky_combine_bwd(const sky_rows_shape* shape, const void* rows, const void* dy, const int32_t* row,
                           const float* weight, void* drows, float* dweight, void* stream) {
  ABI_GUARD_BEGIN
  return erows::run(shape, rows, dy, row, weight, drows, dweight, erows::BACKWARD, stream);
  ABI_GUARD_END
}

}  // extern "C"
