// Routing of tokens to experts (sky_experts.h): the top k logits of every token, their
// weights, and the plan that sorts the choices by expert, then by token.
//
// A warp holds a token's logits, expert lane + 32 j in lane's register j, as unsigned
// integers in the order of the numbers.  A choice is one warp reduction for the largest and
// one for the lowest index that has it.  Choosing is bound by the instructions issued, so up to
// 16 experts 16 or 8 lanes hold a token and a warp has two or four (16384 x 8 logits, two choices,
// us at 32 / 16 / 8 lanes: 9.1 7.1 5.7; 65536 x 8: 22.6 15.3 10.7).
//
// The sort is a counting sort over blocks of consecutive tokens.  A token chooses an expert
// at most once, so a block's choices of an expert are a bit mask over its tokens: the block's
// count is the mask's population, and a choice's rank the population below its token's bit.
// Setting bits needs no order, so the plan is deterministic.  The counts of all blocks go
// through the workspace, and a second launch adds up what lies before each block; up to
// SMALL tokens one CTA does everything in one launch.  At these sizes (8192 x 64 logits are
// 2 MB) all of it is latency: launches and the chain of reductions.
#include <algorithm>
#include <cmath>

#include "../../include/sky_experts.h"
#include "abi.h"
#include "common.cuh"

namespace sky {
namespace route {
namespace {

constexpr int MAX_EXPERTS = 1024, MAX_TOP_K = 32;
constexpr int THREADS = 256, WIDE = 1024, SMALL = 64;
constexpr int MOST_BLOCK = 256;     // tokens of a block
// Counts that every block adds up for itself (us so and scanned: 15000 counts 16.2 17.5, 20480 13.0 12.0).
constexpr int MOST_COUNTS = 16384;
constexpr int AT_ONCE = 4;          // of them that a thread waits for together
constexpr int32_t kStatusNaN = 4;

struct Params {
  int tokens, experts, top_k, block;  // block: tokens of one, a multiple of 32
  int blocks;
  bool over_all, scanned;
  const void* logits;
  int32_t* expert;
  float* weight;
  int32_t* row;
  int32_t* offset;
  int32_t* counts;  // [blocks][experts], and when scanned [experts] totals behind them
  int32_t* status;
};

// A logit's place in the order of numbers; 0 for NaN.  -0 counts as 0.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return x != x ? 0u : (b >> 31 ? ~b : b | 0x80000000u);
}
__device__ __forceinline__ float number_of(uint32_t o) {
  return __uint_as_float(o >> 31 ? o & 0x7fffffffu : ~o);
}
constexpr uint32_t LOWEST = 0x007fffffu;  // of -inf: nothing up to here is chosen

// exp(x - top), where equal infinities count as equal.
__device__ __forceinline__ float exp_below(float x, float top) { return x == top ? 1.f : expf(x - top); }

// A token's logits as they lie in a warp, or in one of its groups of lanes.
template <typename T, int V>
__device__ __forceinline__ void load_logits(const Params& p, int t, int lane, T (&x)[V]) {
  const T* row = static_cast<const T*>(p.logits) + static_cast<int64_t>(t) * p.experts;
#pragma unroll
  for (int j = 0; j < V; ++j)
    if (lane + 32 * j < p.experts) x[j] = row[lane + 32 * j];
}

// Over groups of G lanes.
template <int G>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
  if constexpr (G == 32) {
    return __reduce_max_sync(0xffffffffu, v);
  } else {
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
  }
}
template <int G>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// The choices of one token, by G lanes (32, or fewer where V is 1): lane c of them gets choice c.
// `there`: there is a token.  Every lane of the warp calls.
template <typename T, int V, int G>
__device__ __forceinline__ void choose(const Params& p, const T (&x)[V], int lane, bool there, int& mine, float& weight) {
  uint32_t key[V];
  bool nan = false;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const float f = there && lane + 32 * j < p.experts ? to_f32<T>(x[j]) : -INFINITY;
    nan |= f != f;
    key[j] = order_of(f);
  }
  if (nan && p.status) atomicOr(p.status, kStatusNaN);
  float all = 0.f, value = -INFINITY, top = 0.f;
  mine = -1;
  for (int c = 0; c < p.top_k; ++c) {
    uint32_t best = key[0];
#pragma unroll
    for (int j = 1; j < V; ++j) best = max(best, key[j]);
    best = group_max<G>(best);
    const bool some = best > LOWEST;  // the same in a group
    if (G == 32 ? !some : !__any_sync(0xffffffffu, some)) break;  // warp-uniform
    if (c == 0 && some) {
      top = number_of(best);
      if (p.over_all) {
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (key[j] > LOWEST) all += exp_below(number_of(key[j]), top);
      }
    }
    int at = MAX_EXPERTS;
    if constexpr (G == 32) {
#pragma unroll
      for (int j = V - 1; j >= 0; --j)
        if (key[j] == best) at = lane + 32 * j;
      at = __reduce_min_sync(0xffffffffu, at);
    } else {
      const uint32_t equal = __ballot_sync(0xffffffffu, key[0] == best) >> (threadIdx.x & 31 & ~(G - 1));
      at = __ffs(equal) - 1;
    }
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (at == lane + 32 * j) key[j] = 0;
    if (some && lane == c) {
      mine = at;
      value = number_of(best);
    }
  }
  const float e = mine >= 0 ? exp_below(value, top) : 0.f;
  const float total = group_sum<G>(p.over_all ? all : e);
  weight = mine >= 0 ? e / total : 0.f;
}

// Exclusive sums over the experts of what `total` holds, by a whole CTA: consecutive experts a
// thread, the warps' sums scanned by every warp for itself.
__device__ __forceinline__ void scan_experts(int* total, int experts, int* warp_sums) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  const int per = (experts + blockDim.x - 1) / blockDim.x;
  int own = 0;
  for (int i = 0; i < per; ++i)
    if (tid * per + i < experts) own += total[tid * per + i];
  const auto scan = [&](int v) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += up;
    }
    return v;
  };
  const int sum = scan(own);
  if (lane == 31) warp_sums[warp] = sum;
  __syncthreads();
  const int upto = scan(lane < warps ? warp_sums[lane] : 0);
  int before = sum - own + (warp > 0 ? __shfl_sync(0xffffffffu, upto, (warp + 31) & 31) : 0);
  for (int i = 0; i < per; ++i)
    if (tid * per + i < experts) {
      const int n = total[tid * per + i];
      total[tid * per + i] = before;
      before += n;
    }
  __syncthreads();
}

// The places of a block's choices, whose masks are set: base[e] + rank.
__device__ __forceinline__ void place_block(const Params& p, int t0, const uint32_t* mask, const int* base) {
  const int words = p.block / 32, n = min(p.block, p.tokens - t0) * p.top_k;
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const int64_t at = static_cast<int64_t>(t0) * p.top_k + i;
    const int e = p.expert[at], t = i / p.top_k;
    int place = -1;
    if (e >= 0) {
      place = base[e];
      for (int w = 0; w < t / 32; ++w) place += __popc(mask[e * words + w]);
      place += __popc(mask[e * words + t / 32] & ((1u << (t & 31)) - 1u));
    }
    p.row[at] = place;
  }
}

// Chooses for a block of tokens and sets its masks.
template <typename T, int V, int G>
__device__ __forceinline__ void choose_block(const Params& p, int t0, uint32_t* mask) {
  const int lane = threadIdx.x % G, words = p.block / 32;
  for (int i = threadIdx.x; i < p.experts * words; i += blockDim.x) mask[i] = 0;
  __syncthreads();
  const int last = min(p.block, p.tokens - t0), groups = blockDim.x / G;
  T x[V] = {}, next[V] = {};
  int t = threadIdx.x / G;
  if (t < last) load_logits<T, V>(p, t0 + t, lane, next);
  for (int first = (threadIdx.x >> 5) * (32 / G); first < last; first += groups, t += groups) {  // (a warp's first token)
    int e;
    float w;
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = next[j];
    if (t + groups < last) load_logits<T, V>(p, t0 + t + groups, lane, next);
    choose<T, V, G>(p, x, lane, t < last, e, w);
    if (t < last && lane < p.top_k) {
      const int64_t at = static_cast<int64_t>(t0 + t) * p.top_k + lane;
      p.expert[at] = e;
      p.weight[at] = w;
      if (e >= 0) atomicOr(&mask[e * words + t / 32], 1u << (t & 31));
    }
  }
  __syncthreads();
}

__device__ __forceinline__ int count_of(const uint32_t* mask, int e, int words) {
  int n = 0;
  for (int w = 0; w < words; ++w) n += __popc(mask[e * words + w]);
  return n;
}

// Threads where warps choose: with 32 experts a lane, half as many, whose keys take the registers.
constexpr int choosers(int v) { return v == 32 ? WIDE / 2 : WIDE; }

// Everything, for one block of tokens.
template <typename T, int V, int G>
__global__ void __launch_bounds__(choosers(V)) route_small(const Params p) {
  extern __shared__ uint32_t sm[];
  __shared__ int sums[32];
  uint32_t* mask = sm;
  int* base = reinterpret_cast<int*>(mask + p.experts * (p.block / 32));
  pdl_wait();
  pdl_trigger();
  choose_block<T, V, G>(p, 0, mask);
  for (int e = threadIdx.x; e < p.experts; e += blockDim.x) base[e] = count_of(mask, e, p.block / 32);
  __syncthreads();
  const int last = base[p.experts - 1];
  __syncthreads();
  scan_experts(base, p.experts, sums);
  for (int e = threadIdx.x; e < p.experts; e += blockDim.x) p.offset[e] = base[e];
  if (threadIdx.x == 0) p.offset[p.experts] = base[p.experts - 1] + last;
  place_block(p, 0, mask, base);  // (what it reads of p.expert this CTA wrote before a barrier)
}

template <typename T, int V, int G>
__global__ void __launch_bounds__(choosers(V)) route_choose(const Params p) {
  extern __shared__ uint32_t sm[];
  pdl_wait();
  pdl_trigger();
  choose_block<T, V, G>(p, blockIdx.x * p.block, sm);
  for (int e = threadIdx.x; e < p.experts; e += blockDim.x)
    p.counts[static_cast<int64_t>(blockIdx.x) * p.experts + e] = count_of(sm, e, p.block / 32);
}

// Many blocks: counts[b][e] becomes what the blocks before b have, the totals follow.  A warp
// takes an expert, 32 blocks at a time.
__global__ void __launch_bounds__(THREADS) route_scan(const Params p) {
  pdl_wait();
  pdl_trigger();
  const int e = blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (e >= p.experts) return;
  int before = 0;
  for (int b0 = 0; b0 < p.blocks; b0 += 32) {
    const int b = b0 + lane;
    int32_t* at = p.counts + static_cast<int64_t>(b) * p.experts + e;
    const int own = b < p.blocks ? *at : 0;
    int sum = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += up;
    }
    if (b < p.blocks) *at = before + sum - own;
    before += __shfl_sync(0xffffffffu, sum, 31);
  }
  if (lane == 0) p.counts[static_cast<int64_t>(p.blocks) * p.experts + e] = before;
}

__global__ void __launch_bounds__(WIDE) route_place(const Params p) {
  extern __shared__ uint32_t sm[];
  __shared__ int sums[WIDE / 32];
  const int words = p.block / 32, t0 = blockIdx.x * p.block;
  uint32_t* mask = sm;
  int* base = reinterpret_cast<int*>(mask + p.experts * words);  // totals, then starts
  int* before = base + p.experts;
  for (int i = threadIdx.x; i < p.experts * words; i += blockDim.x) mask[i] = 0;
  for (int e = threadIdx.x; e < p.experts; e += blockDim.x) base[e] = before[e] = 0;
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  const int n = min(p.block, p.tokens - t0) * p.top_k;
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const int e = p.expert[static_cast<int64_t>(t0) * p.top_k + i], t = i / p.top_k;
    if (e >= 0) atomicOr(&mask[e * words + t / 32], 1u << (t & 31));
  }
  if (p.scanned) {
    for (int e = threadIdx.x; e < p.experts; e += blockDim.x) {
      base[e] = p.counts[static_cast<int64_t>(p.blocks) * p.experts + e];
      before[e] = p.counts[static_cast<int64_t>(blockIdx.x) * p.experts + e];
    }
  } else {
    // thread (expert, part) adds up every parts-th block; whole numbers, so any order will do
    const int parts = max(1, static_cast<int>(blockDim.x) / p.experts);
    for (int i = threadIdx.x; i < p.experts * parts; i += blockDim.x) {
      const int e = i % p.experts;
      int total = 0, mine = 0;
      for (int b0 = i / p.experts; b0 < p.blocks; b0 += AT_ONCE * parts) {
        int c[AT_ONCE];  // on their way together, the last ones too
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) c[k] = b0 + k * parts < p.blocks ? p.counts[(b0 + k * parts) * p.experts + e] : 0;
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
          total += c[k];
          if (b0 + k * parts < static_cast<int>(blockIdx.x)) mine += c[k];
        }
      }
      if (total) atomicAdd(&base[e], total);
      if (mine) atomicAdd(&before[e], mine);
    }
  }
  __syncthreads();
  const int last = base[p.experts - 1];
  __syncthreads();
  scan_experts(base, p.experts, sums);
  if (blockIdx.x == 0) {
    for (int e = threadIdx.x; e < p.experts; e += blockDim.x) p.offset[e] = base[e];
    if (threadIdx.x == 0) p.offset[p.experts] = base[p.experts - 1] + last;
  }
  for (int e = threadIdx.x; e < p.experts; e += blockDim.x) before[e] += base[e];
  __syncthreads();
  place_block(p, t0, mask, before);
}

// dlogits of a token by a warp.
template <typename T, int V>
__global__ void __launch_bounds__(THREADS) route_backward(const Params p, const float* dweight, T* out) {
  const int lane = threadIdx.x & 31, t = blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5);
  pdl_wait();
  pdl_trigger();
  if (t >= p.tokens) return;
  const T* x = static_cast<const T*>(p.logits) + static_cast<int64_t>(t) * p.experts;
  const int64_t at = static_cast<int64_t>(t) * p.top_k + lane;
  const int mine = lane < p.top_k ? p.expert[at] : -1;
  const float dmine = lane < p.top_k ? dweight[at] : 0.f;
  float v[V], dw[V];
  uint32_t chosen = 0;  // bit j: expert lane + 32 j
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int e = lane + 32 * j;
    v[j] = e < p.experts ? to_f32<T>(x[e]) : -INFINITY;
    if (v[j] != v[j]) v[j] = -INFINITY;
    dw[j] = 0.f;
  }
  for (int c = 0; c < p.top_k; ++c) {
    const int e = __shfl_sync(0xffffffffu, mine, c);
    const float d = __shfl_sync(0xffffffffu, dmine, c);
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (e == lane + 32 * j) {
        chosen |= 1u << j;
        dw[j] += d;
      }
  }
  float top = -INFINITY;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    if (!p.over_all && !(chosen >> j & 1)) v[j] = -INFINITY;
    top = fmaxf(top, v[j]);
  }
  top = warp_max(top);
  float total = 0.f, mean = 0.f;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    v[j] = v[j] > -INFINITY ? exp_below(v[j], top) : 0.f;
    total += v[j];
    if (chosen >> j & 1) mean += v[j] * dw[j];
  }
  total = warp_sum(total);
  mean = warp_sum(mean);
  const float inv = total > 0.f ? 1.f / total : 0.f;
  mean *= inv;
  T* y = out + static_cast<int64_t>(t) * p.experts;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int e = lane + 32 * j;
    const float pr = v[j] * inv;
    if (e < p.experts) y[e] = from_f32<T>(pr == 0.f ? 0.f : pr * ((chosen >> j & 1 ? dw[j] : 0.f) - mean));
  }
}

sky_status check(const sky_route_shape* s) {
  SKY_CHECK(s, SKY_ERR_INVALID_ARG, "null shape");
  SKY_CHECK(s->tokens > 0 && s->experts > 0 && s->top_k > 0 && s->top_k <= s->experts, SKY_ERR_INVALID_ARG, "bad sizes");
  SKY_CHECK(s->dtype == SKY_DTYPE_BF16 || s->dtype == SKY_DTYPE_FP32, SKY_ERR_INVALID_ARG, "unknown dtype");
  SKY_CHECK(s->weights == SKY_ROUTE_OVER_ALL || s->weights == SKY_ROUTE_OVER_CHOSEN, SKY_ERR_INVALID_ARG,
            "unknown kind of weights");
  SKY_CHECK(s->experts <= MAX_EXPERTS && s->top_k <= MAX_TOP_K, SKY_ERR_UNSUPPORTED,
            "routing to more than %d experts or of more than %d choices", MAX_EXPERTS, MAX_TOP_K);
  SKY_CHECK(static_cast<int64_t>(s->tokens) * s->experts < (int64_t{1} << 31) &&
                static_cast<int64_t>(s->tokens) * s->top_k < (int64_t{1} << 31),
            SKY_ERR_UNSUPPORTED, "routing of 2^31 logits or choices or more");
  return SKY_OK;
}

bool on(const void* p, size_t grid) { return reinterpret_cast<uintptr_t>(p) % grid == 0; }

// Tokens of a block: 32, or what keeps the blocks to 128 or fewer, each of which adds up the counts
// of all (8192 x 64 logits, four choices, us at up to 64 / 128 / 256 blocks: 11.0 8.2 10.3; 4495 x 190,
// six, 20.4 13.5 12.5).
int block_of(int tokens) {
  int b = 32;
  while (b < MOST_BLOCK && ceil_div(tokens, b) > 128) b *= 2;
  return b;
}

size_t workspace(const sky_route_shape& s) {
  if (s.tokens <= SMALL) return 16;
  return (static_cast<size_t>(ceil_div(s.tokens, block_of(s.tokens))) + 1) * s.experts * sizeof(int32_t);
}

// How a token's experts lie: V a lane, over G lanes.
template <int V_, int G_>
struct Lie {
  static constexpr int V = V_, G = G_;
};
// Up to 16 experts several tokens share a warp.
template <typename F>
auto by_experts(int experts, F&& f) {
  if (experts <= 8) return f(Lie<1, 8>());
  if (experts <= 16) return f(Lie<1, 16>());
  if (experts <= 32) return f(Lie<1, 32>());
  if (experts <= 64) return f(Lie<2, 32>());
  if (experts <= 128) return f(Lie<4, 32>());
  if (experts <= 256) return f(Lie<8, 32>());
  return f(Lie<32, 32>());
}

template <typename T>
sky_status forward(Params p, cudaStream_t st) {
  cudaError_t e;
  if (p.tokens <= SMALL) {
    p.block = ceil_div(p.tokens, 32) * 32;
    p.blocks = 1;
    const size_t smem = static_cast<size_t>(p.experts) * (p.block / 32 + 1) * 4;
    e = by_experts(p.experts, [&](auto lie) {
      using L = decltype(lie);
      const int threads = std::min(choosers(L::V), 32 * p.tokens);
      return launch_pdl(route_small<T, L::V, L::G>, dim3(1), dim3(threads), smem, st, 1, p);
    });
    count_launches(1);
    return e == cudaSuccess ? SKY_OK : cuda_fail(e, "routing launch");
  }
  p.block = block_of(p.tokens);
  p.blocks = ceil_div(p.tokens, p.block);
  p.scanned = static_cast<int64_t>(p.blocks) * p.experts > MOST_COUNTS;
  const size_t masks = static_cast<size_t>(p.experts) * (p.block / 32) * 4;  // up to 32 KiB
  const size_t starts = 2 * p.experts * 4;
  // (As much shared memory as route_place, whose CTAs come while these run: where the two would make an
  // SM divide its first-level memory differently, 16384 x 128 logits, six choices, 27.0 us for 16.3.)
  e = by_experts(p.experts, [&](auto lie) {
    using L = decltype(lie);
    return launch_pdl(route_choose<T, L::V, L::G>, dim3(p.blocks), dim3(choosers(L::V)),
                      masks + starts + sizeof(int) * WIDE / 32, st, 1, p);
  });
  count_launches(1);
  if (e == cudaSuccess && p.scanned) {
    e = launch_pdl(route_scan, dim3(ceil_div(p.experts, THREADS / 32)), dim3(THREADS), 0, st, 1, p);
    count_launches(1);
  }
  if (e == cudaSuccess) {
    e = launch_pdl(route_place, dim3(p.blocks), dim3(WIDE), masks + starts, st, 1, p);
    count_launches(1);
  }
  return e == cudaSuccess ? SKY_OK : cuda_fail(e, "routing launch");
}

template <typename T>
sky_status backward(const Params& p, const float* dweight, void* dlogits, cudaStream_t st) {
  const cudaError_t e = by_experts(p.experts, [&](auto lie) {
    return launch_pdl(route_backward<T, decltype(lie)::V>, dim3(ceil_div(p.tokens, THREADS / 32)), dim3(THREADS), 0, st,
                      1, p, dweight, static_cast<T*>(dlogits));
  });
  count_launches(1);
  return e == cudaSuccess ? SKY_OK : cuda_fail(e, "routing backward launch");
}

Params params(const sky_route_shape& s, const void* logits, int32_t* expert) {
  Params p{};
  p.tokens = s.tokens; p.experts = s.experts; p.top_k = s.top_k;
  p.over_all = s.weights == SKY_ROUTE_OVER_ALL;
  p.logits = logits;
  p.expert = expert;
  return p;
}

}  // namespace
}  // namespace route
}  // namespace sky

using namespace sky;

extern "C" {

size_t sky_route_workspace_bytes(const sky_route_shape* shape) {
  return shape && route::check(shape) == SKY_OK ? route::workspace(*shape) : 0;
}

sky_status sky_route_fwd(const sky_route_shape* shape, const void* logits, int32_t* expert, float* weight, int32_t* row,
                         int32_t* offset, void* workspace, size_t workspace_bytes, int32_t* d_status, void* stream) {
  ABI_GUARD_BEGIN
  const sky_status ok = route::check(shape);
  if (ok != SKY_OK) return ok;
  SKY_CHECK(logits && expert && weight && row && offset && workspace, SKY_ERR_INVALID_ARG, "null argument");
  SKY_CHECK(route::on(logits, shape->dtype == SKY_DTYPE_BF16 ? 2 : 4) && route::on(expert, 4) && route::on(weight, 4) &&
                route::on(row, 4) && route::on(offset, 4) && route::on(workspace, 4) && route::on(d_status, 4),
            SKY_ERR_INVALID_ARG, "a pointer off its type's grid");
  SKY_CHECK(workspace_bytes >= route::workspace(*shape), SKY_ERR_INVALID_ARG, "workspace too small");
  route::Params p = route::params(*shape, logits, expert);
  p.weight = weight;
  p.row = row;
  p.offset = offset;
  p.counts = static_cast<int32_t*>(workspace);
  p.status = d_status;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return shape->dtype == SKY_DTYPE_BF16 ? route::forward<__nv_bfloat16>(p, st) : route::forward<float>(p, st);
  ABI_GUARD_END
}

sky_status sky_route_bwd(const sky_route_shape* shape, const void* logits, const int32_t* expert, const float* dweight,
                         void* dlogits, void* stream) {
  ABI_GUARD_BEGIN
  const sky_status ok = route::check(shape);
  if (ok != SKY_OK) return ok;
  SKY_CHECK(logits && expert && dweight && dlogits, SKY_ERR_INVALID_ARG, "null argument");
  const size_t g = shape->dtype == SKY_DTYPE_BF16 ? 2 : 4;
  SKY_CHECK(route::on(logits, g) && route::on(dlogits, g) && route::on(expert, 4) && route::on(dweight, 4),
            SKY_ERR_INVALID_ARG, "a pointer off its type's grid");
  const route::Params p = route::params(*shape, logits, const_cast<int32_t*>(expert));
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return shape->dtype == SKY_DTYPE_BF16 ? route::backward<__nv_bfloat16>(p, dweight, dlogits, st)
                                        : route::backward<float>(p, dweight, dlogits, st);
  ABI_GUARD_END
}

}  // extern "C"
