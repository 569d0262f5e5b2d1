// bf16 products grouped by expert for few rows (a decoder's new tokens): the weights of every
// group that has a row are read once, for a handful of tokens each, so HBM bounds them and what
// counts is that all SMs read at once and how soon.  And for few tiles with long sums, where the
// pairs of grouped_tc.cu would leave most SMs without work.
//
// As in grouped_tc.cu the weights are the M side: a tile is 128 features by up to 32 tokens of one
// group, by one CTA, and the sum may be split over the CTAs of a cluster.  Two CTAs an SM, each
// with four 20 KiB stages on the way.  With a split every CTA owns a share of the features: the
// others send it their partial sums through distributed shared memory, and behind one cluster
// barrier it adds them in split order and finishes.  One unit a CTA; how many there are is known
// on the device only, and those that are too many leave at once.
//   warp 0 TMA producer, warp 1 MMA issuer, warps 2..5 epilogue
#include <cuda.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "common.cuh"
#include "gemm.h"
#include "grouped.cuh"
#include "grouped.h"
#include "ptx.cuh"
#include "residency.h"

namespace sky {
namespace grouped {
namespace {

constexpr int BM = 128, BK = 64, TOKENS = 32, STAGES = 4;
constexpr int A_BYTES = BM * BK * 2, SBYTES = A_BYTES + TOKENS * BK * 2, CHUNK_BYTES = 64 * BK * 2;
constexpr int THREADS = 192;
constexpr int RECV_OFF = STAGES * SBYTES, RECV_BYTES = BM * TOKENS * 4;
constexpr int BAR_OFF = RECV_OFF + RECV_BYTES;
constexpr int SMEM = BAR_OFF + 256 + 1024;
static_assert(SMEM >= kClusterProductSmem, "see residency.h");
static_assert(2 * (SMEM + kSmemPerCta) <= kSmemPerSM, "two CTAs an SM");

struct Params {
  const int32_t* offset;
  int groups, rows, features;
  int f_blocks, k_blocks, ks;
  __nv_bfloat16* C;
  const __nv_bfloat16* bias;
  const __half* aux;
  __half* aux_out;
  int32_t* status;
  Fault fault;
};
struct Maps {
  CUtensorMap weights;
  CUtensorMap rows[2];  // boxes of 16 and 32 rows
};

template <bool W_MN, int EPI>
__global__ void __launch_bounds__(THREADS, 2) grouped_few_tc(const __grid_constant__ Maps maps, const __grid_constant__ Params p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = ptx::smem_u32(smem_raw);
  uint8_t* smem = smem_raw + (((raw_addr + 1023u) & ~1023u) - raw_addr);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + BAR_OFF);
  uint64_t* empty = full + STAGES;
  uint64_t* tfull = empty + STAGES;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tfull + 1);
  // Set in every CTA of the cluster by one whose accumulator did not come: nothing is stored then.
  const uint32_t lost = ptx::smem_u32(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int split = static_cast<int>(blockIdx.x) % p.ks, u = static_cast<int>(blockIdx.x) / p.ks;
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      ptx::mbar_init(&full[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    ptx::mbar_init(tfull, 1);
    ptx::st_shared_u32(lost, 0);
    ptx::fence_cluster();  // with the arrival below: before a peer writes it
    ptx::fence_mbar_init();
    ptx::fence_proxy_async_smem();
    ptx::prefetch_tensormap(&maps.weights);
  }
  if (warp == 1) {
    ptx::tmem_alloc(tmem_slot, TOKENS);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_wait();
  if (blockIdx.x == 0) check_offsets(p.offset, p.groups, p.rows, p.status);
  const Found at = find_tile(p.offset, p.groups, p.rows, u / p.f_blocks, [](int n) { return (n + TOKENS - 1) / TOKENS; });
  if (at.group < 0) {  // (every CTA of the cluster)
    if (warp == 1) ptx::tmem_dealloc(tmem_base, TOKENS);
    return;
  }
  if (p.ks > 1) ptx::cluster_arrive();  // this CTA runs: its peers may write its shared memory
  const int f0 = u % p.f_blocks * BM, row = at.lo + at.tile * TOKENS, count = min(TOKENS, at.hi - row);
  const int n_pad = (count + 15) & ~15;  // the N side
  const int kb0 = split * p.k_blocks / p.ks, kb1 = (split + 1) * p.k_blocks / p.ks;

  if (warp == 0) {
    const bool issuer = ptx::elect_one();
    const uint32_t missing = p.fault.missing(split);
    int stage = 0, issued = 0;
    uint32_t phase = 0;
    for (int kb = kb0; kb < kb1; ++kb) {
      if (!__all_sync(0xffffffffu, ptx::mbar_wait(&empty[stage], phase ^ 1u, p.fault.wait_ns, p.status))) break;
      if (issuer) {
        uint8_t* sa = smem + stage * SBYTES;
        ptx::mbar_arrive_expect_tx(&full[stage], A_BYTES + n_pad * BK * 2 + missing);
        const int k0 = kb * BK;
        if (W_MN) {
          ptx::tma_load_3d(sa, &maps.weights, &full[stage], f0, k0, at.group);
          ptx::tma_load_3d(sa + CHUNK_BYTES, &maps.weights, &full[stage], f0 + 64, k0, at.group);
        } else {
          ptx::tma_load_3d(sa, &maps.weights, &full[stage], k0, f0, at.group);
        }
        ptx::tma_load_2d(sa + A_BYTES, &maps.rows[n_pad / 16 - 1], &full[stage], k0, row);
      }
      __syncwarp();
      ++issued;
      if (++stage == STAGES) { stage = 0; phase ^= 1u; }
    }
    const int n_tail = min(issued, STAGES);  // drain (bounded): the loads still in flight
    for (int i = 0; i < n_tail; ++i) {
      if (--stage < 0) { stage = STAGES - 1; phase ^= 1u; }
      ptx::mbar_wait(&full[stage], phase, p.fault.wait_ns, p.status);
    }
  } else if (warp == 1) {
    const bool issuer = ptx::elect_one();
    const uint32_t idesc = ptx::idesc_bf16_f32(BM, 0, W_MN, false) | static_cast<uint32_t>(n_pad >> 3) << 17;
    const uint32_t s0 = ptx::smem_u32(smem);
    const uint64_t da = W_MN ? ptx::smem_desc_sw128(s0, CHUNK_BYTES, 1024) : ptx::smem_desc_sw128(s0, 16, 1024);
    const uint64_t db = ptx::smem_desc_sw128(s0 + A_BYTES, 16, 1024);
    int stage = 0;
    uint32_t phase = 0;
    bool good = true;
    int kb = kb0;
    for (; kb < kb1; ++kb) {
      good = __all_sync(0xffffffffu, ptx::mbar_wait(&full[stage], phase, p.fault.wait_ns, p.status));
      if (!good) break;
      ptx::tc_fence_after();
      if (issuer) {
        const uint64_t off = static_cast<uint64_t>(stage * (SBYTES >> 4));
#pragma unroll
        for (int kk = 0; kk < BK / 16; ++kk)
          ptx::tc_mma_f16(tmem_base, da + off + kk * (W_MN ? 128 : 2), db + off + kk * 2, idesc, kb > kb0 || kk > 0);
        ptx::tc_commit(&empty[stage]);
      }
      __syncwarp();
      if (++stage == STAGES) { stage = 0; phase ^= 1u; }
    }
    // The issued MMAs have to finish before TMEM is released; after a time-out they do so
    // behind the barrier of the stage before the one that did not come.
    if (good) {
      if (issuer) ptx::tc_commit(tfull);
      __syncwarp();
      ptx::mbar_wait(tfull, 0, p.fault.wait_ns, p.status);
    } else if (kb > kb0) {
      const int last = stage > 0 ? stage - 1 : STAGES - 1;
      ptx::mbar_wait(&empty[last], stage > 0 ? phase : phase ^ 1u, p.fault.wait_ns, p.status);
    }
  }
  // ------------------------------------------------------------------ epilogue
  const int q = warp & 3, own = BM / p.ks;  // TMEM lanes 32 q ..; features that a CTA finishes
  const uint32_t recv = ptx::smem_u32(smem) + RECV_OFF;
  // 16 bytes (four tokens from 4 j) of feature f of the partial sums, 128 bytes a feature
  const auto piece = [](int f, int j) { return static_cast<uint32_t>(f * 128 + ((j ^ (f & 7)) << 4)); };
  uint32_t r[32];
  if (warp >= 2) {
    const bool ok = __all_sync(0xffffffffu, ptx::mbar_wait(tfull, 0, p.fault.wait_ns, p.status));
    ptx::tc_fence_after();
    if (ok) {
      ptx::tmem_ld_32x32b_x32(tmem_base + (static_cast<uint32_t>(q * 32) << 16), r);
      ptx::tmem_ld_wait();
    }
    if (p.ks > 1) ptx::cluster_wait();  // every peer runs
    if (!ok && lane < p.ks) ptx::st_cluster_u32(p.ks > 1 ? ptx::mapa_shared(lost, lane) : lost, 1);
    if (ok) {
      const int f = q * 32 + lane;
      const uint32_t to = p.ks > 1 ? ptx::mapa_shared(recv, f / own) : recv;
#pragma unroll
      for (int j = 0; j < TOKENS / 4; ++j)
        if (4 * j < count)
          ptx::st_cluster_v4(to + split * own * 128 + piece(f % own, j), r[4 * j], r[4 * j + 1], r[4 * j + 2], r[4 * j + 3]);
    }
  } else if (p.ks > 1) {
    ptx::cluster_wait();
  }
  pdl_trigger();
  ptx::tc_fence_before();
  __syncwarp();
  if (p.ks > 1) ptx::cluster_sync();  // every partial sum is where it is added
  else __syncthreads();
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem_base, TOKENS);
  }
  if (warp < 2 || ptx::ld_shared_u32(lost) != 0) return;
  // Thread et takes feature et % own of the CTA's and every (128 / own)-th token: neighbours write
  // neighbouring features.
  const int et = static_cast<int>(threadIdx.x) - 64, fl = et % own, f = f0 + split * own + fl;
  if (f >= p.features) return;
  float bias = 0.f;
  if (EPI != SKY_EPI_GELU_BWD && p.bias) bias = __bfloat162float(p.bias[static_cast<int64_t>(at.group) * p.features + f]);
  for (int t = et / own; t < count; t += BM / own) {
    const int64_t off = static_cast<int64_t>(row + t) * p.features + f;
    float part[8];
#pragma unroll
    for (int s = 0; s < 8; ++s)
      part[s] = s < p.ks ? __uint_as_float(ptx::ld_shared_u32(recv + s * own * 128 + piece(fl, t >> 2) + (t & 3) * 4)) : 0.f;
    float v = part[0];
#pragma unroll
    for (int s = 1; s < 8; ++s) v += part[s];
    if constexpr (EPI == SKY_EPI_GELU_BWD) {
      v *= __half2float(p.aux[off]);
    } else {
      v += bias;
    }
    if constexpr (EPI == SKY_EPI_BIAS_GELU) {
      float2 g, gp;
      gelu_and_grad2(v, 0.f, g, gp);  // (one value a step; it is the weights that are waited for)
      v = g.x;
      p.aux_out[off] = __float2half_rn(gp.x);
    }
    p.C[off] = __float2bfloat16_rn(v);
  }
}

template <bool W_MN, int EPI>
cudaError_t launch_one(const Maps& maps, const Params& p, int64_t units, cudaStream_t st) {
  auto kern = grouped_few_tc<W_MN, EPI>;
  static OncePerDevice once;
  const cudaError_t attr = allow_smem(once, kern, SMEM);
  if (attr != cudaSuccess) return attr;
  return launch_pdl(kern, dim3(static_cast<unsigned>(units * p.ks)), dim3(THREADS), SMEM, st, p.ks, maps, p);
}

// Tiles of tokens that the rows may make.
int64_t tiles_of(const Call& c) { return c.rows / TOKENS + static_cast<int64_t>(std::min(c.groups, c.rows)); }

}  // namespace

// Where the tiles that the rows may make fit the SMs at once, two an SM, and up to 64 rows.  us of
// the pairs of grouped_tc.cu and here (best split), 8 groups of 4096 x 1024 with GELU: 1 row 6.6
// 4.2, 8 rows 14.5 12.9, 32 rows 15.3 14.6, 64 rows (over two an SM) 15.5 15.5; 1024 x 4096: 1 row
// 13.1 4.6, 8 rows 16.7 13.0, 64 rows 17.4 14.6, 256 rows 18.0 18.5; 768 x 768: 64 rows 5.3 4.7, 128
// rows 5.4 5.7; 64 groups of 768 x 768 (384 tiles), 64 rows 15.2 17.7.
// With more rows where the tiles leave room for splits and the sum is long enough for them: one
// group, 256 rows of 1024 x 1024 (72 tiles) 8.8 6.9, of 1024 x 4096 21.4 9.6, 1024 rows of 256 x 2048 (66)
// 13.0 7.6, of 1024 x 2048 (264) 13.1 14.1; 4 groups, 256 rows of 1024 x 1024 (96) 6.3 7.3, of 768 x 768 (72,
// 12 blocks) 5.7 6.4.
bool few_pays(const Call& c, int sms) {
  if (c.form == SKY_GEMM_XTW) return false;
  const bool xw = c.form == SKY_GEMM_XW;
  const int64_t units = tiles_of(c) * ceil_div(xw ? c.in : c.out, BM);
  return units <= (c.rows <= 64 ? 2 * sms : ceil_div(xw ? c.out : c.in, BK) >= 16 ? sms / 2 : 0);
}

sky_status launch_few(const Call& c, int sms, cudaStream_t st) {
  const bool xw = c.form == SKY_GEMM_XW;
  Params p{};
  p.offset = c.offset;
  p.groups = c.groups;
  p.rows = c.rows;
  p.features = xw ? c.in : c.out;
  const int k = xw ? c.out : c.in;
  p.f_blocks = ceil_div(p.features, BM);
  p.k_blocks = ceil_div(k, BK);
  p.C = static_cast<__nv_bfloat16*>(c.C);
  p.bias = static_cast<const __nv_bfloat16*>(c.bias);
  p.aux = static_cast<const __half*>(c.aux);
  p.aux_out = static_cast<__half*>(c.aux_out);
  p.status = c.status;
  const int64_t units = tiles_of(c) * p.f_blocks;
  // Splits: no more CTAs than two an SM, and three k-blocks or more each.  us at 1 / 2 / 4 / 8: 8
  // groups of 4096 x 1024, 2 rows (64 tiles) 5.7 4.9 5.2 8.9, 1024 x 4096, 2 rows (16) 13.9 8.8 6.0
  // 5.0, 8 rows (64) 20.5 14.9 13.0 16.9; 768 x 768, 8 rows (48) 5.0 4.4 4.3 7.4.
  p.ks = 1;
  while (p.ks < 8 && units * p.ks * 2 <= 2 * sms && p.k_blocks >= 6 * p.ks) p.ks *= 2;
  SKY_CHECK(units * p.ks <= 0x3fffffff, SKY_ERR_UNSUPPORTED, "grouped product too large");
  p.fault = fault_of(p.ks);
  Maps m;
  const bool ok = gemm::make_map_3d(&m.weights, c.B, c.groups, c.out, c.in, xw ? 64 : BM, 64, false) &&
                  gemm::make_map(&m.rows[0], c.A, c.rows, k, 16) && gemm::make_map(&m.rows[1], c.A, c.rows, k, 32);
  SKY_CHECK(ok, SKY_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d x %d x %d)", c.groups, c.out, c.in);
  cudaError_t e;
  if (!xw)
    e = c.epi == SKY_EPI_BIAS_GELU ? launch_one<false, SKY_EPI_BIAS_GELU>(m, p, units, st)
                                   : launch_one<false, SKY_EPI_STORE>(m, p, units, st);
  else
    e = c.epi == SKY_EPI_GELU_BWD ? launch_one<true, SKY_EPI_GELU_BWD>(m, p, units, st)
                                  : launch_one<true, SKY_EPI_STORE>(m, p, units, st);
  count_launches(1);
  return e == cudaSuccess ? SKY_OK : cuda_fail(e, "grouped product of few rows launch");
}

}  // namespace grouped
}  // namespace sky
