// bf16 weight gradients grouped by expert where the tiles are few: the pairs of grouped_tc.cu would
// leave most SMs without work while a handful go through all rows of a group.
//
// A tile is 128 of `out` by up to 128 of `in`, by one CTA, and the rows of its group are split over
// the CTAs of a cluster, in blocks of 64.  As in grouped_tc.cu a tensor-core sum is over 512 rows and
// the parts are added in fp32, here in TMEM, and the rows of the next group that the last block
// brings with it are cleared in shared memory, in both operands.  Every CTA of a cluster owns a share
// of the tile's rows: the others send it their sums through distributed shared memory, and behind
// one cluster barrier it adds them in split order and stores them.
//   warp 0 TMA producer, and the clearing; warp 1 MMA issuer; warps 2..5 epilogue
//
// Bound, like those, by what an SM takes in, 32 KiB a block (0.3 us), twice as much a product as a
// pair's; then by a chain of some 6 us, launch to store.  16384 rows, one group of 512 x 512, 74 us by
// pairs and 25.0 here; 3967 rows of 128 x 104 24.5 and 8.2; 22 rows of 672 x 176 6.6 and 5.6.  Code is
// fetched once a launch, so little of it is unrolled: parts added in registers, 128 columns a thread,
// took 0.4 to 1.9 us more (16384 rows 26.8, 3769 rows of 160 x 80 over 38 groups 7.4 against 6.0).
#include <cuda.h>

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

constexpr int BM = 128, BN = 128, BK = 64, STAGES = 4;
constexpr int CHUNK_BYTES = 64 * BK * 2;  // one 64-wide MN-major box
constexpr int A_BYTES = 2 * CHUNK_BYTES, SBYTES = 2 * A_BYTES;
constexpr int PART_BLOCKS = 8;            // of a tensor-core sum
constexpr int COLUMNS = 512;              // TMEM: two accumulators and the sum of the parts before
constexpr int THREADS = 192;
constexpr int RECV_OFF = STAGES * SBYTES, BAR_OFF = RECV_OFF + BM * BN * 4;
constexpr int SMEM = BAR_OFF + 256 + 1024;
static_assert(SMEM + kSmemPerCta + std::min(kSplitAttentionSmem, kClusterProductSmem) + kSmemPerCta > kSmemPerSM,
              "see residency.h");

struct Params {
  const int32_t* offset;
  int groups, rows, out, in;
  int m_blocks, n_blocks, n_width, ks;  // n_width: of a tile, a multiple of 16
  float* C;
  int32_t* status;
  Fault fault;
};

__global__ void __launch_bounds__(THREADS, 1)
    grouped_grad_few_tc(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                        const __grid_constant__ Params p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = ptx::smem_u32(smem_raw);
  uint8_t* smem = smem_raw + (((raw_addr + 1023u) & ~1023u) - raw_addr);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + BAR_OFF);
  uint64_t* empty = full + STAGES;
  uint64_t* tfull = empty + STAGES;
  uint64_t* tempty = tfull + 2;
  uint64_t* here = tempty + 2;  // the block that has rows to clear has come
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(here + 1);
  // Set in every CTA of the cluster by one whose sums did not come: nothing is stored then.
  const uint32_t lost = ptx::smem_u32(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int split = static_cast<int>(blockIdx.x) % p.ks, u = static_cast<int>(blockIdx.x) / p.ks;
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      ptx::mbar_init(&full[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      ptx::mbar_init(&tfull[a], 1);
      ptx::mbar_init(&tempty[a], 4);
    }
    ptx::mbar_init(here, 1);
    ptx::st_shared_u32(lost, 0);
    ptx::fence_cluster();  // with the arrival below: before a peer writes it
    ptx::fence_mbar_init();
    ptx::fence_proxy_async_smem();
    ptx::prefetch_tensormap(&tmA);
    ptx::prefetch_tensormap(&tmB);
  }
  if (warp == 1) {
    ptx::tmem_alloc(tmem_slot, COLUMNS);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_wait();
  if (blockIdx.x == 0) check_offsets(p.offset, p.groups, p.rows, p.status);
  ptx::cluster_arrive();  // this CTA runs: its peers may write its shared memory
  const int per_group = p.m_blocks * p.n_blocks, group = u / per_group;
  const int m0 = u % per_group / p.n_blocks * BM, n0 = u % p.n_blocks * p.n_width;
  const int2 r = group_rows(p.offset, group, p.rows);
  const int blocks = (r.y - r.x + BK - 1) / BK;
  const int kb0 = static_cast<int>(static_cast<int64_t>(split) * blocks / p.ks);
  const int kb1 = static_cast<int>(static_cast<int64_t>(split + 1) * blocks / p.ks);

  if (warp == 0) {
    const bool issuer = ptx::elect_one();
    const uint32_t missing = p.fault.missing(split);
    const bool two_a = p.out - m0 > 64, two_b = p.n_width > 64;  // boxes
    const uint32_t bytes = (2 + (two_a ? 1 : 0) + (two_b ? 1 : 0)) * CHUNK_BYTES;
    int stage = 0, issued = 0;
    uint32_t phase = 0;
    bool last_here = false;
    for (int kb = kb0; kb < kb1; ++kb) {
      if (!__all_sync(0xffffffffu, ptx::mbar_wait(&empty[stage], phase ^ 1u, p.fault.wait_ns, p.status))) break;
      const int k0 = r.x + kb * BK, left = r.y - k0;
      const bool clear = left < BK && left % 16 != 0;  // (the last block only)
      uint8_t* sa = smem + stage * SBYTES;
      if (issuer) {
        uint64_t* bar = clear ? here : &full[stage];
        ptx::mbar_arrive_expect_tx(bar, bytes + missing);
        ptx::tma_load_2d(sa, &tmA, bar, m0, k0);
        if (two_a) ptx::tma_load_2d(sa + CHUNK_BYTES, &tmA, bar, m0 + 64, k0);
        ptx::tma_load_2d(sa + A_BYTES, &tmB, bar, n0, k0);
        if (two_b) ptx::tma_load_2d(sa + A_BYTES + CHUNK_BYTES, &tmB, bar, n0 + 64, k0);
      }
      __syncwarp();
      if (clear) {
        last_here = true;
        if (!__all_sync(0xffffffffu, ptx::mbar_wait(here, 0, p.fault.wait_ns, p.status))) break;
        const uint32_t to = ptx::smem_u32(sa) + left * 128;
        const int pieces = ((left + 15) / 16 * 16 - left) * 8;  // of 16 bytes, in a box
        for (int b = 0; b < 4; ++b)
          for (int i = lane; i < pieces; i += 32) ptx::st_shared_v4(to + b * CHUNK_BYTES + i * 16, 0, 0, 0, 0);
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&full[stage]);
      }
      ++issued;
      if (++stage == STAGES) { stage = 0; phase ^= 1u; }
    }
    const int n_tail = min(issued, STAGES);  // drain (bounded): the loads still in flight
    for (int i = 0; i < n_tail; ++i) {
      if (--stage < 0) { stage = STAGES - 1; phase ^= 1u; }
      ptx::mbar_wait(&full[stage], phase, p.fault.wait_ns, p.status);
    }
    if (last_here) ptx::mbar_wait(here, 0, p.fault.wait_ns, p.status);
  } else if (warp == 1) {
    const bool issuer = ptx::elect_one();
    const uint32_t idesc = ptx::idesc_bf16_f32(BM, 0, true, true) | static_cast<uint32_t>(p.n_width >> 3) << 17;
    const uint32_t s0 = ptx::smem_u32(smem);
    const uint64_t da = ptx::smem_desc_sw128(s0, CHUNK_BYTES, 1024);
    const uint64_t db = ptx::smem_desc_sw128(s0 + A_BYTES, CHUNK_BYTES, 1024);
    int stage = 0, acc = 0;
    uint32_t phase = 0, aphase = 0;
    bool good = true;
    int kb = kb0;
    for (; kb < kb1; ++kb) {
      const bool first = (kb - kb0) % PART_BLOCKS == 0;
      if (first) good = __all_sync(0xffffffffu, ptx::mbar_wait(&tempty[acc], aphase ^ 1u, p.fault.wait_ns, p.status));
      good = good && __all_sync(0xffffffffu, ptx::mbar_wait(&full[stage], phase, p.fault.wait_ns, p.status));
      if (!good) break;
      ptx::tc_fence_after();
      const int left = r.y - (r.x + kb * BK), steps = left < BK ? (left + 15) / 16 : BK / 16;
      const bool last = kb + 1 == kb1 || (kb + 1 - kb0) % PART_BLOCKS == 0;
      if (issuer) {
        const uint64_t off = static_cast<uint64_t>(stage * (SBYTES >> 4));
#pragma unroll
        for (int kk = 0; kk < BK / 16; ++kk)
          if (kk < steps)
            ptx::tc_mma_f16(tmem_base + acc * BN, da + off + kk * 128, db + off + kk * 128, idesc, !first || kk > 0);
        ptx::tc_commit(&empty[stage]);
        if (last) ptx::tc_commit(&tfull[acc]);
      }
      __syncwarp();
      if (last && ++acc == 2) { acc = 0; aphase ^= 1u; }
      if (++stage == STAGES) { stage = 0; phase ^= 1u; }
    }
    // The issued MMAs have to finish before TMEM is released: behind the barrier of the last
    // stage that they read.
    if (kb > kb0) {
      const int at = stage > 0 ? stage - 1 : STAGES - 1;
      ptx::mbar_wait(&empty[at], stage > 0 ? phase : phase ^ 1u, p.fault.wait_ns, p.status);
    }
  }
  // ------------------------------------------------------------------ epilogue
  const int own = BM / p.ks;  // rows of the tile that a CTA finishes
  const uint32_t recv = ptx::smem_u32(smem) + RECV_OFF;
  // 16 bytes (four columns from 4 j) of a row of the sums, 512 bytes a row
  const auto piece = [](int row, int j) { return static_cast<uint32_t>(row * 512 + ((j ^ (row & 7)) << 4)); };
  if (warp >= 2) {
    const int q = warp & 3, row = q * 32 + lane;  // TMEM lanes 32 q ..
    ptx::cluster_wait();                          // every peer runs
    const uint32_t to = ptx::mapa_shared(recv, row / own) + split * own * 512;
    const uint32_t base = tmem_base + (static_cast<uint32_t>(q * 32) << 16), run = base + 2 * BN;
    int acc = 0;
    uint32_t aphase = 0;
    bool ok = true;
    for (int kb = kb0; kb == kb0 || kb < kb1; kb += PART_BLOCKS) {
      const bool any = kb < kb1, last = kb + PART_BLOCKS >= kb1;
      if (any) ok = __all_sync(0xffffffffu, ptx::mbar_wait(&tfull[acc], aphase, p.fault.wait_ns, p.status));
      if (!ok) break;
      ptx::tc_fence_after();
#pragma unroll 1
      for (int c = 0; c < p.n_width; c += 16) {
        uint32_t v[16] = {}, before[16] = {};
        if (any) ptx::tmem_ld_32x32b_x16(base + acc * BN + c, v);
        if (kb > kb0) ptx::tmem_ld_32x32b_x16(run + c, before);
        ptx::tmem_ld_wait();
        if (kb > kb0) {
#pragma unroll
          for (int e = 0; e < 16; ++e) v[e] = __float_as_uint(__uint_as_float(before[e]) + __uint_as_float(v[e]));
        }
        if (!last) {
          ptx::tmem_st_32x32b_x16(run + c, v);
        } else if (m0 + row < p.out) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            ptx::st_cluster_v4(to + piece(row % own, c / 4 + j), v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        }
      }
      if (!last) {
        ptx::tmem_st_wait();
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&tempty[acc]);
      }
      if (++acc == 2) { acc = 0; aphase ^= 1u; }
    }
    if (!ok && lane < p.ks) ptx::st_cluster_u32(ptx::mapa_shared(lost, lane), 1);
  } else {
    ptx::cluster_wait();
  }
  pdl_trigger();
  ptx::tc_fence_before();
  __syncwarp();
  ptx::cluster_sync();  // every sum is where it is added
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem_base, COLUMNS);
  }
  if (ptx::ld_shared_u32(lost) != 0) return;
  const int first = m0 + split * own, width = min(p.n_width, p.in - n0) >> 2;  // columns in fours
  float* out = p.C + (static_cast<int64_t>(group) * p.out + first) * p.in + n0;
  for (int i = threadIdx.x; i < own * width; i += THREADS) {
    const int row = i / width, j = i % width;
    if (first + row >= p.out) break;
    uint32_t v[8][4];
#pragma unroll
    for (int s = 0; s < 8; ++s)
      if (s < p.ks) ptx::ld_shared_v4(recv + s * own * 512 + piece(row, j), v[s]);
    float4 sum = make_float4(__uint_as_float(v[0][0]), __uint_as_float(v[0][1]), __uint_as_float(v[0][2]),
                             __uint_as_float(v[0][3]));
#pragma unroll
    for (int s = 1; s < 8; ++s)
      if (s < p.ks) {
        sum.x += __uint_as_float(v[s][0]);
        sum.y += __uint_as_float(v[s][1]);
        sum.z += __uint_as_float(v[s][2]);
        sum.w += __uint_as_float(v[s][3]);
      }
    *reinterpret_cast<float4*>(out + static_cast<int64_t>(row) * p.in + 4 * j) = sum;
  }
}

}  // namespace

// As many CTAs a tile as have their rows and leave all clusters on the device at once (76, 36 and 15
// of them, less a few on some): a second round costs what the first does.  us at 2 / 4 / 8, one group of
// 128 inner columns, and by pairs: 14 tiles, 256 rows 6.4 6.4 7.0, 6.9; 512 rows 6.9 6.7 7.2, 7.9;
// 1024 rows 7.9 7.2 7.4, 10.0; 4096 rows 16.8 11.6 9.8, 22.5; 64 tiles, 64 rows 6.3 13.2 32, 6.3; 4096 rows
// 20.7 28 51, 24.1.
int grad_few_splits(const Call& c, int sms) {
  static OncePerDevice once;
  if (c.form != SKY_GEMM_XTW || allow_smem(once, grouped_grad_few_tc, SMEM) != cudaSuccess) return 1;
  static CountPerDevice count[3];
  const auto most = [&](int splits) {
    return clusters_at_once(count[splits / 4], grouped_grad_few_tc, splits, THREADS, SMEM, sms);
  };
  const int64_t units = static_cast<int64_t>(c.groups) * ceil_div(c.out, BM) * ceil_div(c.in, BN);
  const int rows = ceil_div(c.rows, c.groups);  // of a mean group
  if (rows >= 1024 && units <= most(8)) return 8;
  if (rows >= 512 && units <= most(4)) return 4;
  return units <= most(2) ? 2 : 1;
}

sky_status launch_grad_few(const Call& c, int splits, cudaStream_t st) {
  Params p{c.offset, c.groups, c.rows, c.out, c.in, ceil_div(c.out, BM), ceil_div(c.in, BN), 0, splits,
           static_cast<float*>(c.C), c.status, fault_of(splits)};
  p.n_width = ceil_div(ceil_div(c.in, p.n_blocks), 16) * 16;
  CUtensorMap ta, tb;
  const bool ok = gemm::make_map(&ta, c.A, c.rows, c.out, 64) && gemm::make_map(&tb, c.B, c.rows, c.in, 64);
  SKY_CHECK(ok, SKY_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d x %d x %d)", c.groups, c.out, c.in);
  const int ctas = c.groups * p.m_blocks * p.n_blocks * splits;
  const cudaError_t e = launch_pdl(grouped_grad_few_tc, dim3(ctas), dim3(THREADS), SMEM, st, splits, ta, tb, p);
  count_launches(1);
  return e == cudaSuccess ? SKY_OK : cuda_fail(e, "grouped weight gradient launch");
}

}  // namespace grouped
}  // namespace sky
