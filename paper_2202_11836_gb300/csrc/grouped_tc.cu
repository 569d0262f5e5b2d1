// bf16 products grouped by expert on the 5th-generation tensor cores.
//
// XWT and XW (the forward and the data gradient) are computed transposed: a tile has 256
// features of the weights as its M side, on a pair of SMs (cta_group::2), and up to 256 tokens of
// one group as its N side.  N is free in steps of 32, so a group of any size is cut into equal
// tiles that are at most 31 rows too wide, where 256-row tiles on the M side would compute half a
// tile for nothing per group on average.  Rows of the next group that a tile's loads pick up only
// reach columns that are not stored.
//   warp 0      TMA producer into a ring of 64-deep stages (weights 128 rows a CTA, half of the
//               tile's tokens a CTA, in the smallest box of 16, 32, 64 or 128 rows that has them)
//   warp 1      MMA issuer of the pair's leader; two accumulators of 256 TMEM columns
//   warps 2..9  epilogue: features are TMEM lanes and tokens columns, so a row of the output
//               lies across lanes.  16x256b loads put it into the layout of an mma.sync
//               accumulator, whose 16-bit pairs stmatrix writes transposed: 32 tokens by 32
//               features in shared memory, which TMA stores.
// XTW (weight gradients; grouped_grad_few.cu has those of few tiles) sums over the rows of a group:
// 256 x 256 tiles on a pair, K the rows in blocks of 64.  The last block's steps of 16 may reach into the next group's rows; there a warp
// clears them in shared memory between the copy and the product, in both operands, since what
// they hold may be anything.
// The groups' sizes are on the device only: every warp finds its next tile from the offsets
// itself, 32 groups at a time (grouped.cuh).
//
// What bounds them: a 256 x 256 tile on a pair takes 64 bytes a clock and SM of operands at the
// tensor cores' full rate, which is what an SM takes in, and what it sends out competes with that.
// 16384 rows, 8 groups of 4096 x 1024, a few calls: stored as it is 80 us (1.7 PFLOP/s), bias and
// GELU with their two outputs 100, a gradient through GELU' 90, weight gradients (134 MB out) 91; without
// their stores the second and the last take 83 and 79.  Kept up for a second the power cap takes 13%
// more.  Stores of the GELU tile, us, with a GELU of fewer terms that takes one less: 64 bytes of a row by
// lanes 118, four bytes a lane 121, by TMA from a buffer a warp 102, from two 98, from two that two warps
// share (128 bytes a row) 109, from two for one output at a time 105; sixteen warps 111.  Weight gradients
// by TMA in rows of 128 bytes 91, of 64 bytes 100, by lanes 94.  Two pairs of a cluster that load their
// shared operand once (multicast): 80, 100, 90 and 98, since clusters of four leave eight SMs without work.
#include <cuda.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "common.cuh"
#include "gemm.h"
#include "grouped.cuh"
#include "grouped.h"
#include "ptx.cuh"

namespace sky {
namespace grouped {
namespace {

constexpr int BM = 128, BK = 64;             // of a CTA: features; K of a stage
constexpr int TILE_M = 2 * BM, TILE_N = 256; // of a pair
constexpr int A_BYTES = BM * BK * 2, B_BYTES = TILE_N / 2 * BK * 2, SBYTES = A_BYTES + B_BYTES;
constexpr int CHUNK_BYTES = 64 * BK * 2;     // one 64-wide MN-major box
constexpr uint32_t SLEEP_NS = 20000;         // suspend hint of the epilogue's accumulator wait

// Launch shape of XWT and XW: eight epilogue warps, each with two staging buffers of 32 x 32 16-bit
// values (of GELU's two outputs: two pairs, for a stage less).
template <int EPI>
struct Shape {
  static constexpr bool GELU = EPI == SKY_EPI_BIAS_GELU;
  static constexpr int EW = 8, STAGES = GELU ? 5 : 6;
  static constexpr int BUFFER = GELU ? 4096 : 2048, STAGING = 2 * BUFFER;  // of an epilogue warp
  static constexpr int THREADS = 64 + 32 * EW;
  static constexpr int EPI_OFF = STAGES * SBYTES;
  static constexpr int BAR_OFF = EPI_OFF + EW * STAGING;
  static constexpr int SMEM = BAR_OFF + 256 + 1024;
  static_assert(SMEM <= 232448, "shared memory per CTA");
};
// Weight gradients: eight epilogue warps with a box of 32 rows by 32 fp32 each, and the
// clearing warp.
struct GradShape {
  static constexpr int EW = 8, STAGES = 6, STAGING = 4096;
  static constexpr int THREADS = 96 + 32 * EW;
  static constexpr int EPI_OFF = STAGES * SBYTES;
  static constexpr int BAR_OFF = EPI_OFF + EW * STAGING;
  static constexpr int SMEM = BAR_OFF + 512 + 1024;
  static_assert(SMEM <= 232448, "shared memory per CTA");
};

struct Params {
  const int32_t* offset;
  int groups, rows;
  int features, k;         // of a row of the output; of the sum
  int f_blocks, k_blocks;  // 256 features; 64 of the sum
  __nv_bfloat16* C;
  const __nv_bfloat16* bias;
  const __half* aux;
  __half* aux_out;
  int32_t* status;
  Fault fault;
};
struct Maps {
  CUtensorMap weights, C, aux_out;
  CUtensorMap rows[4];  // boxes of 16, 32, 64 and 128 rows
};

struct Tile {
  int group, row, count;  // first row, rows
};

// Finds tiles in ascending order; every lane of a warp calls it.
struct Walk {
  const int32_t* offset;
  int groups, rows, g0 = 0, before = 0, total = 0;
  int lo = 0, hi = 0, n = 0, upto = 0;  // of group g0 + lane
  __device__ __forceinline__ Walk(const int32_t* o, int g, int r) : offset(o), groups(g), rows(r) { load(); }
  __device__ __forceinline__ void load() {
    const int lane = threadIdx.x & 31;
    int2 r = make_int2(0, 0);
    if (g0 + lane < groups) r = group_rows(offset, g0 + lane, rows);
    lo = r.x;
    hi = r.y;
    upto = n = (hi - lo + TILE_N - 1) / TILE_N;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += up;
    }
    total = __shfl_sync(0xffffffffu, upto, 31);
  }
  // The j-th tile of tokens; false behind the last.
  __device__ __forceinline__ bool find(int j, Tile& t) {
    while (j >= before + total) {
      before += total;
      g0 += 32;
      if (g0 >= groups) return false;
      load();
    }
    const uint32_t past = __ballot_sync(0xffffffffu, j - before < upto);
    const int at = __ffs(past) - 1;
    const int a = __shfl_sync(0xffffffffu, lo, at), b = __shfl_sync(0xffffffffu, hi, at);
    const int tiles = __shfl_sync(0xffffffffu, n, at), tile = j - before - __shfl_sync(0xffffffffu, upto - n, at);
    const int each = ((b - a + tiles - 1) / tiles + 31) & ~31;  // equal tiles; at most TILE_N
    t.group = g0 + at;
    t.row = a + tile * each;
    t.count = min(each, b - t.row);
    return true;
  }
};

template <bool W_MN, int EPI>
__global__ void __launch_bounds__(Shape<EPI>::THREADS, 1)
    grouped_rows_tc(const __grid_constant__ Maps maps, const __grid_constant__ Params p) {
  using SH = Shape<EPI>;
  constexpr int NST = SH::STAGES, EW = SH::EW;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = ptx::smem_u32(smem_raw);
  uint8_t* smem = smem_raw + (((raw_addr + 1023u) & ~1023u) - raw_addr);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + SH::BAR_OFF);
  uint64_t* empty = full + NST;
  uint64_t* tfull = empty + NST;
  uint64_t* tempty = tfull + 2;
  uint64_t* done = tempty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = ptx::cluster_ctarank();
  const bool leader = rank == 0;
  const int cid = blockIdx.x >> 1, ncl = gridDim.x >> 1;
  if (threadIdx.x == 0) {
    for (int s = 0; s < NST; ++s) {
      ptx::mbar_init(&full[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      ptx::mbar_init(&tfull[a], 1);
      ptx::mbar_init(&tempty[a], 2 * EW);
    }
    ptx::mbar_init(done, 1);
    ptx::fence_mbar_init_cluster();
    ptx::fence_proxy_async_smem();
    ptx::prefetch_tensormap(&maps.weights);
  }
  if (warp == 1) {
    ptx::tmem_alloc_pair(tmem_slot, 512);
    ptx::tmem_relinquish_pair();
  }
  ptx::tc_fence_before();
  __syncwarp();
  ptx::cluster_sync();
  ptx::tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_wait();
  if (blockIdx.x == 0) check_offsets(p.offset, p.groups, p.rows, p.status);

  Walk walk(p.offset, p.groups, p.rows);
  Tile t;
  if (warp == 0) {
    const bool issuer = ptx::elect_one();
    int stage = 0, issued = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int u = cid; ok && walk.find(u / p.f_blocks, t); u += ncl) {
      const int f0 = u % p.f_blocks * TILE_M + static_cast<int>(rank) * BM;
      const int half = ((t.count + 31) & ~31) / 2;  // tokens whose rows this CTA loads
      const int box = half <= 16 ? 0 : half <= 32 ? 1 : half <= 64 ? 2 : 3;
      const uint32_t bytes = 2 * (A_BYTES + (16 << box) * BK * 2) + p.fault.missing(0);
      const int r0 = t.row + static_cast<int>(rank) * half;
      for (int kb = 0; kb < p.k_blocks; ++kb) {
        ok = __all_sync(0xffffffffu, ptx::mbar_wait(&empty[stage], phase ^ 1u, p.fault.wait_ns, p.status));
        if (!ok) break;
        if (issuer) {
          uint8_t* sa = smem + stage * SBYTES;
          if (leader) ptx::mbar_arrive_expect_tx(&full[stage], bytes);
          const uint32_t bar = ptx::mapa_shared(ptx::smem_u32(&full[stage]), 0);
          const int k0 = kb * BK;
          if (W_MN) {
            ptx::tma_load_3d_pair(sa, &maps.weights, bar, f0, k0, t.group);
            ptx::tma_load_3d_pair(sa + CHUNK_BYTES, &maps.weights, bar, f0 + 64, k0, t.group);
          } else {
            ptx::tma_load_3d_pair(sa, &maps.weights, bar, k0, f0, t.group);
          }
          ptx::tma_load_2d_pair(sa + A_BYTES, &maps.rows[box], bar, k0, r0);
        }
        __syncwarp();
        ++issued;
        if (++stage == NST) { stage = 0; phase ^= 1u; }
      }
    }
    // drain (bounded): the loads still in flight, counted on the leader's barriers
    const int n_tail = leader ? min(issued, NST) : 0;
    for (int i = 0; i < n_tail; ++i) {
      if (--stage < 0) { stage = NST - 1; phase ^= 1u; }
      ptx::mbar_wait(&full[stage], phase, p.fault.wait_ns, p.status);
    }
  } else if (warp == 1) {
    // the whole warp walks, so that descriptors stay warp-uniform, and one lane issues
    if (leader) {
      const bool issuer = ptx::elect_one();
      const uint32_t s0 = ptx::smem_u32(smem);
      const uint64_t da = W_MN ? ptx::smem_desc_sw128(s0, CHUNK_BYTES, 1024) : ptx::smem_desc_sw128(s0, 16, 1024);
      const uint64_t db = ptx::smem_desc_sw128(s0 + A_BYTES, 16, 1024);
      int stage = 0, acc = 0;
      uint32_t phase = 0, aphase = 0;
      bool ok = true;
      for (int u = cid; ok && walk.find(u / p.f_blocks, t); u += ncl) {
        const uint32_t idesc =
            ptx::idesc_bf16_f32(TILE_M, 0, W_MN, false) | static_cast<uint32_t>(((t.count + 31) & ~31) >> 3) << 17;
        if (!__all_sync(0xffffffffu, ptx::mbar_wait_cluster(&tempty[acc], aphase ^ 1u, p.fault.wait_ns, p.status))) break;
        ptx::tc_fence_after();
        const uint32_t d_tmem = tmem_base + acc * TILE_N;
        for (int kb = 0; kb < p.k_blocks; ++kb) {
          ok = __all_sync(0xffffffffu, ptx::mbar_wait(&full[stage], phase, p.fault.wait_ns, p.status));
          if (!ok) break;
          ptx::tc_fence_after();
          if (issuer) {
            const uint64_t off = static_cast<uint64_t>(stage * (SBYTES >> 4));
#pragma unroll
            for (int kk = 0; kk < BK / 16; ++kk)
              ptx::tc_mma_f16_pair(d_tmem, da + off + kk * (W_MN ? 128 : 2), db + off + kk * 2, idesc, kb > 0 || kk > 0);
            ptx::tc_commit_pair(&empty[stage], 3);
          }
          __syncwarp();
          if (++stage == NST) { stage = 0; phase ^= 1u; }
        }
        if (!ok) break;
        if (issuer) ptx::tc_commit_pair(&tfull[acc], 3);
        __syncwarp();
        if (++acc == 2) { acc = 0; aphase ^= 1u; }
      }
      // All issued MMAs must finish before TMEM is released.
      if (issuer) ptx::tc_commit_pair(done, 1);
      __syncwarp();
      ptx::mbar_wait(done, 0, p.fault.wait_ns, p.status);
    }
  } else {
    // Warp w has TMEM lanes 32 q .. (features) and every (EW / 4)-th chunk of 32 tokens.  One lane
    // hands the accumulator back once the last chunk is in registers.
    constexpr int PARTS = EW / 4, CHUNKS = TILE_N / 32 / PARTS;
    const int q = warp & 3, part = (warp - 2) >> 2;
    uint8_t* const staging = smem + SH::EPI_OFF + (warp - 2) * SH::STAGING;
    // 16-byte piece i of token row t of a staging buffer: 64 bytes a row, swizzled as TMA wants it
    const auto piece_at = [](uint32_t buffer, int t, int i) { return buffer + t * 64 + ((i ^ ((t >> 1) & 3)) << 4); };
    const int t_at = lane >> 2, f_lane = (lane & 3) * 8;  // where rows are moved by lanes: token of eight, features
    int turn = 0;  // staging buffer
    int acc = 0;
    uint32_t aphase = 0;
    // the tile that comes, and its bias at features lane / 4 + 8 i, one tile ahead
    Tile next;
    float next_bias[4] = {};
    const auto look = [&](int u) {
      if (!walk.find(u / p.f_blocks, next)) return false;
      if (EPI != SKY_EPI_GELU_BWD && p.bias) {
        const int f0 = u % p.f_blocks * TILE_M + static_cast<int>(rank) * BM + q * 32 + (lane >> 2);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          next_bias[i] = f0 + 8 * i < p.features
                             ? __bfloat162float(p.bias[static_cast<int64_t>(next.group) * p.features + f0 + 8 * i]) : 0.f;
      }
      return true;
    };
    bool more = look(cid);
    for (int u = cid; more; u += ncl) {
      t = next;
      float bias[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) bias[i] = next_bias[i];
      const int f0 = u % p.f_blocks * TILE_M + static_cast<int>(rank) * BM + q * 32, f_at = f0 + f_lane;
      const bool f_ok = f_at < p.features;
      uint4 pre[EPI == SKY_EPI_GELU_BWD ? CHUNKS : 1][4];
      if constexpr (EPI == SKY_EPI_GELU_BWD) {  // the tile's GELU', before the accumulator is waited for
#pragma unroll
        for (int cc = 0; cc < CHUNKS; ++cc)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int n = (cc * PARTS + part) * 32 + 8 * i + t_at;
            pre[cc][i] = f_ok && n < t.count ? __ldg(reinterpret_cast<const uint4*>(
                                                   p.aux + static_cast<int64_t>(t.row + n) * p.features + f_at))
                                             : make_uint4(0u, 0u, 0u, 0u);
          }
      }
      more = look(u + ncl);
      if (EPI == SKY_EPI_GELU_BWD && more) {  // the next tile's, on its way into L2
        const int f = (u + ncl) % p.f_blocks * TILE_M + static_cast<int>(rank) * BM + q * 32;
#pragma unroll
        for (int cc = 0; cc < CHUNKS; ++cc) {
          const int n = (cc * PARTS + part) * 32 + lane;
          if (f < p.features && n < next.count) ptx::prefetch_l2(p.aux + static_cast<int64_t>(next.row + n) * p.features + f);
        }
      }
      if (!__all_sync(0xffffffffu, ptx::mbar_wait(&tfull[acc], aphase, p.fault.wait_ns, p.status, SLEEP_NS))) break;
      ptx::tc_fence_after();
      const uint32_t taddr = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + acc * TILE_N;
      // of a chunk's 8 tokens b: r[4 b ..] features lane / 4 and + 8, r[16 + 4 b ..] + 16 and + 24;
      // a chunk ahead
      uint32_t r[2][32];
      const auto load = [&](int cc) {
        const int t0 = (cc * PARTS + part) * 32;
        if (t0 >= t.count) return;  // warp-uniform
        ptx::tmem_ld_16x256b_x4(taddr + t0, r[cc & 1]);
        ptx::tmem_ld_16x256b_x4(taddr + t0 + (16u << 16), r[cc & 1] + 16);
      };
      load(0);
#pragma unroll
      for (int cc = 0; cc < CHUNKS; ++cc) {
        const int t0 = (cc * PARTS + part) * 32;
        ptx::tmem_ld_wait();
        if (cc + 1 < CHUNKS) {
          load(cc + 1);
        } else {  // the accumulator is in registers
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive_cluster_relaxed(ptx::mapa_shared(ptx::smem_u32(&tempty[acc]), 0));
          if (++acc == 2) { acc = 0; aphase ^= 1u; }
        }
        if (t0 >= t.count) continue;
        uint8_t* const box = staging + turn * SH::BUFFER;
        const uint32_t buffer = ptx::smem_u32(box);
        if (lane == 0) ptx::bulk_wait_group_read<1>();  // what was stored from here has left it
        __syncwarp();
        uint32_t sl[4][4];  // GELU' in the accumulator's layout
        if constexpr (EPI == SKY_EPI_GELU_BWD) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            ptx::st_shared_v4(piece_at(buffer, 8 * i + t_at, lane & 3), pre[cc][i].x, pre[cc][i].y, pre[cc][i].z, pre[cc][i].w);
          __syncwarp();
#pragma unroll
          for (int b = 0; b < 4; ++b) ptx::ldmatrix_x4_trans(piece_at(buffer, 8 * b + (lane & 7), lane >> 3), sl[b]);
          __syncwarp();
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          uint32_t o[4], x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int at = (i >> 1) * 16 + 4 * b + (i & 1) * 2;
            float v0 = __uint_as_float(r[cc & 1][at]), v1 = __uint_as_float(r[cc & 1][at + 1]);
            if constexpr (EPI == SKY_EPI_GELU_BWD) {
              const float2 s = __half22float2(*reinterpret_cast<const __half2*>(&sl[b][i]));
              v0 *= s.x;
              v1 *= s.y;
            } else {
              v0 += bias[i];
              v1 += bias[i];
            }
            if constexpr (EPI == SKY_EPI_BIAS_GELU) {
              float2 g, gp;
              gelu_and_grad2(v0, v1, g, gp);
              o[i] = ptx::pack_bf16(g.x, g.y);
              const __half2 h = __floats2half2_rn(gp.x, gp.y);
              x[i] = *reinterpret_cast<const uint32_t*>(&h);
            } else {
              o[i] = ptx::pack_bf16(v0, v1);
            }
          }
          const uint32_t to = piece_at(buffer, 8 * b + (lane & 7), lane >> 3);
          ptx::stmatrix_x4_trans(to, o[0], o[1], o[2], o[3]);
          if constexpr (EPI == SKY_EPI_BIAS_GELU) ptx::stmatrix_x4_trans(to + 2048, x[0], x[1], x[2], x[3]);
        }
        if (t0 + 32 <= t.count) {  // all of its tokens are the group's: by TMA, which leaves out what is behind the features
          ptx::fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0 && f0 < p.features) {
            ptx::tma_store_2d(&maps.C, box, f0, t.row + t0);
            if constexpr (EPI == SKY_EPI_BIAS_GELU) ptx::tma_store_2d(&maps.aux_out, box + 2048, f0, t.row + t0);
          }
        } else {
          __syncwarp();
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int n = 8 * i + t_at;
            uint32_t v[4];
            const bool in = f_ok && t0 + n < t.count;
            const int64_t off = static_cast<int64_t>(t.row + t0 + n) * p.features + f_at;
            ptx::ld_shared_v4(piece_at(buffer, n, lane & 3), v);
            if (in) *reinterpret_cast<uint4*>(p.C + off) = make_uint4(v[0], v[1], v[2], v[3]);
            if constexpr (EPI == SKY_EPI_BIAS_GELU) {
              ptx::ld_shared_v4(piece_at(buffer, n, lane & 3) + 2048, v);
              if (in) *reinterpret_cast<uint4*>(p.aux_out + off) = make_uint4(v[0], v[1], v[2], v[3]);
            }
          }
          __syncwarp();  // before lane 0 goes on to say that the buffer is free
        }
        if (lane == 0) ptx::bulk_commit_group();  // (an empty one behind stores by lanes)
        turn ^= 1;
      }
    }
    if (lane == 0) ptx::bulk_wait_group_read0();  // before the CTA's memory goes
  }
  pdl_trigger();
  ptx::tc_fence_before();
  __syncwarp();
  ptx::cluster_sync();  // no CTA leaves while its peer may still signal it
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc_pair(tmem_base, 512);
  }
}

// Rows of a group whose products one accumulator takes: the tensor cores cut off where they
// add up, so a long sum is made of parts, added in fp32 in the epilogue's registers.  Off by 4.4 to
// 4.8e-7 of the norm at any length; as one sum 1.6e-6 over 2000 rows, and growing with them.
constexpr int PART_ROWS = 512;

// The groups by size, largest first, for up to 32 of them (lane g holds group g's rank, and the
// group of rank g); the pairs take the tiles of such a list to and fro, so that none gets the
// larger ones of every round.  More groups come in their own order.
struct BySize {
  bool sorted;
  int at_rank = 0;
  __device__ __forceinline__ BySize(const int32_t* offset, int groups, int rows) : sorted(groups <= 32) {
    if (!sorted) return;
    const int lane = threadIdx.x & 31;
    int2 r = make_int2(0, -1);
    if (lane < groups) r = group_rows(offset, lane, rows);
    const int size = r.y - r.x;
    int rank = 0;
#pragma unroll
    for (int o = 0; o < 32; ++o) {
      const int other = __shfl_sync(0xffffffffu, size, o);
      rank += other > size || (other == size && o < lane);
    }
#pragma unroll
    for (int o = 0; o < 32; ++o)
      if (__shfl_sync(0xffffffffu, rank, o) == lane) at_rank = o;
  }
  __device__ __forceinline__ int group(int rank) const { return sorted ? __shfl_sync(0xffffffffu, at_rank, rank) : rank; }
};
// The unit of a pair's i-th round.
__device__ __forceinline__ int to_and_fro(int i, int cid, int ncl) { return i * ncl + (i & 1 ? ncl - 1 - cid : cid); }

struct GradParams {
  const int32_t* offset;
  int groups, rows, out, in;
  int m_blocks, n_blocks;  // 256 of out; of in
  int32_t* status;
  Fault fault;
};

__global__ void __launch_bounds__(GradShape::THREADS, 1)
    grouped_grad_tc(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                    const __grid_constant__ CUtensorMap tmC, const __grid_constant__ GradParams p) {
  using SH = GradShape;
  constexpr int NST = SH::STAGES, EW = SH::EW;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = ptx::smem_u32(smem_raw);
  uint8_t* smem = smem_raw + (((raw_addr + 1023u) & ~1023u) - raw_addr);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + SH::BAR_OFF);
  uint64_t* empty = full + NST;
  uint64_t* here = empty + NST;    // a block that has rows to clear: this CTA's copies have come
  uint64_t* cleared = here + NST;  // and both CTAs have cleared theirs (the leader's counts)
  uint64_t* tfull = cleared + NST;
  uint64_t* tempty = tfull + 2;
  uint64_t* done = tempty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done + 1);
  const uint32_t sent = ptx::smem_u32(tmem_slot + 1);  // blocks that this CTA's producer has sent

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = ptx::cluster_ctarank();
  const bool leader = rank == 0;
  const int cid = blockIdx.x >> 1, ncl = gridDim.x >> 1;
  if (threadIdx.x == 0) {
    for (int s = 0; s < NST; ++s) {
      ptx::mbar_init(&full[s], 1);
      ptx::mbar_init(&empty[s], 1);
      ptx::mbar_init(&here[s], 1);
      ptx::mbar_init(&cleared[s], 2);
    }
    for (int a = 0; a < 2; ++a) {
      ptx::mbar_init(&tfull[a], 1);
      ptx::mbar_init(&tempty[a], 2 * EW);
    }
    ptx::mbar_init(done, 1);
    ptx::st_shared_u32(sent, 0);
    ptx::fence_mbar_init_cluster();
    ptx::fence_proxy_async_smem();
    ptx::prefetch_tensormap(&tmA);
    ptx::prefetch_tensormap(&tmB);
  }
  if (warp == 1) {
    ptx::tmem_alloc_pair(tmem_slot, 512);
    ptx::tmem_relinquish_pair();
  }
  ptx::tc_fence_before();
  __syncwarp();
  ptx::cluster_sync();
  ptx::tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_wait();
  if (blockIdx.x == 0) check_offsets(p.offset, p.groups, p.rows, p.status);

  const int per_group = p.m_blocks * p.n_blocks, units = p.groups * per_group;
  const BySize by_size(p.offset, p.groups, p.rows);
  if (warp == 0) {
    const bool issuer = ptx::elect_one();
    int stage = 0, issued = 0;
    uint32_t phase = 0, here_phase = 0, by_here = 0;  // a bit a stage: parity of `here`; the last copies count there
    bool ok = true;
    for (int i = 0, u; ok && (u = to_and_fro(i, cid, ncl)) < units; ++i) {
      const int2 r = group_rows(p.offset, by_size.group(u / per_group), p.rows);
      const int m0 = u % per_group / p.n_blocks * TILE_M + static_cast<int>(rank) * BM;
      const int n0 = u % p.n_blocks * TILE_N + static_cast<int>(rank) * (TILE_N / 2);
      for (int k0 = r.x; k0 < r.y; k0 += BK) {
        ok = __all_sync(0xffffffffu, ptx::mbar_wait(&empty[stage], phase ^ 1u, p.fault.wait_ns, p.status));
        if (!ok) break;
        const bool clear = r.y - k0 < BK && (r.y - k0) % 16 != 0;
        if (issuer) {
          uint8_t* sa = smem + stage * SBYTES;
          uint8_t* sb = sa + A_BYTES;
          if (clear) {
            if (leader) ptx::mbar_arrive(&full[stage]);
            ptx::mbar_arrive_expect_tx(&here[stage], SBYTES + p.fault.missing(0));
            ptx::tma_load_2d(sa, &tmA, &here[stage], m0, k0);
            ptx::tma_load_2d(sa + CHUNK_BYTES, &tmA, &here[stage], m0 + 64, k0);
            ptx::tma_load_2d(sb, &tmB, &here[stage], n0, k0);
            ptx::tma_load_2d(sb + CHUNK_BYTES, &tmB, &here[stage], n0 + 64, k0);
          } else {
            if (leader) ptx::mbar_arrive_expect_tx(&full[stage], 2 * SBYTES + p.fault.missing(0));
            const uint32_t bar = ptx::mapa_shared(ptx::smem_u32(&full[stage]), 0);
            ptx::tma_load_2d_pair(sa, &tmA, bar, m0, k0);
            ptx::tma_load_2d_pair(sa + CHUNK_BYTES, &tmA, bar, m0 + 64, k0);
            ptx::tma_load_2d_pair(sb, &tmB, bar, n0, k0);
            ptx::tma_load_2d_pair(sb + CHUNK_BYTES, &tmB, bar, n0 + 64, k0);
          }
        }
        __syncwarp();
        by_here = (by_here & ~(1u << stage)) | (clear ? 1u << stage : 0u);
        if (clear) here_phase ^= 1u << stage;
        ++issued;
        if (issuer) ptx::st_shared_u32(sent, issued);
        if (++stage == NST) { stage = 0; phase ^= 1u; }
      }
    }
    // drain (bounded): every stage's last copies
    const int n_tail = min(issued, NST);
    for (int i = 0; i < n_tail; ++i) {
      if (--stage < 0) { stage = NST - 1; phase ^= 1u; }
      if (by_here >> stage & 1) ptx::mbar_wait(&here[stage], (here_phase >> stage & 1) ^ 1u, p.fault.wait_ns, p.status);
      else if (leader) ptx::mbar_wait(&full[stage], phase, p.fault.wait_ns, p.status);
    }
  } else if (warp == 1) {
    if (leader) {
      constexpr uint32_t idesc = ptx::idesc_bf16_f32(TILE_M, TILE_N, true, true);
      const bool issuer = ptx::elect_one();
      const uint32_t s0 = ptx::smem_u32(smem);
      const uint64_t da = ptx::smem_desc_sw128(s0, CHUNK_BYTES, 1024);
      const uint64_t db = ptx::smem_desc_sw128(s0 + A_BYTES, CHUNK_BYTES, 1024);
      int stage = 0, acc = 0;
      uint32_t phase = 0, aphase = 0, c_phase = 0;  // c_phase: a bit a stage
      bool ok = true;
      for (int i = 0, u; ok && (u = to_and_fro(i, cid, ncl)) < units; ++i) {
        const int2 r = group_rows(p.offset, by_size.group(u / per_group), p.rows);
        uint32_t d_tmem = 0;
        for (int k0 = r.x; k0 < r.y; k0 += BK) {
          const bool first = (k0 - r.x) % PART_ROWS == 0;
          if (first) {
            ok = __all_sync(0xffffffffu, ptx::mbar_wait_cluster(&tempty[acc], aphase ^ 1u, p.fault.wait_ns, p.status));
            if (!ok) break;
            ptx::tc_fence_after();
            d_tmem = tmem_base + acc * TILE_N;
          }
          const int left = r.y - k0, steps = left < BK ? (left + 15) / 16 : BK / 16;
          bool got = ptx::mbar_wait(&full[stage], phase, p.fault.wait_ns, p.status);
          if (left < BK && left % 16 != 0) {
            got = got && ptx::mbar_wait_cluster(&cleared[stage], c_phase >> stage & 1, p.fault.wait_ns, p.status);
            c_phase ^= 1u << stage;
          }
          ok = __all_sync(0xffffffffu, got);
          if (!ok) break;
          ptx::tc_fence_after();
          if (issuer) {
            const uint64_t off = static_cast<uint64_t>(stage * (SBYTES >> 4));
#pragma unroll
            for (int kk = 0; kk < BK / 16; ++kk)
              if (kk < steps)
                ptx::tc_mma_f16_pair(d_tmem, da + off + kk * 128, db + off + kk * 128, idesc, !first || kk > 0);
            ptx::tc_commit_pair(&empty[stage], 3);
          }
          if (++stage == NST) { stage = 0; phase ^= 1u; }
          if (k0 + BK >= r.y || (k0 + BK - r.x) % PART_ROWS == 0) {  // the part is complete
            if (issuer) ptx::tc_commit_pair(&tfull[acc], 3);
            if (++acc == 2) { acc = 0; aphase ^= 1u; }
          }
          __syncwarp();
        }
      }
      if (issuer) ptx::tc_commit_pair(done, 1);
      __syncwarp();
      ptx::mbar_wait(done, 0, p.fault.wait_ns, p.status);
    }
  } else if (warp == 2 + EW) {
    // ------------------------------------------- rows behind a group's last
    int at = 0;  // blocks so far
    uint32_t phase = 0;
    bool ok = true;
    for (int i = 0, u; ok && (u = to_and_fro(i, cid, ncl)) < units; ++i) {
      const int2 r = group_rows(p.offset, by_size.group(u / per_group), p.rows);
      const int left = (r.y - r.x) % BK, blocks = (r.y - r.x + BK - 1) / BK;
      at += blocks;
      if (left % 16 == 0) continue;
      const int stage = (at - 1) % NST;
      // Whole tiles may lie between two such blocks, so this wait goes on while others are being sent.
      bool got = false;
      for (uint32_t before = ~0u;;) {
        got = ptx::mbar_wait(&here[stage], phase >> stage & 1, p.fault.wait_ns, nullptr);
        const uint32_t now = ptx::ld_shared_u32(sent);
        if (got || now == before) break;
        before = now;
      }
      ok = __all_sync(0xffffffffu, got);
      phase ^= 1u << stage;
      if (!ok) {
        if (lane == 0 && p.status) atomicOr(p.status, kStatusTimeout);
        break;
      }
      const uint32_t s = ptx::smem_u32(smem) + stage * SBYTES;
      const int pieces = ((left + 15) / 16 * 16 - left) * 8;  // of 16 bytes, in a 64-wide box
#pragma unroll
      for (int b = 0; b < 4; ++b)
        for (int i = lane; i < pieces; i += 32) ptx::st_shared_v4(s + b * CHUNK_BYTES + left * 128 + i * 16, 0, 0, 0, 0);
      ptx::fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive_cluster(ptx::mapa_shared(ptx::smem_u32(&cleared[stage]), 0));
    }
  } else {
    // Warp w has TMEM lanes 32 q .. (rows of the tile) and one half of its columns.
    const int q = warp & 3, half = (warp - 2) >> 2;
    uint8_t* const staging = smem + SH::EPI_OFF + (warp - 2) * SH::STAGING;
    int acc = 0;
    uint32_t aphase = 0;
    bool ok = true;
    for (int i = 0, u; ok && (u = to_and_fro(i, cid, ncl)) < units; ++i) {
      const int group = by_size.group(u / per_group);
      const int2 rr = group_rows(p.offset, group, p.rows);
      const int m0 = u % per_group / p.n_blocks * TILE_M + static_cast<int>(rank) * BM + q * 32;
      const int n0 = u % p.n_blocks * TILE_N + half * (TILE_N / 2);
      float sum[4][32] = {};  // (all of it, for a group without rows)
      for (int k0 = rr.x; k0 < rr.y; k0 += PART_ROWS) {
        ok = __all_sync(0xffffffffu, ptx::mbar_wait(&tfull[acc], aphase, p.fault.wait_ns, p.status, SLEEP_NS));
        if (!ok) break;
        ptx::tc_fence_after();
        const uint32_t taddr = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + acc * TILE_N + half * (TILE_N / 2);
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          uint32_t r[16];
          ptx::tmem_ld_32x32b_x16(taddr + 16 * c, r);
          ptx::tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 16; ++e) sum[c >> 1][(c & 1) * 16 + e] += __uint_as_float(r[e]);
        }
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive_cluster_relaxed(ptx::mapa_shared(ptx::smem_u32(&tempty[acc]), 0));
        if (++acc == 2) { acc = 0; aphase ^= 1u; }
      }
      if (!ok) break;
#pragma unroll
      for (int c = 0; c < TILE_N / 2 / 32; ++c) {
        if (lane == 0) ptx::bulk_wait_group_read0();  // the box before has left the buffer
        __syncwarp();
        const uint32_t to = ptx::smem_u32(staging) + lane * 128;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          ptx::st_shared_v4(to + ((j ^ (lane & 7)) << 4), __float_as_uint(sum[c][4 * j]), __float_as_uint(sum[c][4 * j + 1]),
                            __float_as_uint(sum[c][4 * j + 2]), __float_as_uint(sum[c][4 * j + 3]));
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          if (m0 < p.out && n0 + 32 * c < p.in)  // (what lies outside out x in is not written)
            ptx::tma_store_3d(&tmC, staging, n0 + 32 * c, m0, group);
          ptx::bulk_commit_group();
        }
      }
    }
    if (lane == 0) ptx::bulk_wait_group_read0();  // before the CTA's memory goes
  }
  pdl_trigger();
  ptx::tc_fence_before();
  __syncwarp();
  ptx::cluster_sync();
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc_pair(tmem_base, 512);
  }
}

template <bool W_MN, int EPI>
cudaError_t launch_rows(const Maps& maps, const Params& p, int64_t units, int sms, cudaStream_t st) {
  using SH = Shape<EPI>;
  auto kern = grouped_rows_tc<W_MN, EPI>;
  static OncePerDevice once;
  const cudaError_t attr = allow_smem(once, kern, SH::SMEM);
  if (attr != cudaSuccess) return attr;
  static CountPerDevice count;
  const int most = clusters_at_once(count, kern, 2, SH::THREADS, SH::SMEM, sms);
  if (most < 1) return cudaErrorLaunchOutOfResources;
  const int pairs = static_cast<int>(std::min<int64_t>(units, most));
  return launch_pdl(kern, dim3(2 * pairs), dim3(SH::THREADS), SH::SMEM, st, 2, maps, p);
}

cudaError_t launch_grad(const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& tc, const GradParams& p, int sms,
                        cudaStream_t st) {
  using SH = GradShape;
  static OncePerDevice once;
  const cudaError_t attr = allow_smem(once, grouped_grad_tc, SH::SMEM);
  if (attr != cudaSuccess) return attr;
  static CountPerDevice count;
  const int most = clusters_at_once(count, grouped_grad_tc, 2, SH::THREADS, SH::SMEM, sms);
  if (most < 1) return cudaErrorLaunchOutOfResources;
  const int64_t units = static_cast<int64_t>(p.groups) * p.m_blocks * p.n_blocks;
  const int pairs = static_cast<int>(std::min<int64_t>(units, most));
  return launch_pdl(grouped_grad_tc, dim3(2 * pairs), dim3(SH::THREADS), SH::SMEM, st, 2, ta, tb, tc, p);
}

}  // namespace

sky_status launch_tc(const Call& c, cudaStream_t st) {
  const int sms = sm_count();
  SKY_CHECK(sms > 0, SKY_ERR_CUDA, "no CUDA device");
  if (few_pays(c, sms)) return launch_few(c, sms, st);
  if (const int splits = grad_few_splits(c, sms); splits > 1) return launch_grad_few(c, splits, st);
  cudaError_t e;
  if (c.form == SKY_GEMM_XTW) {
    CUtensorMap ta, tb, tc;
    const bool ok = gemm::make_map(&ta, c.A, c.rows, c.out, 64) && gemm::make_map(&tb, c.B, c.rows, c.in, 64) &&
                    gemm::make_map_3d(&tc, c.C, c.groups, c.out, c.in, 32, 32, true);
    SKY_CHECK(ok, SKY_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d x %d x %d)", c.groups, c.out, c.in);
    const GradParams p{c.offset, c.groups, c.rows, c.out, c.in, ceil_div(c.out, TILE_M), ceil_div(c.in, TILE_N),
                       c.status, fault_of(1)};
    SKY_CHECK(static_cast<int64_t>(p.groups) * p.m_blocks * p.n_blocks <= 0x3fffffff, SKY_ERR_UNSUPPORTED,
              "grouped weight gradient too large");
    e = launch_grad(ta, tb, tc, p, sms, st);
  } else {
    const bool xw = c.form == SKY_GEMM_XW;
    Params p{};
    p.offset = c.offset;
    p.groups = c.groups;
    p.rows = c.rows;
    p.features = xw ? c.in : c.out;
    p.k = xw ? c.out : c.in;
    p.f_blocks = ceil_div(p.features, TILE_M);
    p.k_blocks = ceil_div(p.k, BK);
    p.C = static_cast<__nv_bfloat16*>(c.C);
    p.bias = static_cast<const __nv_bfloat16*>(c.bias);
    p.aux = static_cast<const __half*>(c.aux);
    p.aux_out = static_cast<__half*>(c.aux_out);
    p.status = c.status;
    p.fault = fault_of(1);
    // tiles of tokens: every group that has any may end inside one
    const int64_t units = (c.rows / TILE_N + static_cast<int64_t>(std::min(c.groups, c.rows))) * p.f_blocks;
    SKY_CHECK(units <= 0x3fffffff, SKY_ERR_UNSUPPORTED, "grouped product too large");
    Maps m;
    bool ok = gemm::make_map_3d(&m.weights, c.B, c.groups, c.out, c.in, xw ? 64 : BM, 64, false);
    for (int b = 0; b < 4; ++b) ok = ok && gemm::make_map(&m.rows[b], c.A, c.rows, p.k, 16 << b);
    ok = ok && gemm::make_store_map(&m.C, c.C, c.rows, p.features, false);
    if (c.epi == SKY_EPI_BIAS_GELU) ok = ok && gemm::make_store_map(&m.aux_out, c.aux_out, c.rows, p.features, true);
    else m.aux_out = m.C;
    SKY_CHECK(ok, SKY_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d x %d x %d)", c.groups, c.out, c.in);
    if (!xw)
      e = c.epi == SKY_EPI_BIAS_GELU ? launch_rows<false, SKY_EPI_BIAS_GELU>(m, p, units, sms, st)
                                     : launch_rows<false, SKY_EPI_STORE>(m, p, units, sms, st);
    else
      e = c.epi == SKY_EPI_GELU_BWD ? launch_rows<true, SKY_EPI_GELU_BWD>(m, p, units, sms, st)
                                    : launch_rows<true, SKY_EPI_STORE>(m, p, units, sms, st);
  }
  count_launches(1);
  return e == cudaSuccess ? SKY_OK : cuda_fail(e, "grouped tensor-core product launch");
}

}  // namespace grouped
}  // namespace sky
