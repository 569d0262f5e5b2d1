// Products grouped by expert in fp32 arithmetic on the CUDA cores: the tiles of gemm_f32.cu,
// each over the rows of one group.  Bound as those are, by the FMA pipe or, with few rows, by
// the latency of a slab (grouped_few_f32.cu has the forward of those); the number of tiles is known
// on the device only, so the grid holds as many as the rows may make and those that are too many
// leave at once.
#include <algorithm>

#include "common.cuh"
#include "f32_tile.cuh"
#include "grouped.cuh"
#include "grouped.h"
#include "ptx.cuh"

namespace sky {
namespace grouped {
namespace {

using gemm::F_THREADS;
using gemm::TK;
using gemm::TM;
using gemm::TN;

struct Params {
  Call c;
  int m_tiles, n_tiles, ks;  // m_tiles: XTW only
};

template <int FORM, bool VEC>
__global__ void __launch_bounds__(F_THREADS, 4) grouped_simt(const __grid_constant__ Params p) {
  const Call& c = p.c;
  pdl_wait();
  const int split = static_cast<int>(blockIdx.x) % p.ks, tile = static_cast<int>(blockIdx.x) / p.ks;
  if (blockIdx.x == 0) check_offsets(c.offset, c.groups, c.rows, c.status);
  const float *A = static_cast<const float*>(c.A), *B = static_cast<const float*>(c.B);
  gemm::F32Operands o;
  int m0, n0, g;
  int64_t row0 = 0;
  if constexpr (FORM == SKY_GEMM_XTW) {
    g = tile / (p.m_tiles * p.n_tiles);
    const int in_group = tile % (p.m_tiles * p.n_tiles);
    m0 = in_group / p.n_tiles * TM;
    n0 = in_group % p.n_tiles * TN;
    const int2 r = group_rows(c.offset, g, c.rows);
    o = {A + static_cast<int64_t>(r.x) * c.out, B + static_cast<int64_t>(r.x) * c.in, c.out, c.in, c.out, c.in, r.y - r.x};
  } else {
    const Found f = find_tile(c.offset, c.groups, c.rows, tile / p.n_tiles, [](int n) { return (n + TM - 1) / TM; });
    if (f.group < 0) return;  // (every CTA of a cluster)
    g = f.group;
    m0 = f.tile * TM;
    n0 = tile % p.n_tiles * TN;
    row0 = f.lo;
    const int K = FORM == SKY_GEMM_XWT ? c.in : c.out, N = FORM == SKY_GEMM_XWT ? c.out : c.in;
    o = {A + row0 * K, B + static_cast<int64_t>(g) * c.out * c.in, K, c.in, f.hi - f.lo, N, K};
  }
  if (p.ks > 1) ptx::cluster_arrive();  // this CTA runs: its peers may write its shared memory
  const int slabs = (o.K + TK - 1) / TK;
  const int s0 = static_cast<int>(static_cast<int64_t>(split) * slabs / p.ks);
  const int s1 = static_cast<int>(static_cast<int64_t>(split + 1) * slabs / p.ks);
  auto finish = [&](int m, int n, float v) {
    if (m >= o.M || n >= o.N) return;
    if constexpr (FORM == SKY_GEMM_XTW) {
      static_cast<float*>(c.C)[(static_cast<int64_t>(g) * c.out + m) * c.in + n] = v;
    } else {
      const int64_t off = (row0 + m) * o.N + n;
      if (FORM == SKY_GEMM_XWT && c.bias) v += static_cast<const float*>(c.bias)[static_cast<int64_t>(g) * c.out + n];
      if (c.epi == SKY_EPI_GELU_BWD) v *= static_cast<const float*>(c.aux)[off];
      if (c.epi == SKY_EPI_BIAS_GELU) {
        static_cast<float*>(c.aux_out)[off] = gelu_grad_f(v);
        v = gelu_f(v);
      }
      static_cast<float*>(c.C)[off] = v;
    }
  };
  gemm::f32_tile<FORM != SKY_GEMM_XTW, FORM == SKY_GEMM_XWT, VEC>(o, m0, n0, p.ks, split, s0, s1, finish);
}

template <int FORM>
sky_status launch(const Call& c, cudaStream_t st) {
  const int sms = sm_count();
  SKY_CHECK(sms > 0, SKY_ERR_CUDA, "no CUDA device");
  Params p{};
  p.c = c;
  const int N = FORM == SKY_GEMM_XWT ? c.out : c.in;
  p.n_tiles = ceil_div(N, TN);
  p.m_tiles = FORM == SKY_GEMM_XTW ? ceil_div(c.out, TM) : 0;
  // tiles of rows: every group that has any may end inside one
  const int64_t m_tiles = FORM == SKY_GEMM_XTW ? static_cast<int64_t>(c.groups) * p.m_tiles
                                               : c.rows / TM + static_cast<int64_t>(std::min(c.groups, c.rows));
  const int64_t tiles = m_tiles * p.n_tiles;
  // Splits, by the slabs of a mean group: the most of 8, 4 and 2 that make no more than four CTAs an
  // SM and have slabs enough.  us at 1 / 2 / 4 / 8 (tiles that the rows may make, slabs): 257 x 512 x
  // 128 with GELU, 4 groups (64, 4) 10.0 7.9 6.2 7.9; 1000 x 128 x 512, 16 groups (62, 16) 21.5 13.5
  // 12.0 10.3; 1000 x 768 x 768 (228, 24) 58 36 38 40; 40 x 200 x 300, 20 groups (80, 10) 16.1 12.7 11.4
  // 13.7; 4000 x 300 x 200 (320, 7) 21.4 23.6 25.2 31.5; weight gradients of 257 rows (64, 3) 6.7 6.2 4.8
  // 6.8, of 1000 over 16 groups (256, 2) 9.4 9.9 12.4 19.8, of 4000 over 2 (40, 63) 111 57 36 26.
  const int K = FORM == SKY_GEMM_XWT ? c.in : FORM == SKY_GEMM_XW ? c.out : ceil_div(c.rows, c.groups);
  const int slabs = ceil_div(K, TK);
  p.ks = 1;
  for (int ks = 8; ks >= 2 && p.ks == 1; ks /= 2)
    if (tiles * ks <= 4 * sms && slabs >= (ks == 8 ? 16 : ks == 4 ? 3 : 4)) p.ks = ks;
  SKY_CHECK(tiles * p.ks <= 0x7fffffff, SKY_ERR_UNSUPPORTED, "grouped product too large");
  const auto a16 = [](const void* q) { return (reinterpret_cast<uintptr_t>(q) & 15) == 0; };
  const bool vec = c.in % 4 == 0 && c.out % 4 == 0 && a16(c.A) && a16(c.B);
  const dim3 grid(static_cast<unsigned>(tiles * p.ks));
  const cudaError_t e = vec ? launch_pdl(grouped_simt<FORM, true>, grid, dim3(F_THREADS), 0, st, p.ks, p)
                            : launch_pdl(grouped_simt<FORM, false>, grid, dim3(F_THREADS), 0, st, p.ks, p);
  count_launches(1);
  return e == cudaSuccess ? SKY_OK : cuda_fail(e, "grouped product launch");
}

}  // namespace

sky_status launch_simt(const Call& c, cudaStream_t st) {
  if (few_f32_pays(c)) return launch_few_f32(c, st);
  if (c.form == SKY_GEMM_XWT) return launch<SKY_GEMM_XWT>(c, st);
  if (c.form == SKY_GEMM_XW) return launch<SKY_GEMM_XW>(c, st);
  return launch<SKY_GEMM_XTW>(c, st);
}

}  // namespace grouped
}  // namespace sky
