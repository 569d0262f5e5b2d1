// fp32 SIMT GEMM: exact fp32 FMA accumulation for the tight-tolerance fp32
// slice (tensor-core TF32 would not reach a 1e-4 relative error).  Same
// three contraction forms and epilogues as the bf16 tensor-core kernel.
//
// Bound by the FMA pipe (128 a clock and SM) where there is work enough, else by
// the latency of a slab.  A CTA of four warps computes a 64 x 64 tile, 8 x 4 a
// thread, from 32-deep slabs of A and B in shared memory (double-buffered, the
// next slab's loads in flight in registers), two adjacent columns to a packed
// FMA.  8 x 8 a thread, or 16-deep slabs, were slower: fewer warps, and less in
// flight.  The layer's products have few such tiles (404 x 768: 84 for 152 SMs,
// each SM wanting four CTAs or more), so the K range is split over a cluster of
// up to eight CTAs.  Each owns a share of the tile's rows; the others send it
// theirs through distributed shared memory, and it adds them in split order
// (reading them from the peers, behind a second barrier, cost 0.7 us a launch:
// 2-layer slice of width 128 219 -> 186 us).  Against the kernel before (64 x 64, 4 x 4 a
// thread, scalar loads, no split), alone: 404 x 768 x 3072 196 -> 52 us (37
// TFLOP/s), 1000 x 2304 x 768 -> 77 us (46 TFLOP/s);
// the error against float64 falls with the shorter sums (9.9e-7 -> 3.5e-7).
#include "common.cuh"
#include "f32_tile.cuh"
#include "gemm.h"
#include "ptx.cuh"

namespace sky {
namespace gemm {

namespace {

struct F32Params {
  int M, N, K, n_tiles, ks, k_slabs;
  const float *A, *B;
  int64_t lda, ldb;
  float* C;
  int epi;
  const float *bias, *aux;
  float* aux_out;
};

template <bool AK, bool BK, bool VEC>
__global__ void __launch_bounds__(F_THREADS) gemm_f32_kernel(const F32Params p) {
  if (p.ks > 1) ptx::cluster_arrive();  // this CTA runs: its peers may write its shared memory
  pdl_wait();
  const int split = static_cast<int>(blockIdx.x) % p.ks, tile = static_cast<int>(blockIdx.x) / p.ks;
  const int m0 = (tile / p.n_tiles) * TM, n0 = (tile % p.n_tiles) * TN;
  const int s0 = split * p.k_slabs / p.ks, s1 = (split + 1) * p.k_slabs / p.ks;
  auto finish = [&](int m, int n, float v) {
    if (m >= p.M || n >= p.N) return;
    const int64_t off = static_cast<int64_t>(m) * p.N + n;
    if (p.bias) v += p.bias[n];
    if (p.epi == SKY_EPI_GELU_BWD) v *= p.aux[off];
    if (p.epi == SKY_EPI_BIAS_GELU) {
      p.aux_out[off] = gelu_grad_f(v);
      v = gelu_f(v);
    }
    p.C[off] = v;
  };
  f32_tile<AK, BK, VEC>(F32Operands{p.A, p.B, p.lda, p.ldb, p.M, p.N, p.K}, m0, n0, p.ks, split, s0, s1, finish);
}
}  // namespace

sky_status launch_f32(sky_gemm_form form, int M, int N, int K, const float* A, const float* B,
                      float* C, int epi, const float* bias, const float* aux, float* aux_out,
                      cudaStream_t stream) {
  SKY_CHECK(epi != SKY_EPI_BIAS_GELU || (bias && aux_out), SKY_ERR_INVALID_ARG,
            "BIAS_GELU epilogue needs bias and aux_out");
  SKY_CHECK(epi == SKY_EPI_STORE || epi == SKY_EPI_BIAS_GELU || epi == SKY_EPI_GELU_BWD,
            SKY_ERR_INVALID_ARG, "unknown epilogue %d", epi);
  SKY_CHECK(epi != SKY_EPI_GELU_BWD || aux, SKY_ERR_INVALID_ARG, "GELU' epilogue needs aux");
  const bool ak = form != SKY_GEMM_XTW, bk = form == SKY_GEMM_XWT;  // K-major operands
  F32Params p{};
  p.M = M; p.N = N; p.K = K;
  p.A = A; p.B = B; p.C = C;
  p.lda = ak ? K : M;
  p.ldb = bk ? K : N;
  p.epi = epi;
  p.bias = bias; p.aux = aux; p.aux_out = aux_out;
  p.n_tiles = ceil_div(N, TN);
  p.k_slabs = ceil_div(K, TK);
  const int64_t tiles = static_cast<int64_t>(ceil_div(M, TM)) * p.n_tiles;
  const int sms = sm_count() > 0 ? sm_count() : 148;
  // Splits: a lone CTA waits for its loads, so an SM wants several.  Eight splits up
  // to eleven CTAs an SM, else four, each of two slabs or more.  Where the tiles are
  // few, one slab is enough, and eight only if every CTA has an SM to itself or that
  // halves the longest one's slabs.
  // Never two, whose pairs land on one SM.  us at 1 / 2 / 4 / 8 splits: 404 x 768 x
  // 3072 99 / - / 61 / 51, 404 x 2304 x 768 42 / - / 38 / 40, 1000 x 768 x 3072 171 / - /
  // 115 / 106, 1000 x 2304 x 768 77 / 82 / 83 / 85, 512 x 2048 x 97 9.9 / 16.1 / 13.1 / -,
  // 128 x 384 x 128 5.8 / 7.7 / 3.7 / -; 256 x 384 x 384 (12 slabs) 5.8 at four, 7.0 at
  // eight, 384 x 384 x 256 (8) 6.5 and 6.0, 150 x 448 x 448 (14) 6.8 and 6.5.
  p.ks = 1;
  const bool few = 4 * tiles <= sms;
  const bool halves = 2 * ceil_div(p.k_slabs, 8) <= ceil_div(p.k_slabs, 4);
  for (int ks = 8; ks >= 4 && p.ks == 1; ks /= 2) {
    const bool one_slab = few && p.k_slabs >= ks && (ks == 4 || 8 * tiles <= sms || halves);
    if (tiles * ks <= 11 * sms && (p.k_slabs >= 2 * ks || one_slab)) p.ks = ks;
  }
  const bool vec = p.lda % 4 == 0 && p.ldb % 4 == 0 && (reinterpret_cast<uintptr_t>(A) & 15) == 0 &&
                   (reinterpret_cast<uintptr_t>(B) & 15) == 0;
  SKY_CHECK(tiles * p.ks <= 0x7fffffff, SKY_ERR_INVALID_ARG, "GEMM too large (M=%d N=%d)", M, N);
  const dim3 grid(static_cast<unsigned>(tiles * p.ks)), blk(F_THREADS);
  auto go = [&](auto kern) { return launch_pdl(kern, grid, blk, 0, stream, p.ks, p); };
  cudaError_t e;
  if (form == SKY_GEMM_XWT) e = vec ? go(gemm_f32_kernel<true, true, true>) : go(gemm_f32_kernel<true, true, false>);
  else if (form == SKY_GEMM_XW) e = vec ? go(gemm_f32_kernel<true, false, true>) : go(gemm_f32_kernel<true, false, false>);
  else e = vec ? go(gemm_f32_kernel<false, false, true>) : go(gemm_f32_kernel<false, false, false>);
  count_launches(1);
  return e == cudaSuccess ? SKY_OK : cuda_fail(e, "gemm_f32_kernel launch");
}

}  // namespace gemm
}  // namespace sky
