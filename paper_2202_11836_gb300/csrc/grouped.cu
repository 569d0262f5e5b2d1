// The C ABI of the products grouped by expert, and their bias gradients (sky_experts.h).
#include <climits>
#include <type_traits>

#include "abi.h"
#include "gemm.h"
#include "grouped.cuh"
#include "grouped.h"
#include "ptx.cuh"

namespace sky {
namespace grouped {
namespace {

constexpr int MAX_GROUPS = 1024;

bool on(const void* p, size_t grid) { return reinterpret_cast<uintptr_t>(p) % grid == 0; }

// Sizes that every call needs; `in` is 0 where there are no weights.
sky_status check(const sky_grouped_shape* s, bool weights) {
  SKY_CHECK(s, SKY_ERR_INVALID_ARG, "null shape");
  SKY_CHECK(s->groups > 0 && s->rows > 0 && s->out > 0 && (!weights || s->in > 0), SKY_ERR_INVALID_ARG, "bad sizes");
  SKY_CHECK(s->dtype == SKY_DTYPE_BF16 || s->dtype == SKY_DTYPE_FP32, SKY_ERR_INVALID_ARG, "unknown dtype");
  SKY_CHECK(s->groups <= MAX_GROUPS && s->rows < (1 << 28) && s->out <= (1 << 20) && (!weights || s->in <= (1 << 20)),
            SKY_ERR_UNSUPPORTED, "more than %d groups, 2^28 rows or more, or weights wider than 2^20", MAX_GROUPS);
  if (weights) {
    SKY_CHECK(s->dtype == SKY_DTYPE_FP32 || (s->out % 8 == 0 && s->in % 8 == 0), SKY_ERR_UNSUPPORTED,
              "bf16 grouped products need weights of multiples of 8 (got %d x %d)", s->out, s->in);
    SKY_CHECK(static_cast<int64_t>(s->groups) * s->out < (int64_t{1} << 31), SKY_ERR_UNSUPPORTED,
              "2^31 or more rows of weights");
  }
  return SKY_OK;
}

sky_status check_form(sky_gemm_form form, const sky_grouped_shape& s, sky_dtype out_dtype) {
  SKY_CHECK(form == SKY_GEMM_XWT || form == SKY_GEMM_XW || form == SKY_GEMM_XTW, SKY_ERR_INVALID_ARG, "unknown form");
  SKY_CHECK(out_dtype == SKY_DTYPE_BF16 || out_dtype == SKY_DTYPE_FP32, SKY_ERR_INVALID_ARG, "unknown output dtype");
  SKY_CHECK(out_dtype == (form == SKY_GEMM_XTW ? SKY_DTYPE_FP32 : s.dtype), SKY_ERR_UNSUPPORTED,
            "grouped products are in the operands' dtype, weight gradients in fp32");
  return SKY_OK;
}

}  // namespace

Fault fault_of(int splits) {
  const gemm::Debug d = gemm::debug();
  return {d.wait_ns, d.skip_loads == 0 ? INT_MAX : d.skip_loads == 2 ? splits - 1 : 0};
}

namespace {

// Asked for and checked, not used: partial sums go through distributed shared memory.
constexpr size_t WORKSPACE = 16;

// Column sums over the rows of a group: TX threads take TX V columns (512 or 128 bytes of a row), the
// others of a CTA other rows, and their sums are added in order.  A group's rows are shared by
// the CTAs of a cluster (up to eight), whose sums the first adds in order.  Long pieces of rows read
// faster (16384 x 4096 over 8 groups 25.4 us, in short ones 41.0); short ones make more CTAs where
// there would be few (5000 x 768, one group, 8.6 and 5.8).
template <typename T, bool VEC, int TX>
__global__ void __launch_bounds__(256) column_sums(const T* __restrict__ x, const int32_t* offset, int groups, int rows, int N,
                                                   int strips, int parts, float* out, int32_t* status) {
  constexpr int V = VEC ? 16 / sizeof(T) : 4, COLS = TX * V, TY = 256 / TX;
  __shared__ __align__(16) float part[TY][COLS + (TX < 32 ? 4 : 0)];
  __shared__ float all[8][COLS];  // of the cluster's CTAs, in the first
  if (parts > 1) ptx::cluster_arrive();  // this CTA runs: its peers may write its shared memory
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x == 0) check_offsets(offset, groups, rows, status);
  const int mine = blockIdx.x % parts, unit = blockIdx.x / parts, g = unit / strips, strip = unit % strips;
  const int cl = threadIdx.x % TX * V, col = strip * COLS + cl, rl = threadIdx.x / TX;
  const int2 r = group_rows(offset, g, rows);
  const int64_t n = r.y - r.x;
  const int lo = r.x + static_cast<int>(n * mine / parts), hi = r.x + static_cast<int>(n * (mine + 1) / parts);
  float sum[V] = {};
  if (col < N) {
#pragma unroll 8
    for (int i = lo + rl; i < hi; i += TY) {
      const T* p = x + static_cast<int64_t>(i) * N + col;
      if constexpr (VEC) {
        const uint4 u = __ldg(reinterpret_cast<const uint4*>(p));
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int e = 0; e < V; ++e)
          sum[e] += V == 4 ? __uint_as_float(w[e])
                           : __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (col + e < N) sum[e] += to_f32<T>(p[e]);
      }
    }
  }
#pragma unroll
  for (int e = 0; e < V; e += 4)
    *reinterpret_cast<float4*>(&part[rl][cl + e]) = make_float4(sum[e], sum[e + 1], sum[e + 2], sum[e + 3]);
  __syncthreads();
  const int c = threadIdx.x;
  float s = 0.f;
  if (c < COLS) {
    s = part[0][c];
#pragma unroll
    for (int i = 1; i < TY; ++i) s += part[i][c];
  }
  if (parts > 1) {
    ptx::cluster_wait();  // every peer runs
    if (c < COLS) ptx::st_cluster_u32(ptx::mapa_shared(ptx::smem_u32(&all[mine][c]), 0), __float_as_uint(s));
    ptx::cluster_sync();
    if (mine != 0) return;
    if (c < COLS) {
      s = all[0][c];
      for (int i = 1; i < parts; ++i) s += all[i][c];
    }
  }
  if (c < COLS && strip * COLS + c < N) out[static_cast<int64_t>(g) * N + strip * COLS + c] = s;
}

template <typename T, bool VEC, int TX>
cudaError_t launch_strips(const sky_grouped_shape& s, const int32_t* offset, const void* x, float* out, int32_t* status,
                          cudaStream_t st) {
  const int strips = ceil_div(s.out, TX * (VEC ? 16 / static_cast<int>(sizeof(T)) : 4));
  // parts of a mean group's rows, 64 or more each, while the CTAs are no more than 32 an SM
  int parts = 1;
  while (parts < 8 && s.rows / s.groups >= 128 * parts && static_cast<int64_t>(s.groups) * strips * parts * 2 <= 32 * sm_count())
    parts *= 2;
  return launch_pdl(column_sums<T, VEC, TX>, dim3(s.groups * strips * parts), dim3(256), 0, st, parts,
                    static_cast<const T*>(x), offset, s.groups, s.rows, s.out, strips, parts, out, status);
}
template <typename T, bool VEC>
cudaError_t launch_sums(const sky_grouped_shape& s, const int32_t* offset, const void* x, float* out, int32_t* status,
                        cudaStream_t st) {
  const int cols = 32 * (VEC ? 16 / static_cast<int>(sizeof(T)) : 4);
  return static_cast<int64_t>(s.groups) * ceil_div(s.out, cols) * 8 < sm_count()
             ? launch_strips<T, VEC, 8>(s, offset, x, out, status, st)
             : launch_strips<T, VEC, 32>(s, offset, x, out, status, st);
}

}  // namespace
}  // namespace grouped
}  // namespace sky

using namespace sky;

extern "C" {

size_t sky_grouped_gemm_workspace_bytes(sky_gemm_form form, const sky_grouped_shape* shape, sky_dtype out_dtype) {
  if (grouped::check(shape, true) != SKY_OK || grouped::check_form(form, *shape, out_dtype) != SKY_OK) return 0;
  return grouped::WORKSPACE;
}

sky_status sky_grouped_gemm(sky_gemm_form form, const sky_grouped_shape* shape, const int32_t* d_offset, const void* A,
                            const void* B, void* C, sky_dtype out_dtype, sky_epilogue epilogue, const void* bias,
                            const void* aux, void* aux_out, void* workspace, size_t workspace_bytes, int32_t* d_status,
                            void* stream) {
  ABI_GUARD_BEGIN
  sky_status ok = grouped::check(shape, true);
  if (ok == SKY_OK) ok = grouped::check_form(form, *shape, out_dtype);
  if (ok != SKY_OK) return ok;
  SKY_CHECK(d_offset && A && B && C && workspace, SKY_ERR_INVALID_ARG, "null argument");
  SKY_CHECK(epilogue == SKY_EPI_STORE || epilogue == SKY_EPI_BIAS_GELU || epilogue == SKY_EPI_GELU_BWD, SKY_ERR_INVALID_ARG,
            "unknown epilogue");
  SKY_CHECK((epilogue != SKY_EPI_BIAS_GELU || form == SKY_GEMM_XWT) && (epilogue != SKY_EPI_GELU_BWD || form == SKY_GEMM_XW) &&
                (!bias || form == SKY_GEMM_XWT),
            SKY_ERR_UNSUPPORTED, "a grouped product's bias and GELU come with the form XWT, GELU' with XW");
  SKY_CHECK((epilogue != SKY_EPI_BIAS_GELU || aux_out) && (epilogue != SKY_EPI_GELU_BWD || aux), SKY_ERR_INVALID_ARG,
            "GELU needs aux_out, GELU' aux");
  const bool bf16 = shape->dtype == SKY_DTYPE_BF16;
  SKY_CHECK(grouped::on(d_offset, 4) && grouped::on(d_status, 4) && grouped::on(workspace, 16) &&
                grouped::on(bias, bf16 ? 2 : 4) && grouped::on(aux, bf16 ? 2 : 4) && grouped::on(aux_out, bf16 ? 2 : 4) &&
                (bf16 || (grouped::on(A, 4) && grouped::on(B, 4) && grouped::on(C, 4))),
            SKY_ERR_INVALID_ARG, "a pointer off its type's grid");
  SKY_CHECK(!bf16 || (grouped::on(A, 16) && grouped::on(B, 16) && grouped::on(C, 16) &&
                      (epilogue != SKY_EPI_GELU_BWD || grouped::on(aux, 16)) &&
                      (epilogue != SKY_EPI_BIAS_GELU || grouped::on(aux_out, 16))),
            SKY_ERR_UNSUPPORTED, "bf16 grouped products need A, B, C, aux and aux_out 16-byte aligned");
  SKY_CHECK(workspace_bytes >= grouped::WORKSPACE, SKY_ERR_INVALID_ARG, "workspace too small");
  const grouped::Call c{form, shape->groups, shape->rows, shape->out, shape->in, d_offset, A, B, C, epilogue, bias, aux,
                        aux_out, d_status};
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return bf16 ? grouped::launch_tc(c, st) : grouped::launch_simt(c, st);
  ABI_GUARD_END
}

sky_status sky_grouped_column_sum(const sky_grouped_shape* shape, const int32_t* d_offset, const void* x, float* out,
                                  int32_t* d_status, void* stream) {
  ABI_GUARD_BEGIN
  const sky_status ok = grouped::check(shape, false);
  if (ok != SKY_OK) return ok;
  SKY_CHECK(d_offset && x && out, SKY_ERR_INVALID_ARG, "null argument");
  const bool bf16 = shape->dtype == SKY_DTYPE_BF16;
  SKY_CHECK(grouped::on(d_offset, 4) && grouped::on(d_status, 4) && grouped::on(out, 4) && grouped::on(x, bf16 ? 2 : 4),
            SKY_ERR_INVALID_ARG, "a pointer off its type's grid");
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool vec = grouped::on(x, 16) && shape->out % (bf16 ? 8 : 4) == 0;
  const cudaError_t e =
      bf16 ? (vec ? grouped::launch_sums<__nv_bfloat16, true>(*shape, d_offset, x, out, d_status, st)
                  : grouped::launch_sums<__nv_bfloat16, false>(*shape, d_offset, x, out, d_status, st))
           : (vec ? grouped::launch_sums<float, true>(*shape, d_offset, x, out, d_status, st)
                  : grouped::launch_sums<float, false>(*shape, d_offset, x, out, d_status, st));
  count_launches(1);
  return e == cudaSuccess ? SKY_OK : cuda_fail(e, "grouped column sum launch");
  ABI_GUARD_END
}

}  // extern "C"
