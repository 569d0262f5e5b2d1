// The products grouped by expert (sky_experts.h): what their kernels share.
#pragma once
#include <cuda_runtime.h>

#include "../../include/sky_experts.h"

namespace sky {
namespace grouped {

// A call, checked.  Weights are [groups][out][in]; group g owns the rows
// [offset[g], offset[g + 1]) of the ragged matrices.
//   XWT: A [rows, in],  B weights,      C [rows, out]
//   XW:  A [rows, out], B weights,      C [rows, in]
//   XTW: A [rows, out], B [rows, in],   C fp32 [groups][out][in]
struct Call {
  sky_gemm_form form;
  int groups, rows, out, in;
  const int32_t* offset;
  const void *A, *B;
  void* C;
  sky_epilogue epi;
  const void *bias, *aux;
  void* aux_out;
  int32_t* status;
};

// The limit of any one wait of the tensor-core kernels, and the splits, from one on, that expect
// 16 bytes more than their copies bring, so that their waits run out (sky_debug_gemm_fault).  A branch
// around the copies in its place takes 2% more of a small call.
struct Fault {
  uint64_t wait_ns;
  int missing_from;
  __host__ __device__ uint32_t missing(int split) const { return split >= missing_from ? 16 : 0; }
};
Fault fault_of(int splits);

// fp32 arithmetic on the CUDA cores (grouped_f32.cu).
sky_status launch_simt(const Call& c, cudaStream_t st);
// bf16 on the tensor cores (grouped_tc.cu).
sky_status launch_tc(const Call& c, cudaStream_t st);
// The same for few rows (grouped_few.cu), and whether a call is one of those.
bool few_pays(const Call& c, int sms);
sky_status launch_few(const Call& c, int sms, cudaStream_t st);
// XTW of few tiles (grouped_grad_few.cu), and into how many splits of the rows it then pays (1: it does not).
int grad_few_splits(const Call& c, int sms);
sky_status launch_grad_few(const Call& c, int splits, cudaStream_t st);
bool few_f32_pays(const Call& c);  // fp32 (grouped_few_f32.cu)
sky_status launch_few_f32(const Call& c, cudaStream_t st);

}  // namespace grouped
}  // namespace sky
