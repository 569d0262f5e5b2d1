// The head norms of qk_norm.cuh for bf16, a translation unit of their own to build beside
// the others.
#include "qk_norm.cuh"

namespace sky {
namespace qkn {

template sky_status forward<__nv_bfloat16>(const sky_qk_norm_shape&, Params&, cudaStream_t);
template sky_status backward<__nv_bfloat16>(const sky_qk_norm_shape&, Params&, float*, float*, cudaStream_t);

}  // namespace qkn
}  // namespace sky
