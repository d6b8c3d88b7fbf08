// k_linear_tc_bf16.cu -- the tensor-core products of bfloat16 operands.
#include "k_linear_tc.cuh"

namespace pic {
namespace lin {

const void* tc_kernel_bf16(int bn, bool long_parts) {
  return long_parts ? tc_kernel_of<__nv_bfloat16, true>(bn) : tc_kernel_of<__nv_bfloat16, false>(bn);
}

}  // namespace lin
}  // namespace pic
