// k_linear_tc_f16.cu -- the tensor-core products of IEEE half operands.
#include "k_linear_tc.cuh"

namespace pic {
namespace lin {

const void* tc_kernel_f16(int bn, bool long_parts) {
  return long_parts ? tc_kernel_of<__half, true>(bn) : tc_kernel_of<__half, false>(bn);
}

}  // namespace lin
}  // namespace pic
