// k_linear_tc_f16.cu -- the tensor-core products of IEEE half operands.
#include "k_linear_tc.cuh"

namespace pic {
namespace lin {

const void* tc_kernel_f16(int bn) { return tc_kernel_of<__half>(bn); }

}  // namespace lin
}  // namespace pic
