// k_group_tc_bf16.cu -- k_group_tc.cuh's kernels for __nv_bfloat16.
#include "k_group_tc.cuh"

namespace pic {
namespace grp {

GtKernel group_kernel_bf16(TcMode mode, int bn) { return group_kernel_of<__nv_bfloat16>(mode, bn, 35); }

}  // namespace grp
}  // namespace pic
