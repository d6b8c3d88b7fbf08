// k_group_tc_f16.cu -- k_group_tc.cuh's kernels for __half.
#include "k_group_tc.cuh"

namespace pic {
namespace grp {

GtKernel group_kernel_f16(TcMode mode, int bn) { return group_kernel_of<__half>(mode, bn, 26); }

}  // namespace grp
}  // namespace pic
