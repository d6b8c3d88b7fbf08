// k_group_thin_bf16.cu -- the grouped thin products of bfloat16 operands.
#include "k_linear_thin.cuh"

namespace pic {
namespace lin {

ThinKernel thin_group_kernel_bf16(int columns, bool fast) { return thin_kernel_of<__nv_bfloat16, true>(columns, fast); }

}  // namespace lin
}  // namespace pic
