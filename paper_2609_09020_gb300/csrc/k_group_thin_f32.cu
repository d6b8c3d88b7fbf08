// k_group_thin_f32.cu -- the grouped thin products of fp32 operands.
#include "k_linear_thin.cuh"

namespace pic {
namespace lin {

ThinKernel thin_group_kernel_f32(int columns, bool fast) { return thin_kernel_of<float, true>(columns, fast); }

}  // namespace lin
}  // namespace pic
