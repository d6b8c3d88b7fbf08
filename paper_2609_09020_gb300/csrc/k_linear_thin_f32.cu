// k_linear_thin_f32.cu -- the thin products of fp32 operands.
#include "k_linear_thin.cuh"

namespace pic {
namespace lin {

ThinKernel thin_kernel_f32(int columns, bool fast) { return thin_kernel_of<float>(columns, fast); }

}  // namespace lin
}  // namespace pic
