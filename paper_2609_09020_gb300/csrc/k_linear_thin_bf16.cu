// k_linear_thin_bf16.cu -- the thin products of bfloat16 operands.
#include "k_linear_thin.cuh"

namespace pic {
namespace lin {

ThinKernel thin_kernel_bf16(int columns, bool fast) { return thin_kernel_of<__nv_bfloat16>(columns, fast); }

}  // namespace lin
}  // namespace pic
