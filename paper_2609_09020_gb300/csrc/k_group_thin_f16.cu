// k_group_thin_f16.cu -- the grouped thin products of IEEE half operands.
#include "k_linear_thin.cuh"

namespace pic {
namespace lin {

ThinKernel thin_group_kernel_f16(int columns, bool fast) { return thin_kernel_of<__half, true>(columns, fast); }

}  // namespace lin
}  // namespace pic
