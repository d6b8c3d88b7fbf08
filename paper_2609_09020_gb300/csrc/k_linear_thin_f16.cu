// k_linear_thin_f16.cu -- the thin products of IEEE half operands.
#include "k_linear_thin.cuh"

namespace pic {
namespace lin {

ThinKernel thin_kernel_f16(int columns, bool fast) { return thin_kernel_of<__half, false>(columns, fast); }

}  // namespace lin
}  // namespace pic
