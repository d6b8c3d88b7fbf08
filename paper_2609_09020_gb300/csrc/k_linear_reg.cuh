// k_linear_reg.cuh -- what the launch of k_linear_reg.cu's kernel needs.
#pragma once

#include "k_linear_tc.cuh"

namespace pic {
namespace lin {

constexpr int kRegRows = 128, kRegCols = 64;  // a tile

// Operands as the loaders read them, beside the launch's TcParams.
struct RegOperands {
  const void* a;
  const void* b;
  long long lda, ldb;  // elements from one stored row to the next
  int vec_a, vec_b;    // rows on 16-byte boundaries
};

// Takes (TcParams, TcMaps, RegOperands); of the maps it reads y and pre.
struct RegKernel {
  const void* fn;
  int threads, smem;
};
RegKernel reg_kernel_info();

}  // namespace lin
}  // namespace pic
