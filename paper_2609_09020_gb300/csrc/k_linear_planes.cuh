// k_linear_planes.cuh -- what the launch of k_linear_planes.cu's kernels needs.
#pragma once

#include "k_linear_tc.cuh"

namespace pic {
namespace lin {

// Tiles of 256 rows (128 for each CTA of a pair) and 128 columns.
constexpr int kPlRows = 256, kPlCols = 128;
constexpr int kPlBlock = 128;  // rows and columns of a stored matrix that share a mark

// An fp32 matrix as it was, and the marks of its blocks.
struct PlOperand {
  const float* m;
  long long ld;       // elements from one stored row to the next
  const int* marks;   // [row blocks][col_blocks], nonzero: the block has a value from kCutLimit on
  int col_blocks;
};
struct PlOperands {
  PlOperand a, b;
};

struct PlKernel {
  const void* fn;  // takes (TcParams, TcMaps, PlOperands); a and b are maps of three planes
  int threads, smem;
};
PlKernel planes_kernel_info();

// planes[3][rows][ld_out] (bfloat16) and marks, from the fp32 matrix m [rows][cols].
struct CutMatrix {
  const float* m;
  long long ld, rows, cols;
  void* planes;
  long long ld_out;
  int* marks;
};
int cut_planes(const CutMatrix (&m)[2], cudaStream_t s);

}  // namespace lin
}  // namespace pic
