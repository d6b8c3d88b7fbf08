// orth.cuh -- what the kernels of orthogonalised updates (include/pic_orth.h)
// share: the handle's tables and the launch interfaces between their translation
// units.
#pragma once

#include "linear.cuh"
#include "pic_orth.h"

namespace pic {
namespace orth {

// A matrix of the list with its room in the handle's workspace.
struct Matrix {
  const void* grad;
  void* out;
  long long ld_grad, ld_out;
  int rows, cols, dtype;
  int m;         // the smaller side
  int left;      // rows <= cols: A = X X^T
  int part0, parts;  // its runs of squares
  float* x[2];   // [rows][ldx]
  float* a;      // [m][lda]
  float* b;
  long long ldx, lda;
};

// A piece of a matrix for the norm, and for the scaling after it.
struct Piece {
  int matrix, row0, rows, col0, cols;
};

// A tile of a product.
struct Tile {
  int matrix, i, j;
};

struct Coefficients {
  float a, b, c, eps;
};

}  // namespace orth
}  // namespace pic
