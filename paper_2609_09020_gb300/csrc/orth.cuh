// orth.cuh -- what the kernels of orthogonalised updates (include/pic_orth.h)
// share: how X, A and b A + c A^2 are held, the handle's tables and the launch
// interfaces between their translation units.
//
// A value v is held as kScale v in one IEEE half, or in two, the second the nearest half
// to what the first leaves (22 bits in all).  Singular values of at most 2 and |b s^2| +
// |c s^4| of at most 12 bound every element, so that none reaches the largest half; with
// kScale = 4096 an element of the usual size, 1 / sqrt(max(rows, cols)), is far above
// the smallest.
#pragma once

#include <cuda.h>

#include "linear.cuh"
#include "pic_orth.h"

namespace pic {
namespace orth {

using lin::Waits;

constexpr float kScale = 4096.0f;

// A matrix of the list with its room in the handle's workspace.
struct Matrix {
  const void* grad;
  void* out;
  long long ld_grad, ld_out;
  int rows, cols, dtype;
  int m;             // the smaller side
  int left;          // rows <= cols: A = X X^T
  int halves;        // that operands of products have (X itself is always held in two)
  int part0, parts;  // its runs of squares
  __half* x[2];      // [2][rows][ldx]
  __half* a;         // [2][m][lda]
  __half* b;
  long long ldx, lda;
};

// A piece of a matrix for the norm, and for the scaling after it.
struct Piece {
  int matrix, row0, rows, col0, cols;
};

// The tensor maps of a matrix, all in boxes of 64 x 64 of one half.
enum MapOf { kMapX = 0, kMapOtherX = 1, kMapA = 2, kMapB = 3, kMaps = 4 };

// A tile of a product, or a part of one along K.
struct Job {
  int matrix;
  int i, j;            // first row and column of the tile
  int p_map, q_map;    // of the operands; kMapX: of the X that is read
  int p_mn, q_mn;      // the operand lies along i (j)
  int halves;
  int k0, k1;          // slices
  int part, parts;     // along K
  int slot;            // the first of the tile's parts in the workspace
  int mirror;          // the tile is written at (j, i) too
  int pad[2];
};
static_assert(sizeof(Job) == 64, "a job is read in four loads");

struct Coefficients {
  float a, b, c;
};

// Stages of a step: A = X X^T, B = b A + c A^2, X = a X + B X.
enum Stage { kGram = 0, kPolynomial = 1, kUpdate = 2 };

struct StageParams {
  const Matrix* matrices;
  const CUtensorMap* maps;  // [matrices][kMaps]
  const Job* jobs;
  int n;
  Coefficients co;
  int from;   // which X is read
  int last;   // X goes to out
  float4* parts;
  unsigned* counters;
  Waits waits;
};
// With tiles of bn columns: 64 and 128 by one CTA, 256 by a pair.
int launch_stage(Stage stage, int bn, const StageParams& q, cudaStream_t s);

}  // namespace orth
}  // namespace pic
