// orth.cuh -- what the kernels of orthogonalised updates (include/pic_orth.h)
// share: how X, A and b A + c A^2 are held, the handle's tables and the launch
// interfaces between their translation units.
//
// A value v is held as kScale v in one IEEE half, or in two, the second the nearest half
// to what the first leaves (22 bits in all).  Singular values of at most 2 and |b s^2| +
// |c s^4| of at most 12 bound every element, so that none reaches the largest half; with
// kScale = 4096 an element of the usual size, 1 / sqrt(max(rows, cols)), is far above
// the smallest.
//
// The first X is G times a power of two, of which bfloat16's and half's values are exact; the
// rest of 1 / (|G| + eps), `rest` in [1, 2], is in the factors of the first step.  What X's
// second half is for: the steps multiply what is lost by rounding X outside the singular
// vectors that G has by a = 3.44 each, and where G has few directions that would show.  With
// operands of one half (bfloat16, if not small) the last two steps but one leave it out: 2^-12 times 12 is
// no more than out's rounding.
//
// A and b A + c A^2 are symmetric, and only their blocks on and below the diagonal are
// kept (blocks as high as a tile); operands above it are loaded turned.
#pragma once

#include <cuda.h>

#include "k_linear_tc.cuh"
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
  int halves;        // that A, b A + c A^2 and operands of products have
  int part0, parts;  // its runs of squares
  int on16;          // rows of grad start on 16-byte boundaries
  float* rest;       // of 1 / (|G| + eps)
  __half* x[2];      // [2][rows][ldx]
  __half* a;         // [halves][m][lda]
  __half* b;
  long long ldx, lda;
};

// 32 rows (or what there is of them) and up to kPieceCols columns of a matrix, for the
// norm, and for the scaling after it.
constexpr int kPieceCols = 512;
struct Piece {
  int matrix, row0, col0;
};

// The tensor maps of a matrix: of operands in boxes of 64 x 64 of one half, of epilogues'
// panels in boxes of 32 rows x 64.
enum MapOf { kMapX = 0, kMapOtherX = 1, kMapA = 2, kMapB = 3, kMapPanel = 4, kMaps = 8 };

// A tile of a product, or a part of one along K.
struct Job {
  int matrix;
  int i, j;            // first row and column of the tile
  int p_map, q_map;    // of the operands; kMapX: of the X that is read
  int p_mn, q_mn;      // the operand lies along i (j)
  int p_half, q_half;  // of the operand there are blocks on and below the diagonal only
  int halves;
  int k0, k1;          // slices
  int part, parts;     // along K
  int slot;            // the first of the tile's parts in the workspace
  int take;            // slices that an accumulator of two halves sums up before it is taken over
};
static_assert(sizeof(Job) == 64, "a job is read in four loads");

using lin::wait_for_earlier;

struct Coefficients {
  float a, b, c;
};

// |G| + eps from the sum of squares: X is G times f0 times f1, a power of two first, then
// what is left, so that no finite norm leaves fp32's range on the way.
__device__ __forceinline__ void norm_factors(double sum, float eps, float& f0, float& f1) {
  const double norm = sqrt(sum) + eps;
  int e = 0;
  if (norm > 0.0 && norm < 1e300) frexp(norm, &e);
  e = min(max(e, -126), 126);
  f0 = static_cast<float>(ldexp(1.0, -e));
  f1 = static_cast<float>(ldexp(1.0, e) / norm);
}

// Matrices that one CTA takes through all steps by itself: the smaller side at most 128,
// and X, A and b A + c A^2, in two halves each, within kSmallMost bytes of shared memory.
struct SmallShape {
  int rows, cols;  // of X in shared memory, and 8 more halves from row to row
};
__host__ __device__ inline SmallShape small_shape(int m, int n) {
  return {m <= 32 ? 32 : m <= 64 ? 64 : 128, (n + 31) / 32 * 32};
}
constexpr int kSmallMost = 220 * 1024;
__host__ inline long long small_bytes(int m, int n) {
  const SmallShape s = small_shape(m, n);
  return 4LL * s.rows * (s.cols + 8) + 8LL * s.rows * (s.rows + 8);
}
int launch_small(const Matrix* matrices, const int* list, int n, int smem, int steps, const Coefficients& co, float eps,
                 lin::Chain& s);

// Stages of a step: A = X X^T, B = b A + c A^2, X = a X + B X.
enum Stage { kGram = 0, kPolynomial = 1, kUpdate = 2 };

constexpr int kAcquiredFirst = 512;  // up to so many maps, a CTA's threads acquire them all while it waits for the kernel before
struct StageParams {
  const Matrix* matrices;
  const CUtensorMap* maps;  // [matrices][kMaps]
  int n_maps;
  const Job* jobs;
  int n;
  Coefficients co;
  int from;   // which X is read
  int first, last;  // of the steps: X is still to be multiplied by `rest`; X goes to out
  int lo_from, lo_to;  // whether X has second halves, of matrices with operands of one half
  float4* parts;
  unsigned* counters;
  Waits waits;
};
// Tiles: 128 rows x 64 or 128 columns by a CTA; 256 x 256, or, in A and A^2 of lists with
// operands of two halves, 256 x 128, by a pair.
enum TileShape { k64 = 0, k128 = 1, kPair256 = 2, kPair128 = 3, kShapes = 4 };
// both: of k64 and k128, that some matrices have operands of two halves.
int launch_stage(Stage stage, TileShape shape, bool both, const StageParams& q, lin::Chain& s);

}  // namespace orth
}  // namespace pic
