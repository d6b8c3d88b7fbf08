// group.cuh -- what the kernels of the grouped linear layer (include/pic_group.h)
// share: the table of groups and the launch interfaces between their translation
// units.
#pragma once

#include "linear.cuh"
#include "pic_group.h"

namespace pic {
namespace grp {

using lin::Chain;
using lin::wait_for_earlier;
using lin::Waits;

constexpr int kMaxGroups = PIC_MAX_GROUPS;

// A CTA's table of groups, in shared memory: first rows, and the number of tiles of
// `unit` rows before each group's.  An offset counts as the largest so far, within [0, rows].
struct GroupTable {
  int start[kMaxGroups + 1];
  int tiles[kMaxGroups + 1];
  int scan[32];

  __device__ __forceinline__ int rows(int g) const { return start[g + 1] - start[g]; }
  // the group that has tile t, of those in the table
  __device__ __forceinline__ int find(int t, int groups) const {
    int lo = 0, hi = groups - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (tiles[mid + 1] <= t)
        lo = mid + 1;
      else
        hi = mid;
    }
    return lo;
  }
};

// Inclusive scan over the block's threads (at most 1024, whole warps).
template <bool MAX>
__device__ __forceinline__ int block_scan(int v, int* scratch) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const auto join = [](int a, int b) { return MAX ? max(a, b) : a + b; };
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int o = __shfl_up_sync(0xffffffffu, v, d);
    if (lane >= d) v = join(v, o);
  }
  __syncthreads();
  if (lane == 31) scratch[warp] = v;
  __syncthreads();
  int before = 0;  // offsets and counts are not negative
  for (int w = 0; w < warp && w < warps; ++w) before = join(before, scratch[w]);
  return join(before, v);
}

// Filled by all threads of the block; tiles of a group without rows: `least`.  Block
// 0 reports offsets that are not as they must be.
__device__ __forceinline__ void make_table(GroupTable& t, const long long* offsets, int groups, long long rows, int unit,
                                           int least, int* status) {
  const int each = (groups + blockDim.x) / blockDim.x;  // of groups + 1 offsets
  const int first = threadIdx.x * each, last = min(first + each, groups + 1);
  int most = 0;
  bool bad = false;
  for (int i = first; i < last; ++i) {
    const long long o = offsets[i];
    bad |= o < 0 || o > rows;
    const int held = static_cast<int>(min(max(o, 0LL), rows));
    bad |= held < most;
    most = max(most, held);
    t.start[i] = most;
  }
  // the largest of the threads before
  const int upto = block_scan<true>(most, t.scan);
  int before = __shfl_up_sync(0xffffffffu, upto, 1);
  if ((threadIdx.x & 31) == 0) {
    before = 0;
    for (int w = 0; w < static_cast<int>(threadIdx.x >> 5); ++w) before = max(before, t.scan[w]);
  }
  for (int i = first; i < last; ++i) {
    bad |= t.start[i] < before;
    t.start[i] = max(t.start[i], before);
  }
  if (bad && blockIdx.x == 0) atomicOr(status + 1, 1);
  __syncthreads();
  const auto tiles_of = [&](int g) { return t.rows(g) == 0 ? least : (t.rows(g) - 1) / unit + 1; };
  int count = 0;
  for (int g = first; g < min(last, groups); ++g) count += tiles_of(g);
  int at = block_scan<false>(count, t.scan) - count;
  for (int g = first; g < last; ++g) {
    t.tiles[g] = at;
    if (g < groups) at += tiles_of(g);
  }
  __syncthreads();
}

// Products of any types, strides and sizes.  By rows: y[i][j] = sum_k a(i, k) b_g(j, k)
// for the rows i of group g, a(i, k) at a[i * a_i + k], b_g(j, k) at b[g * b_group + j
// * b_j + k * b_k], with the layer's epilogue.  Else y_g[i][j] = sum over the group's
// rows k of a(k, i) b(k, j), a at a[k * a_i + i], b at b[k * b_k + j].
struct GroupProduct {
  bool by_rows;
  const void* a;
  long long a_i;
  const void* a_pre;  // of few rows' gradients: a is multiplied by act'(a_pre); or null
  long long a_pre_i;
  int a_act;
  const void* b;
  long long b_group, b_j, b_k;
  long long rows;  // of all groups, and around them
  long long I;     // columns of a that are rows of y_g (not by_rows)
  long long J, K;  // K: by_rows
  int groups;
  const long long* offsets;
  const void* bias;
  long long bias_group;
  void* y;
  long long ldy, y_group;
  void* pre;
  long long ldpre;
  int act;
  int* status;
};
// (16-bit types by rows only: tc_product takes all their sums.)
int any_product(const GroupProduct& p, int dtype, Chain& s);

// Few rows in a group, eight at a time: any types, strides and sizes.  few_dw makes db too (y
// or db null: not that one).
int few_forward(const GroupProduct& p, int dtype, Chain& s);
int few_dx(const GroupProduct& p, int dtype, Chain& s);
int few_dw(const GroupProduct& p, void* db, long long db_group, int dtype, Chain& s);

// On the tensor cores: 16-bit types.
constexpr long long kTcMostK = 16384;  // of K that one accumulator sums up
bool tc_takes(const GroupProduct& p, int dtype);
long long tc_workspace(const GroupProduct& p, int dtype);
int tc_product(const GroupProduct& p, int dtype, void* ws, const Waits& waits, Chain& s);

// Where part `item` of group g is among the parts of the groups that have several; the
// calling warp's lanes count together.
__device__ __forceinline__ long long part_slot(const GroupTable& t, int g, int item, int chunk, int lane) {
  int whole = 0;
  for (int i = lane; i < g; i += 32) whole += t.rows(i) <= chunk;
  return item - __reduce_add_sync(0xffffffffu, whole);
}

// The sums of the groups' parts (of groups with more than `chunk` rows), in order.  A
// tile's part is [rank][panel of 64 columns][quarter][16][32 rows][4 columns].
struct JoinParams {
  const long long* offsets;
  long long rows, I, J, tiles_i, tiles_j;
  int groups, chunk, bn;
  const float4* parts;
  void* y;
  long long ldy, y_group;
  int* status;
};
// rows: of a tile.
int join_parts(const JoinParams& q, int rows, int dtype, Chain& s);

// fp32 on the tensor cores, cut into planes first.
bool planes_takes(const GroupProduct& p, int dtype);
int planes_product(const GroupProduct& p, lin::Arena& ws, bool launch, const Waits& waits, Chain& s);
// dx and dw of the same dz (their a).
int planes_gradients(const GroupProduct& dx, const GroupProduct& dw, lin::Arena& ws, bool launch, const Waits& waits, Chain& s);

// dz[i][j] = dy act'(pre), rounded (dz null: not written; its rows are on 16-byte
// boundaries and written to the next one), and db_g, the sums of the unrounded dz over
// each group's rows (db null: none).
struct GroupGradAct {
  const void* dy;
  long long lddy;
  const void* pre;
  long long ldpre;
  void* dz;
  long long lddz;
  void* db;
  long long db_group;
  float* parts;
  long long rows, J;
  int groups, act;
  const long long* offsets;
  int* status;
};
long long grad_act_workspace(const GroupGradAct& g, int dtype);
int grad_act(const GroupGradAct& g, int dtype, Chain& s);

}  // namespace grp
}  // namespace pic
