// k_group_any.cu -- grouped products of any stride and size on the FP32 cores (products
// of rows of every type, sums over rows of fp32): tiles of 64 x 64, 16 of K at a time through shared memory, sixteen sums a
// thread.  CTAs are persistent, with the table of groups in shared memory, and take
// tiles one after another.  Measured: 16 of K of such a tile take from 1.3 us to 4 with four
// CTAs on each SM; fp32 400 x 300 -> 300 in four groups 23 us.
#include "group.cuh"

namespace pic {
namespace grp {
namespace {

using lin::act_value;
using lin::from_f32;
using lin::to_f32;

constexpr int kTile = 64, kDeep = 16, kThreads = 256;
constexpr int kSms = 152;

template <typename T, bool ROWS>
__global__ void __launch_bounds__(kThreads) any_kernel(const GroupProduct p) {
  constexpr bool EXACT = sizeof(T) == 4;
  __shared__ GroupTable table;
  __shared__ __align__(16) float sa[kDeep][kTile + 4], sb[kDeep][kTile + 4];
  make_table(table, p.offsets, p.groups, p.rows, kTile, 0, p.status);
  wait_for_earlier();
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const long long tiles_j = (p.J + kTile - 1) / kTile, tiles_i = (p.I + kTile - 1) / kTile;
  const long long work = ROWS ? table.tiles[p.groups] * tiles_j : p.groups * tiles_i * tiles_j;
  const T *a = static_cast<const T*>(p.a), *b = static_cast<const T*>(p.b);
  for (long long w = blockIdx.x; w < work; w += gridDim.x) {
    const long long tj = w % tiles_j, t = w / tiles_j;
    const int g = ROWS ? table.find(static_cast<int>(t), p.groups) : static_cast<int>(t / tiles_i);
    const long long first = table.start[g], len = table.rows(g);
    const long long i0 = (ROWS ? t - table.tiles[g] : t % tiles_i) * kTile, j0 = tj * kTile;
    const long long I = ROWS ? len : p.I, K = ROWS ? p.K : len;
    const T* bg = ROWS ? b + g * p.b_group : b + first * p.b_k;
    float acc[4][4] = {};
    // a thread's elements of the next 16 of K, on their way while these are multiplied
    constexpr int kEach = kTile * kDeep / kThreads;
    const bool along = ROWS && p.b_k == 1;  // neighbouring threads along what is contiguous
    T na[kEach], nb[kEach];
    const auto fetch = [&](long long k0) {
#pragma unroll
      for (int u = 0; u < kEach; ++u) {
        const int e = threadIdx.x + u * kThreads;
        const int ka = ROWS ? e % kDeep : e / kTile, ia = ROWS ? e / kDeep : e % kTile;
        na[u] = nb[u] = from_f32<T>(0.0f);
        if (i0 + ia < I && k0 + ka < K) {
          const long long row = first + (ROWS ? i0 + ia : k0 + ka), col = ROWS ? k0 + ka : i0 + ia;
          na[u] = a[row * p.a_i + col];
        }
        const int kb = along ? e % kDeep : e / kTile, jb = along ? e / kDeep : e % kTile;
        if (j0 + jb < p.J && k0 + kb < K) nb[u] = bg[(j0 + jb) * p.b_j + (k0 + kb) * p.b_k];
      }
    };
    if (K > 0) fetch(0);
    for (long long k0 = 0; k0 < K; k0 += kDeep) {
#pragma unroll
      for (int u = 0; u < kEach; ++u) {
        const int e = threadIdx.x + u * kThreads;
        const int ka = ROWS ? e % kDeep : e / kTile, ia = ROWS ? e / kDeep : e % kTile;
        const int kb = along ? e % kDeep : e / kTile, jb = along ? e / kDeep : e % kTile;
        sa[ka][ia] = to_f32(na[u]);
        sb[kb][jb] = to_f32(nb[u]);
      }
      __syncthreads();
      if (k0 + kDeep < K) fetch(k0 + kDeep);
#pragma unroll
      for (int k = 0; k < kDeep; ++k) {
        const float4 u = *reinterpret_cast<const float4*>(&sa[k][4 * ty]), v = *reinterpret_cast<const float4*>(&sb[k][4 * tx]);
        const float x[4] = {u.x, u.y, u.z, u.w}, y[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[r][c] = fmaf(x[r], y[c], acc[r][c]);
      }
      __syncthreads();
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const long long i = i0 + 4 * ty + r;
      if (i >= I) break;
      const long long row = ROWS ? first + i : i;
      T* y = static_cast<T*>(p.y) + (ROWS ? 0 : g * p.y_group) + row * p.ldy;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const long long j = j0 + 4 * tx + c;
        if (j >= p.J) break;
        float v = acc[r][c];
        if (p.bias) v += to_f32(static_cast<const T*>(p.bias)[g * p.bias_group + j]);
        if (p.pre) static_cast<T*>(p.pre)[row * p.ldpre + j] = from_f32<T>(v);
        y[j] = from_f32<T>(act_value<EXACT>(v, p.act));
      }
    }
  }
}

template <typename T, bool ROWS>
int run(const GroupProduct& p, Chain& s) {
  const long long tiles_j = (p.J + kTile - 1) / kTile, tiles_i = (p.I + kTile - 1) / kTile;
  const long long most = ROWS ? ((p.rows + kTile - 1) / kTile + p.groups) * tiles_j : p.groups * tiles_i * tiles_j;
  const unsigned grid = static_cast<unsigned>(most < 4 * kSms ? most : 4 * kSms);
  return s.launch(any_kernel<T, ROWS>, dim3(grid), kThreads, 0, p);
}

}  // namespace

int any_product(const GroupProduct& p, int dtype, Chain& s) {
  if (dtype == PIC_DTYPE_F32) return p.by_rows ? run<float, true>(p, s) : run<float, false>(p, s);
  // (sums of 16-bit types are the tensor cores', whatever their size)
  if (!p.by_rows) return PIC_ERR_INVALID_ARG;
  return dtype == PIC_DTYPE_F16 ? run<__half, true>(p, s) : run<__nv_bfloat16, true>(p, s);
}

}  // namespace grp
}  // namespace pic
