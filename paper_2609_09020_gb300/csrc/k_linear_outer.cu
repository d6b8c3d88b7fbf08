// k_linear_outer.cu -- dw and db of a layer over few rows (up to kFewRows):
//
//   dw[n][k] = sum_m dz[m][n] x[m][k],  db[n] = sum_m dz[m][n],  dz = dy act'(z)
//
// Bound by writing dw once.  A block takes 64 rows of dw and 32 x 16 bytes of their
// columns; its rows of x and dz are in shared memory as fp32, and a warp holds 8
// rows x 16 bytes a lane in registers, so that a value of x that is read from shared
// memory serves eight sums.  Where dw's rows do not start on 16-byte boundaries a
// lane's columns are 32 apart instead, and its stores one element each.
#include "linear.cuh"

namespace pic {
namespace lin {
namespace {

constexpr int kThreads = 256;
constexpr int kRows = 64, kWarpRows = 8;

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads, 2) outer_kernel(const OuterGrad g, long long col_blocks) {
  constexpr int kV = 16 / sizeof(T), kCols = 32 * kV;
  __shared__ __align__(16) float xs[kFewRows][kCols];
  __shared__ __align__(16) float ds[kFewRows][kRows];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rows = static_cast<int>(g.I);
  const long long n0 = blockIdx.x / col_blocks * kRows, k0 = blockIdx.x % col_blocks * kCols;
  for (int e = threadIdx.x; e < rows * kRows; e += kThreads) {
    const int m = e / kRows;
    const long long n = n0 + e % kRows;
    float d = 0.0f;
    if (n < g.N) {
      d = to_f32(static_cast<const T*>(g.dy)[m * g.lddy + n]);
      if (g.act != PIC_ACT_NONE) d = act_grad<sizeof(T) == 4>(d, to_f32(static_cast<const T*>(g.pre)[m * g.ldpre + n]), g.act);
    }
    ds[m][e % kRows] = d;
  }
  if (g.dw)
    for (int e = threadIdx.x; e < rows * kCols; e += kThreads) {
      const int m = e / kCols;
      const long long k = k0 + e % kCols;
      xs[m][e % kCols] = k < g.K ? to_f32(static_cast<const T*>(g.x)[m * g.ldx + k]) : 0.0f;
    }
  __syncthreads();
  if (g.db && k0 == 0 && threadIdx.x < kRows && n0 + threadIdx.x < g.N) {
    float s = 0.0f;
    for (int m = 0; m < rows; ++m) s += ds[m][threadIdx.x];
    static_cast<T*>(g.db)[n0 + threadIdx.x] = from_f32<T>(s);
  }
  if (!g.dw) return;
  float acc[kWarpRows][kV] = {};
  for (int m = 0; m < rows; ++m) {
    float x[kV], d[kWarpRows];
#pragma unroll
    for (int e = 0; e < kV; e += 4) {
      if constexpr (VEC) {
        const float4 f = *reinterpret_cast<const float4*>(&xs[m][lane * kV + e]);
        x[e] = f.x, x[e + 1] = f.y, x[e + 2] = f.z, x[e + 3] = f.w;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[e + i] = xs[m][lane + 32 * (e + i)];
      }
    }
#pragma unroll
    for (int r = 0; r < kWarpRows; r += 4) {
      const float4 f = *reinterpret_cast<const float4*>(&ds[m][warp * kWarpRows + r]);
      d[r] = f.x, d[r + 1] = f.y, d[r + 2] = f.z, d[r + 3] = f.w;
    }
#pragma unroll
    for (int r = 0; r < kWarpRows; ++r)
#pragma unroll
      for (int e = 0; e < kV; ++e) acc[r][e] = fmaf(d[r], x[e], acc[r][e]);
  }
#pragma unroll
  for (int r = 0; r < kWarpRows; ++r) {
    const long long n = n0 + warp * kWarpRows + r;
    if (n >= g.N) break;
    T* o = static_cast<T*>(g.dw) + n * g.lddw + k0;
    if constexpr (VEC) {
      if (k0 + (lane + 1) * kV <= g.K) {
        uint4 w;
        T* t = reinterpret_cast<T*>(&w);
#pragma unroll
        for (int e = 0; e < kV; ++e) t[e] = from_f32<T>(acc[r][e]);
        *reinterpret_cast<uint4*>(o + lane * kV) = w;
      } else {
#pragma unroll
        for (int e = 0; e < kV; ++e)
          if (k0 + lane * kV + e < g.K) o[lane * kV + e] = from_f32<T>(acc[r][e]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < kV; ++e)
        if (k0 + lane + 32 * e < g.K) o[lane + 32 * e] = from_f32<T>(acc[r][e]);
    }
  }
}

template <typename T>
int run(const OuterGrad& g, cudaStream_t s) {
  constexpr int kCols = 32 * 16 / sizeof(T);
  const long long col_blocks = g.dw ? (g.K + kCols - 1) / kCols : 1, blocks = col_blocks * ((g.N + kRows - 1) / kRows);
  if (blocks > 0x7fffffffLL) return PIC_ERR_INVALID_ARG;
  const bool vec = reinterpret_cast<uintptr_t>(g.dw) % 16 == 0 && g.lddw * sizeof(T) % 16 == 0;
  if (vec)
    outer_kernel<T, true><<<static_cast<unsigned>(blocks), kThreads, 0, s>>>(g, col_blocks);
  else
    outer_kernel<T, false><<<static_cast<unsigned>(blocks), kThreads, 0, s>>>(g, col_blocks);
  return cudaGetLastError() == cudaSuccess ? PIC_OK : PIC_ERR_CUDA;
}

}  // namespace

int outer_grad(const OuterGrad& g, int dtype, cudaStream_t s) {
  if (dtype == PIC_DTYPE_F32) return run<float>(g, s);
  return dtype == PIC_DTYPE_F16 ? run<__half>(g, s) : run<__nv_bfloat16>(g, s);
}

}  // namespace lin
}  // namespace pic
