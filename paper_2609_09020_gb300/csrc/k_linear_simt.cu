// k_linear_simt.cu -- the linear layer's products on the FP32 cores, for any
// type, size, stride and alignment.  A block computes a 64 x 64 tile of C with
// 256 threads (4 x 4 values each) from 64 x 16 slices of A and B in shared
// memory, widened to fp32 there.  A product with few tiles and a long sum
// (dw over the pixels of an image) is cut along K: parts go to the workspace
// in fp32 and are added in order by a second kernel, so that the result does
// not depend on the blocks' order.
#include "linear.cuh"

namespace pic {
namespace lin {
namespace {

constexpr int kTile = 64;
constexpr int kStep = 16;
constexpr int kThreads = 256;
constexpr int kBlocks = 608;  // what a cut product aims for: 4 blocks per SM

struct SimtParams {
  Product p;
  long long tiles_i, tiles_j;
  long long k_part;  // K of one part, a multiple of kStep
  float* parts;      // [splits][I][J], or null: the epilogue runs here
};

template <typename T>
__device__ __forceinline__ void finish(const Product& p, long long i, long long j, float v) {
  if (p.bias) v += to_f32(static_cast<const T*>(p.bias)[j]);
  if (p.pre) static_cast<T*>(p.pre)[i * p.ldpre + j] = from_f32<T>(v);
  v = act_value<true>(v, p.act);
  if (p.residual) v += to_f32(static_cast<const T*>(p.residual)[i * p.ldr + j]);
  static_cast<T*>(p.y)[i * p.ldy + j] = from_f32<T>(v);
}

// Rows [row0, row0 + 64) and columns [k0, k0 + 16) of a matrix into
// s[k][row], zero outside.  Threads run along whichever direction has unit stride.
template <typename T>
__device__ __forceinline__ void load_slice(float (*s)[kTile + 4], const T* m, long long sr, long long sk,
                                           long long row0, long long rows, long long k0, long long k1) {
#pragma unroll
  for (int e = 0; e < kTile * kStep / kThreads; ++e) {
    const int idx = threadIdx.x + e * kThreads;
    const int r = sk == 1 ? idx / kStep : idx % kTile;
    const int k = sk == 1 ? idx % kStep : idx / kTile;
    float v = 0.0f;
    if (row0 + r < rows && k0 + k < k1) v = to_f32(m[(row0 + r) * sr + (k0 + k) * sk]);
    s[k][r] = v;
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) simt_kernel(const SimtParams q) {
  __shared__ float sa[kStep][kTile + 4], sb[kStep][kTile + 4];
  const Product& p = q.p;
  const long long ti = blockIdx.x / q.tiles_j, tj = blockIdx.x % q.tiles_j;
  const long long i0 = ti * kTile, j0 = tj * kTile;
  const long long k0 = blockIdx.y * q.k_part;
  const long long k1 = min(p.K, k0 + q.k_part);
  const int r = threadIdx.x / 16 * 4, c = threadIdx.x % 16 * 4;
  float acc[4][4] = {};
  for (long long k = k0; k < k1; k += kStep) {
    load_slice(sa, static_cast<const T*>(p.a), p.a_i, p.a_k, i0, p.I, k, k1);
    load_slice(sb, static_cast<const T*>(p.b), p.b_j, p.b_k, j0, p.J, k, k1);
    __syncthreads();
#pragma unroll
    for (int kk = 0; kk < kStep; ++kk) {
      const float4 a = *reinterpret_cast<const float4*>(&sa[kk][r]);
      const float4 b = *reinterpret_cast<const float4*>(&sb[kk][c]);
      const float av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) acc[x][y] = fmaf(av[x], bv[y], acc[x][y]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int x = 0; x < 4; ++x)
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const long long i = i0 + r + x, j = j0 + c + y;
      if (i >= p.I || j >= p.J) continue;
      if (q.parts)
        q.parts[(blockIdx.y * p.I + i) * p.J + j] = acc[x][y];
      else
        finish<T>(p, i, j, acc[x][y]);
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) join_kernel(const SimtParams q, int splits) {
  const Product& p = q.p;
  const long long n = p.I * p.J;
  for (long long e = blockIdx.x * static_cast<long long>(kThreads) + threadIdx.x; e < n;
       e += static_cast<long long>(gridDim.x) * kThreads) {
    float v = 0.0f;
    for (int s = 0; s < splits; ++s) v += q.parts[s * n + e];
    finish<T>(p, e / p.J, e % p.J, v);
  }
}

struct Plan {
  long long tiles_i, tiles_j, k_part;
  int splits;
};

Plan plan(const Product& p) {
  Plan r;
  r.tiles_i = (p.I + kTile - 1) / kTile;
  r.tiles_j = (p.J + kTile - 1) / kTile;
  const int s = split_count(r.tiles_i * r.tiles_j, p.K, 4 * kStep, kBlocks);
  r.k_part = ((p.K + s - 1) / s + kStep - 1) / kStep * kStep;
  r.splits = static_cast<int>((p.K + r.k_part - 1) / r.k_part);
  return r;
}

template <typename T>
int run(const Product& p, void* ws, cudaStream_t s) {
  const Plan r = plan(p);
  if (r.tiles_i * r.tiles_j > 0x7fffffffLL) return PIC_ERR_INVALID_ARG;
  SimtParams q{p, r.tiles_i, r.tiles_j, r.k_part, r.splits > 1 ? static_cast<float*>(ws) : nullptr};
  simt_kernel<T><<<dim3(static_cast<unsigned>(r.tiles_i * r.tiles_j), r.splits), kThreads, 0, s>>>(q);
  if (r.splits > 1) {
    long long b = (p.I * p.J + kThreads - 1) / kThreads;
    if (b > 4096) b = 4096;
    join_kernel<T><<<static_cast<unsigned>(b), kThreads, 0, s>>>(q, r.splits);
  }
  return cudaGetLastError() == cudaSuccess ? PIC_OK : PIC_ERR_CUDA;
}

}  // namespace

long long simt_workspace(const Product& p) {
  const Plan r = plan(p);
  return r.splits > 1 ? r.splits * p.I * p.J * 4 : 0;
}

int simt_product(const Product& p, int dtype, void* ws, cudaStream_t s) {
  if (dtype == PIC_DTYPE_F32) return run<float>(p, ws, s);
  if (dtype == PIC_DTYPE_F16) return run<__half>(p, ws, s);
  return run<__nv_bfloat16>(p, ws, s);
}

}  // namespace lin
}  // namespace pic
