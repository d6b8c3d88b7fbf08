// k_linear_grad.cu -- the elementwise part of the linear layer's gradient:
// dz = dy act'(z) and its column sums db.  A block takes 32 columns and a run
// of rows, eight at a time; its column sums go to the workspace and a second
// kernel adds the blocks' sums in a fixed order.
#include "linear.cuh"

namespace pic {
namespace lin {
namespace {

constexpr int kCols = 32, kRows = 8;
constexpr int kRun = 512;  // rows of one block

template <typename T>
__global__ void __launch_bounds__(kCols* kRows) grad_act_kernel(const GradAct g) {
  __shared__ float sums[kRows][kCols];
  const int tx = threadIdx.x % kCols, ty = threadIdx.x / kCols;
  const long long col_blocks = (g.J + kCols - 1) / kCols;
  const long long row_block = blockIdx.x / col_blocks;
  const long long j = blockIdx.x % col_blocks * kCols + tx;
  const long long i0 = row_block * kRun;
  const long long i1 = min(g.I, i0 + kRun);
  float sum = 0.0f;
  if (j < g.J)
    for (long long i = i0 + ty; i < i1; i += kRows) {
      float d = to_f32(static_cast<const T*>(g.dy)[i * g.lddy + j]);
      if (g.act != PIC_ACT_NONE) d = act_grad(d, to_f32(static_cast<const T*>(g.pre)[i * g.ldpre + j]), g.act);
      if (g.dz) static_cast<T*>(g.dz)[i * g.lddz + j] = from_f32<T>(d);
      sum += d;
    }
  if (!g.parts) return;
  sums[ty][tx] = sum;
  __syncthreads();
  if (ty == 0 && j < g.J) {
    for (int r = 1; r < kRows; ++r) sum += sums[r][tx];
    g.parts[row_block * g.J + j] = sum;
  }
}

template <typename T>
__global__ void __launch_bounds__(1024) sum_parts_kernel(const float* parts, long long blocks, long long J, T* out) {
  __shared__ float sums[32][33];
  const int tx = threadIdx.x % 32, ty = threadIdx.x / 32;
  const long long j = blockIdx.x * 32LL + tx;
  float sum = 0.0f;
  if (j < J)
    for (long long b = ty; b < blocks; b += 32) sum += parts[b * J + j];
  sums[ty][tx] = sum;
  __syncthreads();
  if (ty == 0 && j < J) {
    for (int r = 1; r < 32; ++r) sum += sums[r][tx];
    out[j] = from_f32<T>(sum);
  }
}

}  // namespace

long long grad_act_blocks(long long I, long long J) {
  (void)J;
  return (I + kRun - 1) / kRun;
}

int grad_act(const GradAct& g, int dtype, cudaStream_t s) {
  const long long blocks = grad_act_blocks(g.I, g.J) * ((g.J + kCols - 1) / kCols);
  if (blocks > 0x7fffffffLL) return PIC_ERR_INVALID_ARG;
  const unsigned grid = static_cast<unsigned>(blocks);
  if (dtype == PIC_DTYPE_F32)
    grad_act_kernel<float><<<grid, kCols * kRows, 0, s>>>(g);
  else if (dtype == PIC_DTYPE_F16)
    grad_act_kernel<__half><<<grid, kCols * kRows, 0, s>>>(g);
  else
    grad_act_kernel<__nv_bfloat16><<<grid, kCols * kRows, 0, s>>>(g);
  return cudaGetLastError() == cudaSuccess ? PIC_OK : PIC_ERR_CUDA;
}

int sum_parts(const float* parts, long long blocks, long long J, void* out, int dtype, cudaStream_t s) {
  const unsigned grid = static_cast<unsigned>((J + 31) / 32);
  if (dtype == PIC_DTYPE_F32)
    sum_parts_kernel<<<grid, 1024, 0, s>>>(parts, blocks, J, static_cast<float*>(out));
  else if (dtype == PIC_DTYPE_F16)
    sum_parts_kernel<<<grid, 1024, 0, s>>>(parts, blocks, J, static_cast<__half*>(out));
  else
    sum_parts_kernel<<<grid, 1024, 0, s>>>(parts, blocks, J, static_cast<__nv_bfloat16*>(out));
  return cudaGetLastError() == cudaSuccess ? PIC_OK : PIC_ERR_CUDA;
}

}  // namespace lin
}  // namespace pic
