// k_clip.cu -- the global gradient norm and clipping (include/pic_clip.h).
// The handle cuts its tensors into chunks of kChunk elements.  Every thread
// block of the first kernel sums the squares of its chunks: fp32 within a
// thread's part of a chunk (at most kChunk / kThreads squares), fp64 from
// there on.  The blocks of the second kernel each add the blocks' sums in the
// same order, and scale their chunks: no atomics, one result.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

#include "linear.cuh"
#include "pic_clip.h"

struct ClipChunk {
  const void* grad;
  void* out;
  int count;
  int dtype;
};

struct pic_clipper {
  int device;
  int n_chunks;
  int blocks;
  ClipChunk* chunks;  // device
  double* parts;      // device, [blocks]
};

namespace {

using pic::lin::from_f32;
using pic::lin::to_f32;

constexpr int kThreads = 512;
constexpr int kChunk = 32768;
constexpr int kBlocks = 304;

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double sums[kThreads / 32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (threadIdx.x % 32 == 0) sums[threadIdx.x / 32] = v;
  __syncthreads();
  double t = 0.0;
  for (int i = 0; i < kThreads / 32; ++i) t += sums[i];
  __syncthreads();
  return t;
}

template <typename T>
__device__ double thread_squares(const ClipChunk& c) {
  const T* g = static_cast<const T*>(c.grad);
  float s = 0.0f;
  for (int i = threadIdx.x; i < c.count; i += kThreads) {
    const float v = to_f32(g[i]);
    s = fmaf(v, v, s);
  }
  // fp32 left its range: squares below 2^-126 lose bits (2^-90: none that
  // matter beside others of the sum's size), above 2^128 it is infinite
  if (s < 0x1p+127f && (s > 0x1p-90f)) return s;
  double d = 0.0;
  for (int i = threadIdx.x; i < c.count; i += kThreads) {
    const double v = to_f32(g[i]);
    d = fma(v, v, d);
  }
  return d;
}

__global__ void __launch_bounds__(kThreads) squares_kernel(const ClipChunk* chunks, int n, double* parts) {
  double d = 0.0;
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const ClipChunk c = chunks[i];
    if (c.dtype == PIC_DTYPE_F32)
      d += thread_squares<float>(c);
    else if (c.dtype == PIC_DTYPE_F16)
      d += thread_squares<__half>(c);
    else
      d += thread_squares<__nv_bfloat16>(c);
  }
  d = block_sum(d);
  if (threadIdx.x == 0) parts[blockIdx.x] = d;
}

template <typename T>
__device__ void scale(const ClipChunk& c, float coef) {
  const T* g = static_cast<const T*>(c.grad);
  T* o = static_cast<T*>(c.out);
  for (int i = threadIdx.x; i < c.count; i += kThreads) o[i] = from_f32<T>(to_f32(g[i]) * coef);
}

__global__ void __launch_bounds__(kThreads) scale_kernel(const ClipChunk* chunks, int n, const double* parts,
                                                         int n_parts, float max_norm, float* norm_out) {
  double d = 0.0;
  for (int i = threadIdx.x; i < n_parts; i += kThreads) d += parts[i];
  const float norm = static_cast<float>(sqrt(block_sum(d)));
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
  // not fminf: coef is NaN where norm is
  float coef = max_norm / (norm + 1e-6f);
  if (coef > 1.0f || isinf(max_norm)) coef = 1.0f;
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const ClipChunk c = chunks[i];
    if (coef == 1.0f && c.grad == c.out) continue;
    if (c.dtype == PIC_DTYPE_F32)
      scale<float>(c, coef);
    else if (c.dtype == PIC_DTYPE_F16)
      scale<__half>(c, coef);
    else
      scale<__nv_bfloat16>(c, coef);
  }
}

long long elem_bytes(int dtype) { return dtype == PIC_DTYPE_F32 ? 4 : 2; }

struct Range {
  uintptr_t lo, hi;
  bool out;
  int tensor;
};

// Outputs may overlap nothing but their own gradient, and that exactly.
bool outputs_disjoint(const pic_clip_tensor* t, int n) {
  std::vector<Range> r;
  for (int i = 0; i < n; ++i) {
    if (t[i].count == 0) continue;
    const uintptr_t bytes = static_cast<uintptr_t>(t[i].count * elem_bytes(t[i].dtype));
    const uintptr_t g = reinterpret_cast<uintptr_t>(t[i].grad), o = reinterpret_cast<uintptr_t>(t[i].out);
    r.push_back({o, o + bytes, true, i});
    if (g != o) r.push_back({g, g + bytes, false, i});
  }
  std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.lo < b.lo; });
  uintptr_t out_end = 0, any_end = 0;  // the furthest end so far of the outputs, of all
  for (const Range& a : r) {
    if (a.lo < out_end || (a.out && a.lo < any_end)) return false;
    any_end = std::max(any_end, a.hi);
    if (a.out) out_end = std::max(out_end, a.hi);
  }
  return true;
}

}  // namespace

extern "C" {

int pic_clip_create(const pic_clip_tensor* tensors, int n, pic_clipper** out) {
  if (!out) return PIC_ERR_INVALID_ARG;
  *out = nullptr;
  if (n < 0 || (n > 0 && !tensors)) return PIC_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i) {
    const pic_clip_tensor& t = tensors[i];
    if (t.dtype != PIC_DTYPE_F32 && t.dtype != PIC_DTYPE_F16 && t.dtype != PIC_DTYPE_BF16) return PIC_ERR_INVALID_ARG;
    if (t.count < 0 || t.count > (1LL << 45)) return PIC_ERR_INVALID_ARG;
    if (t.count == 0) continue;
    if (!t.grad || !t.out || reinterpret_cast<uintptr_t>(t.grad) % elem_bytes(t.dtype) ||
        reinterpret_cast<uintptr_t>(t.out) % elem_bytes(t.dtype))
      return PIC_ERR_INVALID_ARG;
  }
  int dev = 0, major = 0, minor = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) {
    cudaGetLastError();
    return PIC_ERR_UNSUPPORTED;
  }
  if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev) != cudaSuccess) {
    cudaGetLastError();
    return PIC_ERR_CUDA;
  }
  if (major != 10 || minor != 3) return PIC_ERR_UNSUPPORTED;
  try {
    if (!outputs_disjoint(tensors, n)) return PIC_ERR_INVALID_ARG;
    std::vector<ClipChunk> chunks;
    for (int i = 0; i < n; ++i) {
      const pic_clip_tensor& t = tensors[i];
      const long long e = elem_bytes(t.dtype);
      for (long long at = 0; at < t.count; at += kChunk) {
        if (chunks.size() >= 0x7fffffffu) return PIC_ERR_INVALID_ARG;
        chunks.push_back({static_cast<const char*>(t.grad) + at * e, static_cast<char*>(t.out) + at * e,
                          static_cast<int>(std::min<long long>(kChunk, t.count - at)), t.dtype});
      }
    }
    pic_clipper* c = new pic_clipper{};
    c->device = dev;
    c->n_chunks = static_cast<int>(chunks.size());
    c->blocks = std::max(1, std::min(kBlocks, c->n_chunks));
    const size_t bytes = chunks.size() * sizeof(ClipChunk);
    if (cudaMalloc(&c->parts, c->blocks * sizeof(double)) != cudaSuccess ||
        (bytes && cudaMalloc(&c->chunks, bytes) != cudaSuccess)) {
      cudaGetLastError();
      pic_clip_destroy(c);
      return PIC_ERR_ALLOC;
    }
    if (bytes && cudaMemcpy(c->chunks, chunks.data(), bytes, cudaMemcpyHostToDevice) != cudaSuccess) {
      cudaGetLastError();
      pic_clip_destroy(c);
      return PIC_ERR_CUDA;
    }
    *out = c;
    return PIC_OK;
  } catch (const std::bad_alloc&) {
    return PIC_ERR_ALLOC;
  } catch (...) {
    return PIC_ERR_INVALID_ARG;
  }
}

int pic_clip(pic_clipper* c, float max_norm, float* norm, void* stream) {
  if (!c || !norm || reinterpret_cast<uintptr_t>(norm) % 4 || !(max_norm >= 0.0f)) return PIC_ERR_INVALID_ARG;
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) {
    cudaGetLastError();
    return PIC_ERR_CUDA;
  }
  if (dev != c->device) return PIC_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  squares_kernel<<<c->blocks, kThreads, 0, s>>>(c->chunks, c->n_chunks, c->parts);
  scale_kernel<<<c->blocks, kThreads, 0, s>>>(c->chunks, c->n_chunks, c->parts, c->blocks, max_norm, norm);
  return cudaGetLastError() == cudaSuccess ? PIC_OK : PIC_ERR_CUDA;
}

void pic_clip_destroy(pic_clipper* c) {
  if (!c) return;
  cudaFree(c->chunks);
  cudaFree(c->parts);
  delete c;
}

}  // extern "C"
