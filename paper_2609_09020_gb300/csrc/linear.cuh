// linear.cuh -- what the kernels of the linear layer (include/pic_linear.h)
// share: element types, activations and the launch interfaces between their
// translation units.
#pragma once

#include <cstdint>
#include <type_traits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "pic_common.cuh"
#include "pic_gelu_grad.cuh"
#include "pic_linear.h"

namespace pic {
namespace lin {

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

// A 16- or 32-bit load under a predicate, 0 where it is off, without a branch: the
// loads around it need not wait for it.  (With branches, eight elements that are
// put together are eight memory latencies.)
__device__ __forceinline__ uint32_t load_if(const uint16_t* p, bool on) {
  uint16_t v;
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %2, 0;\n\tmov.u16 %0, 0;\n\t@q ld.global.u16 %0, [%1];\n\t}"
               : "=h"(v)
               : "l"(p), "r"(static_cast<uint32_t>(on)));
  return v;
}
__device__ __forceinline__ uint32_t load_if(const uint32_t* p, bool on) {
  uint32_t v;
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %2, 0;\n\tmov.u32 %0, 0;\n\t@q ld.global.u32 %0, [%1];\n\t}"
               : "=r"(v)
               : "l"(p), "r"(static_cast<uint32_t>(on)));
  return v;
}

// 16 bytes from a 16-byte boundary.  (If one of them is in a tensor, all are in its
// allocation.)
__device__ __forceinline__ uint4 load_if16(const void* p, bool on) {
  uint4 v;
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %5, 0;\n\tmov.u32 %0, 0;\n\tmov.u32 %1, 0;\n\tmov.u32 %2, 0;\n\tmov.u32 %3, 0;\n\t"
      "@q ld.global.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
      : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
      : "l"(p), "r"(static_cast<uint32_t>(on)));
  return v;
}
// Keeps `bytes` bytes of w, from its beginning.
template <typename T>
__device__ __forceinline__ void keep_bytes(uint32_t (&w)[4], int bytes) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = bytes >= 4 * i + 4 ? w[i] : sizeof(T) == 2 && bytes >= 4 * i + 2 ? w[i] & 0xffffu : 0u;
}

// 16 bytes of a row as loaded: one aligned piece (ON16), or the two that have them.
template <bool ON16>
struct Piece16 {
  uint4 lo, hi;
  __device__ __forceinline__ void load(const char* at, int bytes) {  // bytes of the row from `at` on, may be <= 0
    if constexpr (ON16) {
      lo = load_if16(at, bytes > 0);
    } else {
      const int m = static_cast<int>(reinterpret_cast<uintptr_t>(at) & 15);
      lo = load_if16(at - m, bytes > 0);
      hi = load_if16(at - m + 16, m + min(bytes, 16) > 16);
    }
  }
  // the 16 bytes from byte `m` of the two on
  template <typename T>
  __device__ __forceinline__ void get(int m, uint32_t (&w)[4]) const {
    if constexpr (ON16) {
      w[0] = lo.x, w[1] = lo.y, w[2] = lo.z, w[3] = lo.w;
    } else {
      const uint32_t v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
      const bool by2 = (m & 8) != 0, by1 = (m & 4) != 0;
      uint32_t u[6], s[5];
#pragma unroll
      for (int i = 0; i < 6; ++i) u[i] = by2 ? v[i + 2] : v[i];
#pragma unroll
      for (int i = 0; i < 5; ++i) s[i] = by1 ? u[i + 1] : u[i];
      const uint32_t bits = (m & 2) * 8;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = sizeof(T) == 4 ? s[i] : __funnelshift_r(s[i], s[i + 1], bits);
    }
  }
};

// Round to nearest even.
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Two values of a 16-bit type in a word, the first in the low half.
template <typename T>
__device__ __forceinline__ uint32_t pack2_of(float lo, float hi) {
  uint32_t d;
  if constexpr (std::is_same<T, __half>::value)
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
template <typename T>
__device__ __forceinline__ float2 unpack2_of(uint32_t v) {
  if constexpr (std::is_same<T, __half>::value)
    return __half22float2(*reinterpret_cast<const __half2*>(&v));
  else
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}

// act(z), NaN for NaN.  GELU is max(z, 0) - a Phi(-a), a = |z|: no infinity
// meets a zero.  EXACT (fp32 outputs): a Phi(-a) is a power times a polynomial, off
// by 1e-7 with the evaluation's roundings; else the framework's polynomial exponent,
// off by at most 5e-7, far below half an ulp of a 16-bit output but for outputs
// below 2e-3 (fp16: 1e-3) in size.  (erfcf, with its branches, made the fp32
// 2048 x 1024 -> 4096 layer 20 us slower.)
template <bool EXACT>
__device__ __forceinline__ float act_value(float z, int act) {
  if (act == PIC_ACT_NONE) return z;
  if (act == PIC_ACT_RELU) return relu_nan(z);
  if constexpr (EXACT) {
    const float a = fminf(fabsf(z), kGeluGradA);
    float r = gelu_c32(0);
#pragma unroll
    for (int i = 1; i <= kGeluDeg32; ++i) r = fmaf(r, a, gelu_c32(i));
    return fmaf(-ex2_approx(a * a * kGeluGradPower), a >= kGeluGradA ? 0.0f : r, relu_nan(z));
  } else {
    return gelu_approx(z);
  }
}

// GELU of two values, its polynomial in packed instructions; as act_value rounds.
template <bool EXACT>
__device__ __forceinline__ float2 gelu2(float2 z) {
  if constexpr (EXACT) {
    const float2 a = make_float2(fminf(fabsf(z.x), kGeluGradA), fminf(fabsf(z.y), kGeluGradA));
    const unsigned long long a2 = pack2(a.x, a.y);
    unsigned long long r = pack2(gelu_c32(0), gelu_c32(0));
#pragma unroll
    for (int i = 1; i <= kGeluDeg32; ++i) r = fma2(r, a2, pack2(gelu_c32(i), gelu_c32(i)));
    const float2 q = unpack2(r), e = unpack2(mul2(mul2(a2, a2), pack2(kGeluGradPower, kGeluGradPower)));
    return make_float2(fmaf(-ex2_approx(e.x), a.x >= kGeluGradA ? 0.0f : q.x, relu_nan(z.x)),
                       fmaf(-ex2_approx(e.y), a.y >= kGeluGradA ? 0.0f : q.y, relu_nan(z.y)));
  } else {
    return unpack2(gelu_approx2(pack2(z.x, z.y)));
  }
}

// dy act'(z): a derivative of zero gives zero whatever dy is.  At z = NaN GELU's is NaN,
// and ReLU's is zero, as [z > 0] is.  EXACT (fp32): off by the roundings of the evaluation, about 1e-7; else by
// at most 5e-7, far below the rounding of dz to 16 bits.
template <bool EXACT>
__device__ __forceinline__ float act_grad(float dy, float z, int act) {
  if (act == PIC_ACT_NONE) return dy;
  if (act == PIC_ACT_RELU) return z > 0.0f ? dy : 0.0f;
  float a;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(a) : "f"(fabsf(z)), "f"(kGeluGradA));
  float p = EXACT ? gelu_grad_c32(0) : gelu_grad_c(0);
#pragma unroll
  for (int i = 1; i <= (EXACT ? kGeluGradDeg32 : kGeluGradDeg); ++i)
    p = fmaf(p, a, EXACT ? gelu_grad_c32(i) : gelu_grad_c(i));
  // (at a = A, 1 - t rounds to 1)
  const float t = p * ex2_approx(a * a * kGeluGradPower);
  return z <= -kGeluGradA ? 0.0f : dy * (z < 0.0f ? t : 1.0f - t);
}

// The same for two values: the polynomial runs on both in packed instructions.
template <bool EXACT>
__device__ __forceinline__ float2 act_grad2(float2 dy, float2 z, int act) {
  if (act != PIC_ACT_GELU) return make_float2(act_grad<EXACT>(dy.x, z.x, act), act_grad<EXACT>(dy.y, z.y, act));
  float2 a;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(a.x) : "f"(fabsf(z.x)), "f"(kGeluGradA));
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(a.y) : "f"(fabsf(z.y)), "f"(kGeluGradA));
  const unsigned long long a2 = pack2(a.x, a.y);
  const float c0 = EXACT ? gelu_grad_c32(0) : gelu_grad_c(0);
  unsigned long long p = pack2(c0, c0);
#pragma unroll
  for (int i = 1; i <= (EXACT ? kGeluGradDeg32 : kGeluGradDeg); ++i) {
    const float c = EXACT ? gelu_grad_c32(i) : gelu_grad_c(i);
    p = fma2(p, a2, pack2(c, c));
  }
  const float2 e = unpack2(mul2(mul2(a2, a2), pack2(kGeluGradPower, kGeluGradPower)));
  const float2 t2 = unpack2(mul2(p, pack2(ex2_approx(e.x), ex2_approx(e.y))));
  const float dx = z.x < 0.0f ? t2.x : 1.0f - t2.x, dz = z.y < 0.0f ? t2.y : 1.0f - t2.y;
  return make_float2(z.x <= -kGeluGradA ? 0.0f : dy.x * dx, z.y <= -kGeluGradA ? 0.0f : dy.y * dz);
}

// One matrix product C[i][j] = sum_k A(i, k) B(j, k) with what follows it.
// A(i, k) is at a[i * a_i + k * a_k], B(j, k) at b[j * b_j + k * b_k]; one of
// the two strides is 1.
struct Product {
  const void* a;
  const void* b;
  long long a_i, a_k, b_j, b_k;
  long long I, J, K;
  // epilogue: z = C + bias[j]; pre = z; y = act(z) + residual
  const void* bias;
  const void* residual;
  long long ldr;
  void* y;
  long long ldy;
  void* pre;
  long long ldpre;
  int act;
  // A(i, k) = a(i, k) act'(a_pre(i, k)), where there is an a_pre (few_product only)
  const void* a_pre;
  long long a_pre_i;
  int a_act;
  // A is w and B is x: C(i, j) belongs at [j][i] of y, pre and the residual, and to
  // bias[i] (set and read by the fp32 products through registers only)
  int swapped;
};

// Launches a kernel in clusters of `cluster` CTAs along x.
inline int launch_kernel(const void* fn, long long grid, int threads, int smem, int cluster, void** args, cudaStream_t s) {
  const dim3 g(static_cast<unsigned>(grid)), b(threads);
  if (cluster == 1) return cudaLaunchKernel(fn, g, b, args, smem, s) == cudaSuccess ? PIC_OK : PIC_ERR_CUDA;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = cluster;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = g;
  cfg.blockDim = b;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelExC(&cfg, fn, args) == cudaSuccess ? PIC_OK : PIC_ERR_CUDA;
}

// Every function returns a pic_status; `ws` is device workspace.
// What the kernels' bounded waits share: polls that one makes, the device word that
// is set to 1 when one gives up, and the test hook, which has one epilogue warp of
// the first tile withhold an arrival.
struct Waits {
  int* status;
  unsigned spin_limit;
  int test_fault;
};

// On the tensor cores.
long long tc_workspace(const Product& p, int dtype);
int tc_product(const Product& p, int dtype, void* ws, const Waits& waits, cudaStream_t s);

// 16-bit types with at most kFewRows rows of A, which must lie along K: every
// element of B is read once, straight into the operands of warp-level MMAs.
constexpr int kFewRows = 15;
bool few_takes(const Product& p);
int few_product(const Product& p, int dtype, cudaStream_t s);

// The same for fp32 and at most kFewRows32 rows, on the FP32 cores.
constexpr int kFewRows32 = 8;
bool few32_takes(const Product& p);
int few32_product(const Product& p, cudaStream_t s);

// Narrow matrices of any number of rows: at most 128 columns and 128 of K, both along K.
bool thin_takes(const Product& p, int dtype);
int thin_product(const Product& p, int dtype, cudaStream_t s);

// dw = dz^T x and db of at most kFewRows rows, dz = dy act'(z) not rounded before.
struct OuterGrad {
  const void* dy;
  long long lddy;
  const void* pre;
  long long ldpre;
  const void* x;
  long long ldx;
  void* dw;  // null: not asked for, as for db
  long long lddw;
  void* db;
  long long I, N, K;
  int act;
};
int outer_grad(const OuterGrad& g, int dtype, cudaStream_t s);

// dz[i][j] = dy act'(z), rounded (dz null: not written), and db[j], the sums of
// the unrounded dz over the rows (db null: none); parts is workspace.  Rows of dz
// are on 16-byte boundaries and written to the next one.
struct GradAct {
  const void* dy;
  long long lddy;
  const void* pre;
  long long ldpre;
  void* dz;
  long long lddz;
  void* db;
  float* parts;
  long long I, J;
  int act;
};
long long grad_act_workspace(const GradAct& g, int dtype);
int grad_act(const GradAct& g, int dtype, cudaStream_t s);

// The whole gradient of a narrow layer over many rows, in one pass.
struct NarrowGrad {
  const void* dy;
  long long lddy;
  const void* pre;
  long long ldpre;
  const void* x;
  long long ldx;
  const void* w;
  long long ldw;
  void* dx;  // null: not asked for, as for dw and db
  long long lddx;
  void* dw;
  long long lddw;
  void* db;
  long long I;
  int N, K, act;
};
bool narrow_takes(const NarrowGrad& g, int dtype);
long long narrow_workspace(const NarrowGrad& g, int dtype);
int narrow_grad(const NarrowGrad& g, int dtype, void* ws, const Waits& waits, cudaStream_t s);

}  // namespace lin
}  // namespace pic
