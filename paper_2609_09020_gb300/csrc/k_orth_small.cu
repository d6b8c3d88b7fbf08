// k_orth_small.cu -- orthogonalised updates of small matrices: a CTA takes a matrix
// through norm, scaling and all steps by itself, with X, A and b A + c A^2 in shared
// memory as halves (orth.cuh), whichever side is the smaller one first, and warp-level
// MMAs (m16n8k16).  What bounds it is the chain: five steps are 15 products that wait on
// one another, some 0.6 us each for 64 x 64, where launches of the tiled kernels are 6 us
// each.  Measured: 192 matrices of 64 nets (64 x 7, 64 x 64, 3 x 64), fp32, 29 us (by tiles 105).
//
//   A, and b A + c A^2   a warp has 16 rows x 32 columns at a time
//   X = a X + B X        a warp has eight columns of all rows: what it reads of X is what
//                        it then writes, so that X stays in place
#include "orth.cuh"

namespace pic {
namespace orth {
namespace {

using lin::from_f32;
using lin::to_f32;

constexpr int kThreads = 256, kWarps = kThreads / 32;

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], const __half* p) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(p)))
               : "memory");
}
__device__ __forceinline__ void ldsm2_turned(uint32_t (&r)[2], const __half* p) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x2.trans.shared.b16 {%0, %1}, [%2];"
               : "=r"(r[0]), "=r"(r[1])
               : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(p)))
               : "memory");
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// A matrix of halves in shared memory, hi and behind it lo.
struct Held {
  __half* hi;
  int ld, lo;  // halves from hi to lo
  __device__ __forceinline__ float2 get(int at) const {
    const float2 h = __half22float2(*reinterpret_cast<const __half2*>(hi + at));
    const float2 l = __half22float2(*reinterpret_cast<const __half2*>(hi + lo + at));
    return make_float2(h.x + l.x, h.y + l.y);
  }
  __device__ __forceinline__ void put(int at, float x, float y) const {
    const __half2 h = __floats2half2_rn(x, y);
    const float2 f = __half22float2(h);
    *reinterpret_cast<__half2*>(hi + at) = h;
    *reinterpret_cast<__half2*>(hi + lo + at) = __floats2half2_rn(x - f.x, y - f.y);
  }
};

// Rows 16 i.. and columns 32 j.. of P P^T.  An MMA truncates what it adds: the products of
// small halves have sums of their own, and those of the others are 64 of K long and added to
// nearest (4 x 572, fp32, five steps: out is off by 1.1e-5 if all go into one, and by 1.8e-6 so).
constexpr int kRun = 64;
__device__ __forceinline__ void square(float (&acc)[4][4], const Held p, int i, int j, int deep, int lane) {
  float low[4][4] = {};
#pragma unroll
  for (int n = 0; n < 4; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[n][e] = 0.0f;
  const __half* pa = p.hi + (16 * i + (lane & 15)) * p.ld + (lane >> 4) * 8;
  const __half* pb = p.hi + (32 * j + (lane & 7) + (lane >> 4) * 8) * p.ld + (lane >> 3 & 1) * 8;
  for (int k0 = 0; k0 < deep; k0 += kRun) {
    float run[4][4] = {};
    const int k1 = min(deep, k0 + kRun);
#pragma unroll 2
    for (int k = k0; k < k1; k += 16) {
      uint32_t a[4], al[4], b[2][4], bl[2][4];
      ldsm4(a, pa + k);
#pragma unroll
      for (int h = 0; h < 2; ++h) ldsm4(b[h], pb + 16 * h * p.ld + k);
      ldsm4(al, pa + p.lo + k);
#pragma unroll
      for (int h = 0; h < 2; ++h) ldsm4(bl[h], pb + p.lo + 16 * h * p.ld + k);
#pragma unroll
      for (int n = 0; n < 4; ++n) mma(low[n], al, b[n / 2][n % 2 * 2], b[n / 2][n % 2 * 2 + 1]);
#pragma unroll
      for (int n = 0; n < 4; ++n) mma(low[n], a, bl[n / 2][n % 2 * 2], bl[n / 2][n % 2 * 2 + 1]);
#pragma unroll
      for (int n = 0; n < 4; ++n) mma(run[n], a, b[n / 2][n % 2 * 2], b[n / 2][n % 2 * 2 + 1]);
    }
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[n][e] += run[n][e];
  }
#pragma unroll
  for (int n = 0; n < 4; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[n][e] += low[n][e];
}

// STRIPS x 16 rows are those of X.
template <int STRIPS>
__device__ __forceinline__ void steps_of(const Held x, const Held a, const Held b, const int cols, const int steps, const Coefficients co) {
  constexpr int M = 16 * STRIPS;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  for (int step = 0; step < steps; ++step) {
    for (int u = warp; u < STRIPS * (M / 32); u += kWarps) {
      const int i = u % STRIPS, j = u / STRIPS;
      float acc[4][4];
      square(acc, x, i, j, cols, lane);
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          a.put((16 * i + g + 8 * h) * a.ld + 32 * j + 8 * n + 2 * t, acc[n][2 * h] * (1.0f / kScale),
                acc[n][2 * h + 1] * (1.0f / kScale));
    }
    __syncthreads();
    for (int u = warp; u < STRIPS * (M / 32); u += kWarps) {
      const int i = u % STRIPS, j = u / STRIPS;
      float acc[4][4];
      square(acc, a, i, j, M, lane);
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int at = (16 * i + g + 8 * h) * a.ld + 32 * j + 8 * n + 2 * t;
          const float2 old = a.get(at);
          b.put(at, fmaf(co.b, old.x, acc[n][2 * h] * (co.c / kScale)), fmaf(co.b, old.y, acc[n][2 * h + 1] * (co.c / kScale)));
        }
    }
    __syncthreads();
    for (int j = warp; j < cols / 8; j += kWarps) {
      float acc[STRIPS][4] = {};
#pragma unroll 1
      for (int k = 0; k < M; k += 16) {
        uint32_t q[2], ql[2];
        const __half* pq = x.hi + (k + (lane & 15)) * x.ld + 8 * j;
        ldsm2_turned(q, pq);
        ldsm2_turned(ql, pq + x.lo);
#pragma unroll
        for (int i = 0; i < STRIPS; ++i) {
          uint32_t p[4];
          const __half* pp = b.hi + (16 * i + (lane & 15)) * b.ld + (lane >> 4) * 8 + k;
          ldsm4(p, pp);
          uint32_t pl[4];
          ldsm4(pl, pp + b.lo);
          mma(acc[i], pl, q[0], q[1]);
          mma(acc[i], p, ql[0], ql[1]);
          mma(acc[i], p, q[0], q[1]);
        }
      }
      __syncwarp();
#pragma unroll
      for (int i = 0; i < STRIPS; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int at = (16 * i + g + 8 * h) * x.ld + 8 * j + 2 * t;
          const float2 old = x.get(at);
          x.put(at, fmaf(co.a, old.x, acc[i][2 * h] * (1.0f / kScale)), fmaf(co.a, old.y, acc[i][2 * h + 1] * (1.0f / kScale)));
        }
    }
    __syncthreads();
  }
}

// Every element of G (f(row, column, value)), or, without values, every place: neighbouring
// threads along a row, rows side by side where they are short, eight loads at a time.
template <typename T, bool VALUES, typename F>
__device__ __forceinline__ void for_elements(const Matrix& m, F f) {
  const int tx = m.cols >= 128 ? 128 : m.cols > 32 ? 64 : m.cols > 8 ? 32 : 8, ty = kThreads / tx;
  const int rows = m.rows, cols = m.cols;
  const long long ld = m.ld_grad;
  const T* g = static_cast<const T*>(m.grad);
  for (int c = threadIdx.x % tx; c < cols; c += tx)
    for (int r0 = threadIdx.x / tx; r0 < rows; r0 += 8 * ty) {
      T v[8];
      if (VALUES) {
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = r0 + u * ty < rows ? g[(r0 + u * ty) * ld + c] : from_f32<T>(0.0f);
      }
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (r0 + u * ty < rows) f(r0 + u * ty, c, VALUES ? to_f32(v[u]) : 0.0f);
    }
}

template <typename T>
__device__ __forceinline__ void load_scaled(const Matrix& m, const Held x, float eps, double* sums, float* factors) {
  // threads add squares in fp32, 64 at most, and go on in fp64; where a sum leaves the
  // range in which fp32 is good, all again in fp64
  double sum = 0.0;
  float s = 0.0f;
  int n = 0;
  bool bad = false, some = false;  // some: values that are not zero
  for_elements<T, true>(m, [&](int, int, float v) {
    s = fmaf(v, v, s);
    some |= v != 0.0f;
    if (++n == 64) {
      bad |= some && !(s >= 1e-28f && s <= 1e37f);
      sum += s, s = 0.0f, n = 0, some = false;
    }
  });
  bad |= some && !(s >= 1e-28f && s <= 1e37f);
  sum += s;
  if (bad) {
    sum = 0.0;
    for_elements<T, true>(m, [&](int, int, float v) { sum = fma(static_cast<double>(v), static_cast<double>(v), sum); });
  }
#pragma unroll
  for (int d = 16; d > 0; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {  // (in fp64, which is slow: by all threads this took as long as the steps)
    for (int w = 1; w < kWarps; ++w) sum += sums[w];
    norm_factors(sum, eps, factors[0], factors[1]);
  }
  __syncthreads();
  const float f0 = factors[0], f1 = factors[1];
  for_elements<T, true>(m, [&](int r, int c, float value) {
    const float v = value * f0 * (f1 * kScale);
    const int at = m.left ? r * x.ld + c : c * x.ld + r;
    const __half hi = __float2half_rn(v);
    x.hi[at] = hi;
    x.hi[x.lo + at] = __float2half_rn(v - __half2float(hi));
  });
}

template <typename T>
__device__ __forceinline__ void store_out(const Matrix& m, const Held x) {
  T* out = static_cast<T*>(m.out);
  for_elements<T, false>(m, [&](int r, int c, float) {
    const int at = m.left ? r * x.ld + c : c * x.ld + r;
    out[r * m.ld_out + c] = from_f32<T>((__half2float(x.hi[at]) + __half2float(x.hi[x.lo + at])) * (1.0f / kScale));
  });
}

__global__ void __launch_bounds__(kThreads) small_kernel(const Matrix* matrices, const int* list, int steps, Coefficients co,
                                                         float eps) {
  extern __shared__ __align__(16) __half halves[];
  __shared__ double sums[kWarps];
  __shared__ float factors[2];
  const Matrix m = matrices[list[blockIdx.x]];
  const SmallShape s = small_shape(m.m, m.left ? m.cols : m.rows);
  const Held x{halves, s.cols + 8, s.rows * (s.cols + 8)};
  const Held a{halves + 2 * s.rows * (s.cols + 8), s.rows + 8, s.rows * (s.rows + 8)};
  const Held b{a.hi + 2 * s.rows * (s.rows + 8), a.ld, a.lo};
  lin::wait_for_earlier();
  for (int i = threadIdx.x; i < 2 * s.rows * (s.cols + 8) / 8; i += kThreads) reinterpret_cast<uint4*>(halves)[i] = make_uint4(0, 0, 0, 0);
  // (load_scaled has a barrier before it writes to x)
  if (m.dtype == PIC_DTYPE_F32)
    load_scaled<float>(m, x, eps, sums, factors);
  else if (m.dtype == PIC_DTYPE_F16)
    load_scaled<__half>(m, x, eps, sums, factors);
  else
    load_scaled<__nv_bfloat16>(m, x, eps, sums, factors);
  __syncthreads();
  if (s.rows == 32)
    steps_of<2>(x, a, b, s.cols, steps, co);
  else if (s.rows == 64)
    steps_of<4>(x, a, b, s.cols, steps, co);
  else
    steps_of<8>(x, a, b, s.cols, steps, co);
  if (m.dtype == PIC_DTYPE_F32)
    store_out<float>(m, x);
  else if (m.dtype == PIC_DTYPE_F16)
    store_out<__half>(m, x);
  else
    store_out<__nv_bfloat16>(m, x);
}

}  // namespace

int launch_small(const Matrix* matrices, const int* list, int n, int smem, int steps, const Coefficients& co, float eps,
                 lin::Chain& s) {
  if (n == 0) return PIC_OK;
  if (lin::allow_smem(reinterpret_cast<const void*>(small_kernel), 53, kSmallMost) != PIC_OK) return PIC_ERR_CUDA;
  return s.launch(small_kernel, dim3(n), kThreads, smem, matrices, list, steps, co, eps);
}

}  // namespace orth
}  // namespace pic
