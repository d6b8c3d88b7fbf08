// cut3.cuh -- fp32 values as three bfloat16 pieces, for products on the tensor
// cores.
//
// A value is hi + mid + lo, each the nearest bfloat16 (8 significant bits) to what the
// ones before left: mid is at most 2^-8 and lo at most 2^-16 of the value, and the sum is
// the value exactly, but for bits below 2^-133, bfloat16's smallest step: values below
// 2^-110 are held in fewer than 24 bits.  Of the nine products of pieces the six
// largest are formed,
//     hi hi + (hi mid + mid hi) + (mid mid + hi lo + lo hi);
// the three left out are below 2^-23 of the product, of either sign.  (By truncation the
// pieces would be up to 2^-7 and 2^-15, the rest up to 2^-21 and always of the product's
// sign; it takes as many instructions.)  Six MMAs of bfloat16 at 2.25 PFLOP/s nominal are
// 375 TFLOP/s of fp32, five times what the FP32 cores do.
//
// A tensor core truncates when it adds to an accumulator.  So within a slice of 64
// of K the products of small pieces come first (cut_a, cut_b), which leaves few
// truncations at the sum's full size, and after every 128 of K the accumulators are
// taken over into registers and added there to nearest.  Measured on 2048 x 1024 ->
// 4096 (root mean square error, relative): 6.0e-7 with terms of random sign, 5.2e-7 with
// positive ones; fp32 FMAs in order give 6.2e-7.  (With pieces by truncation: 6.8e-7 and
// 2.1e-6; with those and all products of 16 of K together and takeovers every 256, 2.1e-6
// and more; takeovers every 64 take a quarter more time.)
#pragma once

#include <cstdint>

namespace pic {
namespace lin {

constexpr int kPieces = 3;
// pieces of A and of B of the six products, in order
__host__ __device__ constexpr int cut_a(int t) {
  constexpr int p[6] = {2, 0, 1, 1, 0, 0};
  return p[t];
}
__host__ __device__ constexpr int cut_b(int t) {
  constexpr int p[6] = {0, 2, 1, 0, 1, 0};
  return p[t];
}

// From here on hi would be infinite: such values, like infinite and NaN ones, take no
// part in products of pieces.
constexpr uint32_t kCutLimit = 0x7f7f8000u;

// Two values rounded to bfloat16, packed (a in the low half).
__device__ __forceinline__ uint32_t nearest2(float a, float b) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(b), "f"(a));
  return d;
}
// The three pieces of two values below kCutLimit in size, packed (a in the low half).
__device__ __forceinline__ void cut3(uint32_t a, uint32_t b, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
  float ra = __uint_as_float(a), rb = __uint_as_float(b);
  hi = nearest2(ra, rb);
  ra -= __uint_as_float(hi << 16), rb -= __uint_as_float(hi & 0xffff0000u);
  mid = nearest2(ra, rb);
  ra -= __uint_as_float(mid << 16), rb -= __uint_as_float(mid & 0xffff0000u);
  lo = nearest2(ra, rb);
}

// Adds to v[c] the sum over elements [k0, k1) of K for row i
// and N columns from col0, on the FP32 cores, eight columns at a time.  a, b: where
// A(0, 0) and B(0, 0) are; strides per row and per K.  Its callers ask for one
// takeover's K, 128 at most, so that the waits of a CTA's other warps do not grow with K.
template <int N>
__device__ __forceinline__ void sum_again(float (&v)[N], const float* a, long long a_i, long long a_k, const float* b,
                                          long long b_j, long long b_k, long long i, long long I, long long col0,
                                          long long J, long long k0, long long k1) {
  static_assert(N % 8 == 0, "columns in eights");
  a += i * a_i + k0 * a_k, b += col0 * b_j + k0 * b_k;
  const int n = i < I ? static_cast<int>(k1 - k0) : 0, cols = static_cast<int>(min(static_cast<long long>(N), J - col0));
#pragma unroll
  for (int c = 0; c < N; c += 8) {
    float s[8] = {};
#pragma unroll 1
    for (int k = 0; k < n; ++k) {
      const float x = a[k * a_k];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (c + u < cols) s[u] = fmaf(x, b[(c + u) * b_j + k * b_k], s[u]);
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) v[c + u] += s[u];
  }
}

}  // namespace lin
}  // namespace pic
