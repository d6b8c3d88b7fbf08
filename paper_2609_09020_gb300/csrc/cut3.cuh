// cut3.cuh -- fp32 values as three bfloat16 pieces, for products on the tensor
// cores.
//
// A value is hi + mid + lo, each the top 8 significant bits of what the ones
// before left, by truncation: 24 bits in all, so the sum is the value exactly
// (pieces below 2^-126 lose bits).  Of the nine products of pieces the six
// largest are formed,
//     hi hi + (hi mid + mid hi) + (mid mid + hi lo + lo hi);
// the three left out are below 3 x 2^-24 of the product.  Six MMAs of bfloat16 at
// 2.25 PFLOP/s nominal are 375 TFLOP/s of fp32, five times what the FP32 cores do.
//
// A tensor core truncates when it adds to an accumulator.  So within a slice of 64
// of K the products of small pieces come first (cut_a, cut_b), which leaves few
// truncations at the sum's full size, and after every 128 of K the accumulators are
// taken over into registers and added there to nearest.  Measured on 2048 x 1024 ->
// 4096 (root mean square error, relative): 2.1e-6 with all products of 16 of K
// together and takeovers every 256; 7e-7 as it is; 1.6e-7 with takeovers every 64,
// which take a quarter more time; fp32 FMAs in order give 6.2e-7.
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

// The three pieces of two finite fp32 values, packed (a in the low half).
__device__ __forceinline__ void cut3(uint32_t a, uint32_t b, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
  hi = __byte_perm(a, b, 0x7632);
  float ra = __uint_as_float(a) - __uint_as_float(a & 0xffff0000u);
  float rb = __uint_as_float(b) - __uint_as_float(b & 0xffff0000u);
  const uint32_t ma = __float_as_uint(ra), mb = __float_as_uint(rb);
  mid = __byte_perm(ma, mb, 0x7632);
  ra -= __uint_as_float(ma & 0xffff0000u);
  rb -= __uint_as_float(mb & 0xffff0000u);
  lo = __byte_perm(__float_as_uint(ra), __float_as_uint(rb), 0x7632);
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
