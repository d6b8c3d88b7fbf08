// k_linear_few.cu -- the linear layer's products with few rows of x or dz (up
// to kFewRows) and 16-bit types.  Bound by reading the weights once: 2 bytes
// against at most 2 x 15 operations each.  So the weights go from memory
// straight into the fragments of warp-level MMAs (m16n8k16), 16 bytes per lane
// and load: a register is loaded again as soon as its MMA has read it, so that
// 16 loads per lane are in flight throughout, across the ends of groups too;
// which of K's elements a lane holds in which fragment is free as
// long as both operands agree, so no shuffle is needed either.  The few rows
// are in shared memory.
//
//   along    B lies along K (y = x w^T).  A warp takes 16 rows of w at a time as
//            the MMA's 16-row operand, the rows of x as its 8-column operand;
//            the 8 warps of a CTA share K in turns of 32 elements.
//   across   B lies along its rows (dx = dz w): a warp takes 64 columns, the
//            pairs of K that a fragment wants are put together from two rows of
//            w with byte permutations; 8 warps share K in turns of 16.
//
// Each group of columns is then summed over the warps in shared memory.  With
// fewer groups than CTAs fit the GPU, K is cut further over the CTAs of a
// cluster, which add their sums through distributed shared memory.  All sums have
// a fixed order.  (The MMA's places for rows that do not exist read the last row
// again; what they give is not looked at.)
//
// Measured: 1 row of 4096 to 4096 columns 6.5 us with the weights in L2, 11.5 from
// memory (2.9 TB/s: start and end are half of it); 1 x 4352 -> 7424 about 20.
#include <atomic>

#include "linear.cuh"
#include "linear_ptx.cuh"

namespace pic {
namespace lin {
namespace {

constexpr int kSms = 152;
// The few rows in shared memory.  More would leave an SM a single CTA and take
// longer to read than the weights: 4 rows of 16384 to 4096 columns 51 us (tiles of
// 128 rows on tcgen05: 35), 15 rows of 4096, which this just allows, 19 (25).
constexpr int kAlongRowBytes = 124 * 1024;
// Across, a row is read four bytes at a time: 8 rows of dz, 16384 to 4096 columns 43
// us with 64 KB (tiles: 36), 15 rows 81; 4096 to 4096 with 31 KB 15 us (25).
constexpr int kAcrossRowBytes = 48 * 1024;

struct FewParams {
  Product p;
  int groups;   // of columns
  int cluster;  // CTAs that share K
  int k_part;   // K of one of them, a multiple of 32
  int stride;   // bytes from row to row in shared memory
  int a_vec, pre_vec;  // A's (and a_pre's) rows start on 16-byte boundaries
};

// ---- m16n8k16, fp32 accumulators ----------------------------------------------
template <typename T>
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1);
template <>
__device__ __forceinline__ void mma<__half>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                            uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma<__nv_bfloat16>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                   uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Eight elements of a row, of which `n` exist; the weights pass by once.
template <typename T, int ALIGN>
__device__ __forceinline__ uint4 load8(const T* p, int n) {
  if (n <= 0) return make_uint4(0, 0, 0, 0);
  if (ALIGN == 16 && n >= 8) {
    uint4 q;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w)
                 : "l"(p));
    return q;
  }
  if constexpr (ALIGN == 4) {  // words that have an element of the row
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = load_if(reinterpret_cast<const uint32_t*>(p) + i, 2 * i < n);
    keep_bytes<T>(w, 2 * n);
    return make_uint4(w[0], w[1], w[2], w[3]);
  } else {
    uint32_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = load_if(reinterpret_cast<const uint16_t*>(p) + i, i < n);
    return make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
  }
}

// Eight elements of a row of A, or of dz = dy act'(z) rounded to its type.
template <typename T>
__device__ __forceinline__ uint4 load_a(const FewParams& q, int r, long long k, int n) {
  const Product& p = q.p;
  const T* a = static_cast<const T*>(p.a) + r * p.a_i + k;
  const uint4 w = q.a_vec ? load8<T, 16>(a, n) : load8<T, 2>(a, n);
  if (!p.a_pre) return w;
  const T* z = static_cast<const T*>(p.a_pre) + r * p.a_pre_i + k;
  const uint4 v = q.pre_vec ? load8<T, 16>(z, n) : load8<T, 2>(z, n);
  uint4 out;
  const T *d = reinterpret_cast<const T*>(&w), *e = reinterpret_cast<const T*>(&v);
  T* o = reinterpret_cast<T*>(&out);
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = from_f32<T>(act_grad<false>(to_f32(d[i]), to_f32(e[i]), p.a_act));
  return out;
}

// This CTA's part of K of A's rows into shared memory, zero past K's end.
template <typename T>
__device__ __forceinline__ void load_rows(uint8_t* s, const FewParams& q, int k0) {
  const Product& p = q.p;
  const int vecs = q.k_part / 8;
  for (int e = threadIdx.x; e < p.I * vecs; e += blockDim.x) {
    const int r = e / vecs, v = e % vecs;
    const long long left = p.K - k0 - v * 8;
    uint4 w = make_uint4(0, 0, 0, 0);
    if (left > 0) w = load_a<T>(q, r, k0 + v * 8, static_cast<int>(left < 8 ? left : 8));
    *reinterpret_cast<uint4*>(s + r * q.stride + v * 16) = w;
  }
}

template <typename T>
__device__ __forceinline__ void finish(const Product& p, int i, long long j, float v) {
  if (p.bias) v += to_f32(static_cast<const T*>(p.bias)[j]);
  if (p.pre) static_cast<T*>(p.pre)[i * p.ldpre + j] = from_f32<T>(v);
  v = act_value<false>(v, p.act);
  if (p.residual) v += to_f32(static_cast<const T*>(p.residual)[i * p.ldr + j]);
  static_cast<T*>(p.y)[i * p.ldy + j] = from_f32<T>(v);
}

// Sums of one group over the cluster's CTAs (sum[] of each), shared out, and
// out through the epilogue.  COLS columns, element e of sum: see `at`.
template <typename T, int COLS>
__device__ __forceinline__ void finish_group(const FewParams& q, float* sum, int rows, int stride_row, long long j0,
                                             uint32_t rank) {
  __syncwarp();
  tc::cluster_sync();
  for (int e = threadIdx.x + rank * blockDim.x; e < rows * COLS; e += blockDim.x * q.cluster) {
    const int i = e / COLS, c = e % COLS;
    float v = 0.0f;
    const uint32_t mine = tc::smem_addr(sum + i * stride_row + c);
    for (int r = 0; r < q.cluster; ++r) {
      float f;
      asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(f) : "r"(tc::map_rank(mine, r)) : "memory");
      v += f;
    }
    if (j0 + c < q.p.J) finish<T>(q.p, i, j0 + c, v);
  }
  __syncwarp();
  tc::cluster_sync();  // nobody leaves while its sums are read
}

constexpr int kAlongWarps = 8;
constexpr int kAlongSteps = 8;    // turns of 32 elements that a warp loads at a time
constexpr int kAlongStride = 20;  // floats per row of x in a warp's sums: no bank conflicts

template <typename T, int NT, int ALIGN>
__global__ void __launch_bounds__(32 * kAlongWarps, 2) along_kernel(const FewParams q) {
  extern __shared__ __align__(16) uint8_t smem[];
  const Product& p = q.p;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t rank = q.cluster > 1 ? tc::cluster_rank() : 0;
  const int k0 = rank * q.k_part, k1 = static_cast<int>(min(p.K, static_cast<long long>(k0) + q.k_part));
  constexpr int kSums = NT * 8 * kAlongStride;  // floats of one warp
  uint8_t* xs = smem;
  float* sums = reinterpret_cast<float*>(smem + p.I * q.stride);
  const T* w = static_cast<const T*>(p.b);

  uint4 a[kAlongSteps][2];
  auto load = [&](int s, int group, int k) {
    const int kk = k + s * 32 * kAlongWarps + t * 8;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const long long r = group * 16LL + g + 8 * h;
      a[s][h] = load8<T, ALIGN>(w + r * p.b_j + kk, r < p.J ? k1 - kk : 0);
    }
  };
  const int kw = k0 + warp * 32, batch = 32 * kAlongWarps * kAlongSteps, step = gridDim.x / q.cluster;
  int group = blockIdx.x / q.cluster;
#pragma unroll
  for (int s = 0; s < kAlongSteps; ++s) load(s, group, kw);
  load_rows<T>(xs, q, k0);
  __syncthreads();
  const uint8_t* rows[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) rows[n] = xs + min(n * 8 + g, static_cast<int>(p.I) - 1) * q.stride + t * 16;
  for (; group < q.groups; group += step) {
    float c[NT][4] = {};
    for (int k = kw; k < k1 || k == kw; k += batch) {
      const bool last = k + batch >= k1;
      const int next_k = last ? kw : k + batch, next_group = last ? group + step : group;
#pragma unroll
      for (int s = 0; s < kAlongSteps; ++s) {
        const int kk = k + s * 32 * kAlongWarps;
        if (kk < k1) {
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            const uint4 b = *reinterpret_cast<const uint4*>(rows[n] + (kk - k0) * 2);
            mma<T>(c[n], a[s][0].x, a[s][1].x, a[s][0].y, a[s][1].y, b.x, b.y);
            mma<T>(c[n], a[s][0].z, a[s][1].z, a[s][0].w, a[s][1].w, b.z, b.w);
          }
        }
        if (next_group < q.groups) load(s, next_group, next_k);
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float* s = sums + warp * kSums + (n * 8 + 2 * t) * kAlongStride + g;
      s[0] = c[n][0];
      s[kAlongStride] = c[n][1];
      s[8] = c[n][2];
      s[kAlongStride + 8] = c[n][3];
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.I * 16; e += blockDim.x) {
      const int i = e >> 4, col = e & 15;
      float v = 0.0f;
#pragma unroll
      for (int x = 0; x < kAlongWarps; ++x) v += sums[x * kSums + i * kAlongStride + col];
      if (q.cluster > 1)
        sums[i * kAlongStride + col] = v;  // only this thread reads or writes this place of warp 0's
      else if (group * 16LL + col < p.J)
        finish<T>(p, i, group * 16LL + col, v);
    }
    if (q.cluster > 1)
      finish_group<T, 16>(q, sums, static_cast<int>(p.I), kAlongStride, group * 16LL, rank);
    else
      __syncthreads();
  }
}

constexpr int kAcrossWarps = 8;
constexpr int kAcrossSteps = 4;    // turns of 16 elements that a warp loads at a time
constexpr int kAcrossStride = 68;  // floats per row in a warp's sums

// the low (high) halves of two words as one: a in the low half
__device__ __forceinline__ uint32_t low2(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x5410); }
__device__ __forceinline__ uint32_t high2(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x7632); }

template <typename T, int ALIGN>
__global__ void __launch_bounds__(32 * kAcrossWarps, 2) across_kernel(const FewParams q) {
  extern __shared__ __align__(16) uint8_t smem[];
  const Product& p = q.p;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t rank = q.cluster > 1 ? tc::cluster_rank() : 0;
  const int k0 = rank * q.k_part, k1 = static_cast<int>(min(p.K, static_cast<long long>(k0) + q.k_part));
  constexpr int kSums = 16 * kAcrossStride;
  uint8_t* xs = smem;
  float* sums = reinterpret_cast<float*>(smem + p.I * q.stride);
  const T* w = static_cast<const T*>(p.b);

  uint4 b[kAcrossSteps][4];
  auto load = [&](int s, int group, int k) {
    const long long j = group * 64LL + 8 * g;
    const int n = static_cast<int>(min(8LL, p.J - j));
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      // rows of B (elements of K) 2t, 2t + 1, 2t + 8, 2t + 9 of the turn
      const int kk = k + s * 16 * kAcrossWarps + 2 * t + (h & 1) + 8 * (h >> 1);
      b[s][h] = load8<T, ALIGN>(w + kk * p.b_k + j, kk < k1 ? n : 0);
    }
  };
  const int kw = k0 + warp * 16, batch = 16 * kAcrossWarps * kAcrossSteps, step = gridDim.x / q.cluster;
  int group = blockIdx.x / q.cluster;
#pragma unroll
  for (int s = 0; s < kAcrossSteps; ++s) load(s, group, kw);
  load_rows<T>(xs, q, k0);
  __syncthreads();
  const int rows = static_cast<int>(p.I);
  const uint8_t* x0 = xs + min(g, rows - 1) * q.stride + 4 * t;
  const uint8_t* x1 = xs + min(g + 8, rows - 1) * q.stride + 4 * t;
  for (; group < q.groups; group += step) {
    float c[8][4] = {};
    for (int k = kw; k < k1 || k == kw; k += batch) {
      const bool last = k + batch >= k1;
      const int next_k = last ? kw : k + batch, next_group = last ? group + step : group;
#pragma unroll
      for (int s = 0; s < kAcrossSteps; ++s) {
        const int kk = k + s * 16 * kAcrossWarps;
        if (kk < k1) {
          const int at = (kk - k0) * 2;
          const uint32_t a0 = *reinterpret_cast<const uint32_t*>(x0 + at);
          const uint32_t a1 = *reinterpret_cast<const uint32_t*>(x1 + at);
          const uint32_t a2 = *reinterpret_cast<const uint32_t*>(x0 + at + 16);
          const uint32_t a3 = *reinterpret_cast<const uint32_t*>(x1 + at + 16);
          const uint32_t r0[4] = {b[s][0].x, b[s][0].y, b[s][0].z, b[s][0].w};
          const uint32_t r1[4] = {b[s][1].x, b[s][1].y, b[s][1].z, b[s][1].w};
          const uint32_t r2[4] = {b[s][2].x, b[s][2].y, b[s][2].z, b[s][2].w};
          const uint32_t r3[4] = {b[s][3].x, b[s][3].y, b[s][3].z, b[s][3].w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            mma<T>(c[2 * j], a0, a1, a2, a3, low2(r0[j], r1[j]), low2(r2[j], r3[j]));
            mma<T>(c[2 * j + 1], a0, a1, a2, a3, high2(r0[j], r1[j]), high2(r2[j], r3[j]));
          }
        }
        if (next_group < q.groups) load(s, next_group, next_k);
      }
    }
    // MMA j's column n is column 8 n + j of the group
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float* s = sums + warp * kSums + g * kAcrossStride + 16 * t + j;
      s[0] = c[j][0];
      s[8] = c[j][1];
      s[8 * kAcrossStride] = c[j][2];
      s[8 * kAcrossStride + 8] = c[j][3];
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.I * 64; e += blockDim.x) {
      const int i = e >> 6, col = e & 63;
      float v = 0.0f;
#pragma unroll
      for (int x = 0; x < kAcrossWarps; ++x) v += sums[x * kSums + i * kAcrossStride + col];
      if (q.cluster > 1)
        sums[i * kAcrossStride + col] = v;  // only this thread reads or writes this place of warp 0's
      else if (group * 64LL + col < p.J)
        finish<T>(p, i, group * 64LL + col, v);
    }
    if (q.cluster > 1)
      finish_group<T, 64>(q, sums, static_cast<int>(p.I), kAcrossStride, group * 64LL, rank);
    else
      __syncthreads();
  }
}

struct Plan {
  bool ok, along;
  int groups, cluster, k_part, stride, grid, smem, tiles;  // tiles: of 8 rows (along)
};

Plan plan(const Product& p) {
  Plan r{};
  if (p.I > kFewRows || p.a_k != 1 || p.K > 0x7fffff00LL) return r;
  r.along = p.b_k == 1;
  const int cols = r.along ? 16 : 64, turn = r.along ? 32 : 16;
  const long long groups = (p.J + cols - 1) / cols;
  if (groups > 0x7fffffffLL) return r;
  r.groups = static_cast<int>(groups);
  // K over a cluster while that gives CTAs work that have none (two on an SM) and
  // every warp a turn; a row's places 64 (16) bytes past a multiple of 128 apart:
  // no bank conflicts
  const int warps = r.along ? kAlongWarps : kAcrossWarps;
  const auto row_bytes = [&](int cluster) {
    r.k_part = static_cast<int>((p.K + cluster - 1) / cluster + 31) / 32 * 32;
    return (r.k_part * 2LL + 127) / 128 * 128 + (r.along ? 64 : 16);
  };
  r.cluster = 1;
  while (r.cluster < 8 && groups * r.cluster * 2 <= 2 * kSms && p.K >= 2LL * r.cluster * turn * warps) r.cluster *= 2;
  const long long stride = row_bytes(r.cluster);
  if (p.I * stride > (r.along ? kAlongRowBytes : kAcrossRowBytes)) return r;
  r.stride = static_cast<int>(stride);
  r.tiles = r.along ? static_cast<int>((p.I + 7) / 8) : 1;
  const int sums = r.along ? kAlongWarps * r.tiles * 8 * kAlongStride : kAcrossWarps * 16 * kAcrossStride;
  r.smem = static_cast<int>(p.I) * r.stride + sums * 4;
  if (r.smem > 227 * 1024) return r;
  // whole clusters, two CTAs on an SM where their shared memory allows it
  const int most = kSms * (r.smem <= 110 * 1024 ? 2 : 1) / r.cluster * r.cluster;
  const long long want = groups * r.cluster;
  r.grid = static_cast<int>(want < most ? want : most);
  r.ok = true;
  return r;
}

template <typename T, int ALIGN>
const void* kernel_of(const Plan& r) {
  if (!r.along) return reinterpret_cast<const void*>(across_kernel<T, ALIGN>);
  return r.tiles == 1 ? reinterpret_cast<const void*>(along_kernel<T, 1, ALIGN>)
                      : reinterpret_cast<const void*>(along_kernel<T, 2, ALIGN>);
}

template <typename T>
const void* kernel_at(const Plan& r, int align) {
  return align == 2 ? kernel_of<T, 16>(r) : align == 1 ? kernel_of<T, 4>(r) : kernel_of<T, 2>(r);
}

// Allows the kernel all of an SM's shared memory, once per device.
int set_up(const void* fn, int slot) {
  static std::atomic<uint64_t> done[18];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return PIC_ERR_CUDA;
  const uint64_t bit = 1ull << (dev & 63);
  if (done[slot].load(std::memory_order_acquire) & bit) return PIC_OK;
  if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024) != cudaSuccess)
    return PIC_ERR_CUDA;
  done[slot].fetch_or(bit, std::memory_order_release);
  return PIC_OK;
}

}  // namespace

bool few_takes(const Product& p) { return plan(p).ok; }

int few_product(const Product& p, int dtype, cudaStream_t s) {
  const Plan r = plan(p);
  FewParams q{p, r.groups, r.cluster, r.k_part, r.stride, 0, 0};
  q.a_vec = reinterpret_cast<uintptr_t>(p.a) % 16 == 0 && (p.I == 1 || p.a_i % 8 == 0);
  q.pre_vec = reinterpret_cast<uintptr_t>(p.a_pre) % 16 == 0 && (p.I == 1 || p.a_pre_i % 8 == 0);
  const uintptr_t at = reinterpret_cast<uintptr_t>(p.b) | static_cast<uintptr_t>((r.along ? p.b_j : p.b_k) * 2);
  const int align = at % 16 == 0 ? 2 : at % 4 == 0 ? 1 : 0;  // 16, 4 or 2 bytes
  const bool bf16 = dtype == PIC_DTYPE_BF16;
  const void* fn = bf16 ? kernel_at<__nv_bfloat16>(r, align) : kernel_at<__half>(r, align);
  const int slot = ((bf16 ? 3 : 0) + align) * 3 + (r.along ? r.tiles : 0);
  if (set_up(fn, slot) != PIC_OK) return PIC_ERR_CUDA;
  void* args[] = {&q};
  return launch_kernel(fn, r.grid, 32 * (r.along ? kAlongWarps : kAcrossWarps), r.smem, r.cluster, args, s);
}

}  // namespace lin
}  // namespace pic
