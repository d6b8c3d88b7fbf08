// k_linear_few32.cu -- the linear layer's products with few rows of x or dz (up to
// kFewRows32) in fp32, on the FP32 cores.  Bound by reading the weights once: 4 bytes
// against at most 2 x 8 operations each, of which the cores do 2 x 22 in the time of
// 4 bytes.  The organisation is that of k_linear_few.cu, with FMAs on lanes:
//
//   along    (y = x w^T) a warp takes four rows of w, a lane 4 elements of each at a
//            time, so that a value of x read from shared memory serves four rows;
//            the lanes' sums are halved and exchanged until each has its share.
//   across   (dx = dz w) a lane takes 4 columns; the few values of dz that belong to
//            a row of w are read from shared memory, four at a time.
//
// Eight warps of a CTA, and the CTAs of a cluster, share K in turns; they meet to add
// their sums after several groups.  Measured, with weights that come from memory: 1
// row of 4352 to 7424 columns 41 us, 3.2 TB/s, 8 rows 61; of dz, 7424 to 4352, 31 and
// 45.
#include <atomic>

#include "linear.cuh"
#include "linear_ptx.cuh"

namespace pic {
namespace lin {
namespace {

constexpr int kSms = 152;
constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kGroup = 4;         // rows of w of a warp (along)
constexpr int kAlongTurn = 128;   // elements of K of a warp's turn
constexpr int kAlongSteps = 4;    // turns that a warp loads at a time
constexpr int kAlongGroups = 6;   // groups between two meetings of a CTA's, and a cluster's, warps
constexpr int kAcrossCols = 128;  // columns of a warp (across)
constexpr int kAcrossRows = 8;    // rows of w that a warp loads at a time
constexpr int kMaxBytes = 100 * 1024;  // the few rows in shared memory, two CTAs on an SM

struct FewParams {
  Product p;
  int groups, cluster, k_part;  // k_part a multiple of 128
};

// Four elements from p on, of which n exist; not VEC: 32 apart, from p + lane on.
template <bool VEC>
__device__ __forceinline__ float4 load4(const float* p, int n, int lane) {
  uint32_t w[4];
  if constexpr (VEC) {
    n = (n - 4 * lane) * 4;
    const uint4 f = load_if16(p + 4 * lane, n > 0);
    w[0] = f.x, w[1] = f.y, w[2] = f.z, w[3] = f.w;
    keep_bytes<float>(w, n);
  } else {
    p += lane, n -= lane;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = load_if(reinterpret_cast<const uint32_t*>(p) + 32 * i, n > 32 * i);
  }
  return make_float4(__uint_as_float(w[0]), __uint_as_float(w[1]), __uint_as_float(w[2]), __uint_as_float(w[3]));
}

// This CTA's part of K of the rows of A (or of dz = dy act'(z)) to put(i, k, values),
// four elements at a time, zero past K's end; kRowLoads of a thread's loads are under
// way together (one by one, 5 rows of 4352 took longer than 129 MB of weights).
constexpr int kRowLoads = 4;
template <typename Put>
__device__ __forceinline__ void load_rows(const FewParams& q, int k0, Put put) {
  const Product& p = q.p;
  const int per_row = q.k_part / 4, n = static_cast<int>(p.I) * per_row;
  const auto load = [&](const void* m, long long ld, int i, int k) {
    const uint32_t* a = static_cast<const uint32_t*>(m) + i * ld + k;
    const long long left = i < p.I ? p.K - k : 0;
    return make_float4(__uint_as_float(load_if(a, left > 0)), __uint_as_float(load_if(a + 1, left > 1)),
                       __uint_as_float(load_if(a + 2, left > 2)), __uint_as_float(load_if(a + 3, left > 3)));
  };
  for (int e0 = threadIdx.x; e0 < n; e0 += kThreads * kRowLoads) {
    float4 d[kRowLoads], z[kRowLoads];
#pragma unroll
    for (int u = 0; u < kRowLoads; ++u) {
      const int e = e0 + u * kThreads;
      d[u] = load(p.a, p.a_i, e / per_row, k0 + e % per_row * 4);
    }
    if (p.a_pre) {
#pragma unroll
      for (int u = 0; u < kRowLoads; ++u) {
        const int e = e0 + u * kThreads;
        z[u] = load(p.a_pre, p.a_pre_i, e / per_row, k0 + e % per_row * 4);
      }
#pragma unroll
      for (int u = 0; u < kRowLoads; ++u) {
        const float2 lo = act_grad2<true>(make_float2(d[u].x, d[u].y), make_float2(z[u].x, z[u].y), p.a_act);
        const float2 hi = act_grad2<true>(make_float2(d[u].z, d[u].w), make_float2(z[u].z, z[u].w), p.a_act);
        d[u] = make_float4(lo.x, lo.y, hi.x, hi.y);
      }
    }
#pragma unroll
    for (int u = 0; u < kRowLoads; ++u) {
      const int e = e0 + u * kThreads;
      if (e < n) put(e / per_row, e % per_row * 4, d[u]);
    }
  }
}

__device__ __forceinline__ void finish(const Product& p, int i, long long j, float v) {
  if (p.bias) v += static_cast<const float*>(p.bias)[j];
  if (p.pre) static_cast<float*>(p.pre)[i * p.ldpre + j] = v;
  v = act_value<true>(v, p.act);
  if (p.residual) v += static_cast<const float*>(p.residual)[i * p.ldr + j];
  static_cast<float*>(p.y)[i * p.ldy + j] = v;
}

// sums[group][warp][rows][cols] of every CTA of the cluster, added warps first, then
// CTAs, both in order, and out through the epilogue: `count` groups, the first at
// column j0, apart by `apart` columns.
__device__ __forceinline__ void finish_groups(const FewParams& q, float* sums, int mt, int cols, int count, long long j0,
                                              long long apart, uint32_t rank) {
  const Product& p = q.p;
  __syncthreads();
  const int per = static_cast<int>(p.I) * cols, n = count * per, group = kWarps * mt * cols;
  const auto out = [&](int e, float v) {
    const int i = e % per;
    const long long j = j0 + e / per * apart + i % cols;
    if (j < p.J) finish(p, i / cols, j, v);
  };
  for (int e = threadIdx.x; e < n; e += kThreads) {
    float* s = sums + e / per * group + e % per;
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) v += s[w * mt * cols];
    if (q.cluster > 1)
      *s = v;  // only this thread reads or writes this place of warp 0's
    else
      out(e, v);
  }
  __syncwarp();
  if (q.cluster > 1) {
    tc::cluster_sync();
    for (int e = threadIdx.x + rank * kThreads; e < n; e += kThreads * q.cluster) {
      float v = 0.0f;
      for (int r = 0; r < q.cluster; ++r) {
        float f;
        const uint32_t at = tc::map_rank(tc::smem_addr(sums + e / per * group + e % per), r);
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(f) : "r"(at) : "memory");
        v += f;
      }
      out(e, v);
    }
    __syncwarp();
    tc::cluster_sync();  // nobody goes on while its sums are read
  } else {
    __syncthreads();
  }
}

template <int MT, bool VEC>
__global__ void __launch_bounds__(kThreads, 2) along_kernel(const FewParams q) {
  extern __shared__ __align__(16) float smem[];
  const Product& p = q.p;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rows = static_cast<int>(p.I);
  const uint32_t rank = q.cluster > 1 ? tc::cluster_rank() : 0;
  const int k0 = rank * q.k_part, k1 = static_cast<int>(min(p.K, static_cast<long long>(k0) + q.k_part));
  float* xs = smem;                                    // [rows][k_part]
  float* sums = smem + rows * q.k_part;                // [kAlongGroups][warps][MT][kGroup]
  const float* w = static_cast<const float*>(p.b);
  float4 a[kAlongSteps][kGroup];
  auto load = [&](int s, int group, int k) {
    const int kk = k + s * kAlongTurn * kWarps;
#pragma unroll
    for (int r = 0; r < kGroup; ++r) {
      const long long n = group * static_cast<long long>(kGroup) + r;
      a[s][r] = load4<VEC>(w + n * p.b_j + kk, n < p.J ? k1 - kk : 0, lane);
    }
  };
  const int kw = k0 + warp * kAlongTurn, batch = kAlongTurn * kWarps * kAlongSteps, step = gridDim.x / q.cluster;
  int group = blockIdx.x / q.cluster;
#pragma unroll
  for (int s = 0; s < kAlongSteps; ++s) load(s, group, kw);
  load_rows(q, k0, [&](int i, int k, const float4& v) { *reinterpret_cast<float4*>(xs + i * q.k_part + k) = v; });
  __syncthreads();
  int slot = 0;
  for (; group < q.groups; group += step) {
    float c[MT * kGroup] = {};
    for (int k = kw; k < k1 || k == kw; k += batch) {
      const bool last = k + batch >= k1;
      const int next_k = last ? kw : k + batch, next_group = last ? group + step : group;
#pragma unroll
      for (int s = 0; s < kAlongSteps; ++s) {
        const int kk = k + s * kAlongTurn * kWarps;
        if (kk < k1) {
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const float* x = xs + min(m, rows - 1) * q.k_part + kk - k0;
            float4 f;
            if constexpr (VEC)
              f = *reinterpret_cast<const float4*>(x + 4 * lane);
            else
              f = make_float4(x[lane], x[lane + 32], x[lane + 64], x[lane + 96]);
#pragma unroll
            for (int r = 0; r < kGroup; ++r) {
              float& t = c[m * kGroup + r];
              t = fmaf(a[s][r].x, f.x, t);
              t = fmaf(a[s][r].y, f.y, t);
              t = fmaf(a[s][r].z, f.z, t);
              t = fmaf(a[s][r].w, f.w, t);
            }
          }
        }
        if (next_group < q.groups) load(s, next_group, next_k);
      }
    }
    // each exchange halves the sums that a lane answers for, while there is more
    // than one; then the lanes of a sum add theirs
    int mine = 0;  // which sum this lane ends up with
#pragma unroll
    for (int o = 16, n = MT * kGroup; o > 0; o >>= 1) {
      if (n > 1) {
        n /= 2;
        const bool upper = (lane & o) != 0;
#pragma unroll
        for (int i = 0; i < MT * kGroup / 2; ++i)
          if (i < n) {
            const float keep = upper ? c[i + n] : c[i], give = upper ? c[i] : c[i + n];
            c[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
          }
        if (upper) mine += n;
      } else {
        c[0] += __shfl_xor_sync(0xffffffffu, c[0], o);
      }
    }
    sums[(slot * kWarps + warp) * MT * kGroup + mine] = c[0];  // lanes with the same sum write the same value
    if (++slot == kAlongGroups || group + step >= q.groups) {
      const long long j0 = (group - (slot - 1LL) * step) * kGroup;
      finish_groups(q, sums, MT, kGroup, slot, j0, static_cast<long long>(step) * kGroup, rank);
      slot = 0;
    }
  }
}

template <int MT, bool VEC>
__global__ void __launch_bounds__(kThreads, 2) across_kernel(const FewParams q) {
  extern __shared__ __align__(16) float smem[];
  const Product& p = q.p;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rows = static_cast<int>(p.I);
  const uint32_t rank = q.cluster > 1 ? tc::cluster_rank() : 0;
  const int k0 = rank * q.k_part, k1 = static_cast<int>(min(p.K, static_cast<long long>(k0) + q.k_part));
  float* xs = smem;                       // [k_part][MT]
  float* sums = smem + q.k_part * MT;     // [warps][MT][kAcrossCols]
  const float* w = static_cast<const float*>(p.b);
  float4 b[kAcrossRows];
  auto load = [&](int s, int group, int k) {
    const long long j = group * static_cast<long long>(kAcrossCols);
    const int kk = k + s;
    b[s] = load4<VEC>(w + kk * p.b_k + j, kk < k1 ? static_cast<int>(min(static_cast<long long>(kAcrossCols), p.J - j)) : 0, lane);
  };
  const int kw = k0 + warp * kAcrossRows, batch = kAcrossRows * kWarps, step = gridDim.x / q.cluster;
  int group = blockIdx.x / q.cluster;
#pragma unroll
  for (int s = 0; s < kAcrossRows; ++s) load(s, group, kw);
  load_rows(q, k0, [&](int i, int k, const float4& v) {
    const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int c = 0; c < 4; ++c) xs[(k + c) * MT + i] = f[c];
  });
  for (int e = threadIdx.x; e < q.k_part * (MT - rows); e += kThreads)  // rows that do not exist
    xs[e / (MT - rows) * MT + rows + e % (MT - rows)] = 0.0f;
  __syncthreads();
  for (; group < q.groups; group += step) {
    float4 c[MT] = {};
    for (int k = kw; k < k1 || k == kw; k += batch) {
      const bool last = k + batch >= k1;
      const int next_k = last ? kw : k + batch, next_group = last ? group + step : group;
#pragma unroll
      for (int s = 0; s < kAcrossRows; ++s) {
        if (k + s < k1) {
          const float* x = xs + (k + s - k0) * MT;
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            c[m].x = fmaf(x[m], b[s].x, c[m].x);
            c[m].y = fmaf(x[m], b[s].y, c[m].y);
            c[m].z = fmaf(x[m], b[s].z, c[m].z);
            c[m].w = fmaf(x[m], b[s].w, c[m].w);
          }
        }
        if (next_group < q.groups) load(s, next_group, next_k);
      }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      float* s = sums + (warp * MT + m) * kAcrossCols;
      if constexpr (VEC) {
        *reinterpret_cast<float4*>(s + 4 * lane) = c[m];
      } else {
        s[lane] = c[m].x, s[lane + 32] = c[m].y, s[lane + 64] = c[m].z, s[lane + 96] = c[m].w;
      }
    }
    finish_groups(q, sums, MT, kAcrossCols, 1, group * static_cast<long long>(kAcrossCols), 0, rank);
  }
}

struct Plan {
  bool ok, along;
  int groups, cluster, k_part, mt, smem, grid;
};

Plan plan(const Product& p) {
  Plan r{};
  if (p.I > kFewRows32 || p.a_k != 1 || p.K > 0x7fffff00LL) return r;
  r.along = p.b_k == 1;
  r.mt = p.I <= 1 ? 1 : p.I <= 2 ? 2 : p.I <= 4 ? 4 : 8;
  const long long groups = r.along ? (p.J + kGroup - 1) / kGroup : (p.J + kAcrossCols - 1) / kAcrossCols;
  if (groups > 0x7fffffffLL) return r;
  r.groups = static_cast<int>(groups);
  const int turn = r.along ? kAlongTurn : kAcrossRows;
  const auto bytes = [&](int cluster) {
    r.k_part = static_cast<int>((p.K + cluster - 1) / cluster + 127) / 128 * 128;
    return static_cast<long long>(r.along ? p.I : r.mt) * r.k_part * 4;
  };
  // K over a cluster while that gives CTAs work that have none and every warp a turn,
  // and until the rows fit
  r.cluster = 1;
  while (r.cluster < 8 && groups * r.cluster * 2 <= 2 * kSms && p.K >= 2LL * r.cluster * turn * kWarps) r.cluster *= 2;
  while (r.cluster < 8 && bytes(r.cluster) > kMaxBytes) r.cluster *= 2;
  const long long need = bytes(r.cluster);
  if (need > kMaxBytes) return r;
  r.smem = static_cast<int>(need) + kWarps * r.mt * (r.along ? kGroup * kAlongGroups : kAcrossCols) * 4;
  if (r.smem > 113 * 1024) return r;
  const int most = 2 * kSms / r.cluster * r.cluster;
  const long long want = groups * r.cluster;
  r.grid = static_cast<int>(want < most ? want : most);
  r.ok = true;
  return r;
}

template <bool VEC>
const void* kernel_of(const Plan& r) {
  const void* along[] = {reinterpret_cast<const void*>(along_kernel<1, VEC>), reinterpret_cast<const void*>(along_kernel<2, VEC>),
                         reinterpret_cast<const void*>(along_kernel<4, VEC>), reinterpret_cast<const void*>(along_kernel<8, VEC>)};
  const void* across[] = {reinterpret_cast<const void*>(across_kernel<1, VEC>), reinterpret_cast<const void*>(across_kernel<2, VEC>),
                          reinterpret_cast<const void*>(across_kernel<4, VEC>), reinterpret_cast<const void*>(across_kernel<8, VEC>)};
  const int i = r.mt == 1 ? 0 : r.mt == 2 ? 1 : r.mt == 4 ? 2 : 3;
  return r.along ? along[i] : across[i];
}

}  // namespace

bool few32_takes(const Product& p) { return plan(p).ok; }

int few32_product(const Product& p, cudaStream_t s) {
  const Plan r = plan(p);
  FewParams q{p, r.groups, r.cluster, r.k_part};
  const long long ld = r.along ? p.b_j : p.b_k;
  const bool vec = reinterpret_cast<uintptr_t>(p.b) % 16 == 0 && ld % 4 == 0;
  const void* fn = vec ? kernel_of<true>(r) : kernel_of<false>(r);
  // more than 48 KB is allowed once per device and kernel
  static std::atomic<uint64_t> done[16];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return PIC_ERR_CUDA;
  const int slot = (vec ? 8 : 0) + (r.along ? 4 : 0) + (r.mt == 1 ? 0 : r.mt == 2 ? 1 : r.mt == 4 ? 2 : 3);
  const uint64_t bit = 1ull << (dev & 63);
  if (!(done[slot].load(std::memory_order_acquire) & bit)) {
    if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, 113 * 1024) != cudaSuccess) return PIC_ERR_CUDA;
    done[slot].fetch_or(bit, std::memory_order_release);
  }
  void* args[] = {&q};
  return launch_kernel(fn, r.grid, kThreads, r.smem, r.cluster, args, s);
}

}  // namespace lin
}  // namespace pic
