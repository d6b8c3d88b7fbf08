// k_group_few.cu -- grouped layers with few rows in a group, and their gradients: all that
// counts is to read each group's weights, or to write its gradient of them, once.
//
// eight rows at a time, on the FP32 cores (sums and products are fp32 for every type):
//   forward   a warp has four rows of the weights, its lanes 16 bytes of each at a time
//             along K; the eight rows of x are in shared memory as fp32, 1024 of K at a
//             time.  At the end the 32 sums of each lane are added up so that lane l has the
//             l-th.
//   dx        a lane has 16 bytes' worth of columns, the warps take turns at the rows of the
//             weights; dz is in shared memory.  The warps' sums are added at the end.
//   dw, db    a lane has 16 bytes' worth of columns of x, a warp four rows of dw.  A group
//             without rows gets zeros.
// dz = dy act'(z) is made on the way and not rounded: a gradient is two launches.
//
// Weights (and in the gradients x and dw) whose rows are not on 16-byte boundaries: in the
// forward the two aligned pieces that have the 16 bytes, shifted; in the gradients lanes
// have columns 32 apart instead.  Nothing is laid out first, which for weights would be
// three times their traffic.
//
// Measured: 64 groups with 96 rows (half of the groups have none) fp32 2048 -> 2048 110 us, 4.6
// TB/s of weights (tiles of 64 x 64 703); bf16 2047 -> 4096 203 us (laid out first 458).
#include "group.cuh"

namespace pic {
namespace grp {
namespace {

using lin::act_grad;
using lin::act_value;
using lin::from_f32;
using lin::Piece16;
using lin::to_f32;

constexpr int kSms = 152;
constexpr int kThreads = 256, kWarps = 8;
constexpr int kRows = 8;       // of a group at a time
constexpr int kDeep = 1024;    // of K in shared memory
constexpr int kOuts = 4;       // rows of the weights of a warp at a time

struct FewParams {
  const void* x;    // forward, dw: [rows][K]
  long long ldx;
  const void* dy;   // gradients: [rows][N], with pre and act
  long long lddy;
  const void* pre;
  long long ldpre;
  const void* w;
  long long ldw, w_group;
  const void* bias;
  long long bias_group;
  void* y;          // forward: y; gradients: dx, dw
  long long ldy, y_group;
  void* z;          // forward: pre; dw: db
  long long ldz;
  long long rows, K, N;
  int groups, act;
  const long long* offsets;
  int* status;
  int out16;        // rows of dx (dw) are on 16-byte boundaries
};

template <typename T>
__device__ __forceinline__ float dz_at(const FewParams& q, long long row, long long n) {
  const float d = to_f32(static_cast<const T*>(q.dy)[row * q.lddy + n]);
  if (q.act == PIC_ACT_NONE) return d;
  return act_grad<sizeof(T) == 4>(d, to_f32(static_cast<const T*>(q.pre)[row * q.ldpre + n]), q.act);
}

// f with the least of 1, 2, 4 and 8 that is `rows` or more, as a type.
template <typename F>
__device__ __forceinline__ void for_rows(int rows, F f) {
  if (rows > 4)
    f(std::integral_constant<int, 8>{});
  else if (rows > 2)
    f(std::integral_constant<int, 4>{});
  else if (rows > 1)
    f(std::integral_constant<int, 2>{});
  else
    f(std::integral_constant<int, 1>{});
}

// R rows of x (in shared memory) and four, `outs` of them there, of the weights, over `deep` of K.
template <typename T, bool ON16, int R>
__device__ __forceinline__ void forward_chunk(float (&acc)[kOuts * kRows], const float (&xs)[kRows][kDeep], const T* w,
                                              long long ldw, int outs, int deep, int lane) {
  constexpr int V = 16 / sizeof(T);
#pragma unroll 2
  for (int k = lane * V; k < deep; k += 32 * V) {
    uint32_t v[kOuts][4];
    Piece16<ON16> p[kOuts];
    const int bytes = (deep - k) * static_cast<int>(sizeof(T));
#pragma unroll
    for (int o = 0; o < kOuts; ++o) p[o].load(reinterpret_cast<const char*>(w + o * ldw + k), o < outs ? bytes : 0);
#pragma unroll
    for (int o = 0; o < kOuts; ++o) {
      p[o].template get<T>(static_cast<int>(reinterpret_cast<uintptr_t>(w + o * ldw + k) & 15), v[o]);
      if (bytes < 16 || o >= outs) lin::keep_bytes<T>(v[o], o < outs ? bytes : 0);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int h = 0; h < V; h += 4) {
        const float4 a = *reinterpret_cast<const float4*>(&xs[r][k + h]);
        const float x[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int o = 0; o < kOuts; ++o)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            acc[o * kRows + r] = fmaf(to_f32(reinterpret_cast<const T*>(v[o])[h + e]), x[e], acc[o * kRows + r]);
      }
    }
  }
}

template <typename T, bool ON16>
__global__ void __launch_bounds__(kThreads, 2) forward_kernel(const FewParams q) {
  __shared__ GroupTable table;
  __shared__ __align__(16) float xs[kRows][kDeep];
  make_table(table, q.offsets, q.groups, q.rows, kRows, 0, q.status);
  wait_for_earlier();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long blocks = (q.N + kOuts * kWarps - 1) / (kOuts * kWarps), work = table.tiles[q.groups] * blocks;
  for (long long item = blockIdx.x; item < work; item += gridDim.x) {
    const int tile = static_cast<int>(item / blocks), g = table.find(tile, q.groups);
    const long long row0 = table.start[g] + static_cast<long long>(tile - table.tiles[g]) * kRows;
    const int rows = static_cast<int>(min(static_cast<long long>(kRows), table.start[g + 1] - row0));
    const long long n0 = (item % blocks * kWarps + warp) * kOuts;
    const T* w = static_cast<const T*>(q.w) + g * q.w_group;
    float acc[kOuts * kRows] = {};
    for (long long k0 = 0; k0 < q.K; k0 += kDeep) {
      const int deep = static_cast<int>(min(static_cast<long long>(kDeep), q.K - k0));
      __syncthreads();
      for (int e = threadIdx.x; e < kRows * kDeep; e += kThreads) {
        const int r = e / kDeep, k = e % kDeep;
        xs[r][k] = r < rows && k < deep ? to_f32(static_cast<const T*>(q.x)[(row0 + r) * q.ldx + k0 + k]) : 0.0f;
      }
      __syncthreads();
      for_rows(rows, [&](auto r) {
        forward_chunk<T, ON16, decltype(r)::value>(acc, xs, w + n0 * q.ldw + k0, q.ldw, static_cast<int>(min(q.N - n0, static_cast<long long>(kOuts))), deep, lane);
      });
    }
    // lane l adds up the l-th sum: halves of the sums go to the other half of the lanes
#pragma unroll
    for (int d = 16; d > 0; d /= 2) {
      const bool upper = (lane & d) != 0;
#pragma unroll
      for (int i = 0; i < d; ++i) {
        const float give = upper ? acc[i] : acc[i + d], keep = upper ? acc[i + d] : acc[i];
        acc[i] = keep + __shfl_xor_sync(0xffffffffu, give, d);
      }
    }
    const long long n = n0 + lane / kRows;
    const int r = lane % kRows;
    if (r < rows && n < q.N) {
      float z = acc[0];
      if (q.bias) z += to_f32(static_cast<const T*>(q.bias)[g * q.bias_group + n]);
      if (q.z) static_cast<T*>(q.z)[(row0 + r) * q.ldz + n] = from_f32<T>(z);
      static_cast<T*>(q.y)[(row0 + r) * q.ldy + n] = from_f32<T>(act_value<sizeof(T) == 4>(z, q.act));
    }
  }
}

// Column e of a lane's in a block of 32 V, and loads and stores of them.
template <typename T, bool ON16>
struct Columns {
  static constexpr int V = 16 / sizeof(T);
  static __device__ __forceinline__ int at(int lane, int e) { return ON16 ? lane * V + e : lane + 32 * e; }
  static __device__ __forceinline__ void load(float (&v)[V], const T* p, int lane, int cols, bool on) {
    if constexpr (ON16) {
      const uint4 w = lin::load_if16(p + lane * V, on && lane * V < cols);
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = to_f32(reinterpret_cast<const T*>(u)[e]);
    } else {
      T u[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        if constexpr (sizeof(T) == 4) {
          u[e] = __uint_as_float(lin::load_if(reinterpret_cast<const uint32_t*>(p + lane + 32 * e), on && lane + 32 * e < cols));
        } else {
          const uint16_t h = static_cast<uint16_t>(lin::load_if(reinterpret_cast<const uint16_t*>(p + lane + 32 * e), on && lane + 32 * e < cols));
          u[e] = *reinterpret_cast<const T*>(&h);
        }
      }
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = to_f32(u[e]);
    }
  }
  static __device__ __forceinline__ void store(const float (&v)[V], T* p, int lane, int cols, bool on16) {
    if (ON16 && on16 && lane * V + V <= cols) {
      uint32_t u[4];
#pragma unroll
      for (int e = 0; e < V; ++e) reinterpret_cast<T*>(u)[e] = from_f32<T>(v[e]);
      *reinterpret_cast<uint4*>(p + lane * V) = make_uint4(u[0], u[1], u[2], u[3]);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (at(lane, e) < cols) p[at(lane, e)] = from_f32<T>(v[e]);
    }
  }
};

template <typename T, bool ON16>
__global__ void __launch_bounds__(kThreads, 2) dx_kernel(const FewParams q) {
  using C = Columns<T, ON16>;
  constexpr int V = C::V, kCols = 32 * V;
  __shared__ GroupTable table;
  __shared__ __align__(16) float ds[kDeep * kRows];  // [n][row]; at the end four warps' sums
  static_assert(4 * kRows * kCols <= kDeep * kRows, "sums in the place of dz");
  make_table(table, q.offsets, q.groups, q.rows, kRows, 0, q.status);
  wait_for_earlier();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long blocks = (q.K + kCols - 1) / kCols, work = table.tiles[q.groups] * blocks;
  for (long long item = blockIdx.x; item < work; item += gridDim.x) {
    const int tile = static_cast<int>(item / blocks), g = table.find(tile, q.groups);
    const long long row0 = table.start[g] + static_cast<long long>(tile - table.tiles[g]) * kRows;
    const int rows = static_cast<int>(min(static_cast<long long>(kRows), table.start[g + 1] - row0));
    const long long j0 = item % blocks * kCols;
    const int cols = static_cast<int>(min(static_cast<long long>(kCols), q.K - j0));
    const T* w = static_cast<const T*>(q.w) + g * q.w_group + j0;
    float acc[kRows][V] = {};
    for (long long n0 = 0; n0 < q.N; n0 += kDeep) {
      const int deep = static_cast<int>(min(static_cast<long long>(kDeep), q.N - n0));
      __syncthreads();
      for (int e = threadIdx.x; e < kRows * kDeep; e += kThreads) {
        const int r = e / kDeep, n = e % kDeep;
        ds[n * kRows + r] = r < rows && n < deep ? dz_at<T>(q, row0 + r, n0 + n) : 0.0f;
      }
      __syncthreads();
#pragma unroll 4
      for (int n = warp; n < deep; n += kWarps) {  // (for fewer rows by themselves it is no sooner done)
        float v[V];
        C::load(v, w + (n0 + n) * q.ldw, lane, cols, true);
        const float4 a = *reinterpret_cast<const float4*>(&ds[n * kRows]), b = *reinterpret_cast<const float4*>(&ds[n * kRows + 4]);
        const float d[kRows] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
          for (int e = 0; e < V; ++e) acc[r][e] = fmaf(d[r], v[e], acc[r][e]);
      }
    }
    // the warps' sums, the upper half's to the lower's, three times
#pragma unroll
    for (int half = 4; half > 0; half /= 2) {
      __syncthreads();
      if (warp >= half && warp < 2 * half) {
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
          for (int e = 0; e < V; ++e) ds[(((warp - half) * kRows + r) * V + e) * 32 + lane] = acc[r][e];
      }
      __syncthreads();
      if (warp < half) {
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
          for (int e = 0; e < V; ++e) acc[r][e] += ds[((warp * kRows + r) * V + e) * 32 + lane];
      }
    }
    if (warp == 0) {
#pragma unroll
      for (int r = 0; r < kRows; ++r)
        if (r < rows) C::store(acc[r], static_cast<T*>(q.y) + (row0 + r) * q.ldy + j0, lane, cols, q.out16);
    }
  }
}

template <typename T, bool ON16>
__global__ void __launch_bounds__(kThreads, 3) dw_kernel(const FewParams q) {
  using C = Columns<T, ON16>;
  constexpr int V = C::V, kCols = 32 * V, kHigh = kOuts * kWarps;
  __shared__ GroupTable table;
  __shared__ __align__(16) float ds[2][kRows][kHigh];
  make_table(table, q.offsets, q.groups, q.rows, kRows, 0, q.status);
  wait_for_earlier();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long across = q.y ? (q.K + kCols - 1) / kCols : 1, blocks = (q.N + kHigh - 1) / kHigh * across;
  for (long long item = blockIdx.x; item < q.groups * blocks; item += gridDim.x) {
    const int g = static_cast<int>(item / blocks);
    const long long j0 = item % across * kCols, n0 = item % blocks / across * kHigh;
    const int cols = static_cast<int>(min(static_cast<long long>(kCols), q.K - j0));
    const long long first = table.start[g], last = table.start[g + 1];
    float acc[kOuts][V] = {}, sum = 0.0f;
    int buf = 0;
    for (long long r0 = first; r0 < last; r0 += kRows, buf ^= 1) {
      const int rows = static_cast<int>(min(static_cast<long long>(kRows), last - r0));
      for (int e = threadIdx.x; e < kRows * kHigh; e += kThreads) {
        const int r = e / kHigh, n = e % kHigh;
        ds[buf][r][n] = r < rows && n0 + n < q.N ? dz_at<T>(q, r0 + r, n0 + n) : 0.0f;
      }
      __syncthreads();  // (the buffer before may still be read: two take turns)
      if (q.z && j0 == 0 && threadIdx.x < kHigh) {
#pragma unroll
        for (int r = 0; r < kRows; ++r) sum += ds[buf][r][threadIdx.x];
      }
      if (q.y) {
        for (int r = 0; r < rows; ++r) {
          float v[V];
          C::load(v, static_cast<const T*>(q.x) + (r0 + r) * q.ldx + j0, lane, cols, true);
          const float4 a = *reinterpret_cast<const float4*>(&ds[buf][r][kOuts * warp]);
          const float d[kOuts] = {a.x, a.y, a.z, a.w};
#pragma unroll
          for (int o = 0; o < kOuts; ++o)
#pragma unroll
            for (int e = 0; e < V; ++e) acc[o][e] = fmaf(d[o], v[e], acc[o][e]);
        }
      }
    }
    if (q.y) {
#pragma unroll
      for (int o = 0; o < kOuts; ++o) {
        const long long n = n0 + kOuts * warp + o;
        if (n < q.N) C::store(acc[o], static_cast<T*>(q.y) + g * q.y_group + n * q.ldy + j0, lane, cols, q.out16);
      }
    }
    if (q.z && j0 == 0 && threadIdx.x < kHigh && n0 + threadIdx.x < q.N)
      static_cast<T*>(q.z)[g * q.ldz + n0 + threadIdx.x] = from_f32<T>(sum);
    __syncthreads();
  }
}

// Whether the rows of a matrix, or of one for each group, begin on 16-byte boundaries.
bool on16(const void* m, long long ld, long long group, int groups, int elem) {
  return reinterpret_cast<uintptr_t>(m) % 16 == 0 && ld * elem % 16 == 0 && (groups == 1 || group * elem % 16 == 0);
}

unsigned grid(long long work, int ctas) {
  const long long most = static_cast<long long>(kSms) * ctas;
  return static_cast<unsigned>(work < 1 ? 1 : work < most ? work : most);
}

template <typename T>
int forward(FewParams q, Chain& s) {
  const long long work = (q.rows / kRows + q.groups) * ((q.N + kOuts * kWarps - 1) / (kOuts * kWarps));
  if (on16(q.w, q.ldw, q.w_group, q.groups, sizeof(T)))
    return s.launch(forward_kernel<T, true>, dim3(grid(work, 2)), kThreads, 0, q);
  return s.launch(forward_kernel<T, false>, dim3(grid(work, 2)), kThreads, 0, q);
}
template <typename T>
int backward_x(FewParams q, Chain& s) {
  constexpr int kCols = 32 * 16 / sizeof(T);
  const long long work = (q.rows / kRows + q.groups) * ((q.K + kCols - 1) / kCols);
  q.out16 = on16(q.y, q.ldy, 0, 1, sizeof(T));
  if (on16(q.w, q.ldw, q.w_group, q.groups, sizeof(T)))
    return s.launch(dx_kernel<T, true>, dim3(grid(work, 2)), kThreads, 0, q);
  return s.launch(dx_kernel<T, false>, dim3(grid(work, 2)), kThreads, 0, q);
}
template <typename T>
int backward_w(FewParams q, Chain& s) {
  constexpr int kCols = 32 * 16 / sizeof(T), kHigh = kOuts * kWarps;
  const long long work = q.groups * ((q.N + kHigh - 1) / kHigh) * (q.y ? (q.K + kCols - 1) / kCols : 1);
  q.out16 = on16(q.y, q.ldy, q.y_group, q.groups, sizeof(T));
  if (on16(q.x, q.ldx, 0, 1, sizeof(T)) && q.out16)
    return s.launch(dw_kernel<T, true>, dim3(grid(work, 3)), kThreads, 0, q);
  return s.launch(dw_kernel<T, false>, dim3(grid(work, 3)), kThreads, 0, q);
}

FewParams params(const GroupProduct& p) {
  FewParams q{};
  q.w = p.b, q.ldw = p.b_k == 1 ? p.b_j : p.b_k, q.w_group = p.b_group;
  q.rows = p.rows, q.groups = p.groups, q.offsets = p.offsets, q.status = p.status;
  q.y = p.y, q.ldy = p.ldy, q.y_group = p.y_group;
  return q;
}

}  // namespace

int few_forward(const GroupProduct& p, int dtype, Chain& s) {
  FewParams q = params(p);
  q.x = p.a, q.ldx = p.a_i;
  q.K = p.K, q.N = p.J;
  q.bias = p.bias, q.bias_group = p.bias_group, q.z = p.pre, q.ldz = p.ldpre, q.act = p.act;
  if (dtype == PIC_DTYPE_F32) return forward<float>(q, s);
  if (dtype == PIC_DTYPE_F16) return forward<__half>(q, s);
  return forward<__nv_bfloat16>(q, s);
}

int few_dx(const GroupProduct& p, int dtype, Chain& s) {
  FewParams q = params(p);
  q.dy = p.a, q.lddy = p.a_i, q.pre = p.a_pre, q.ldpre = p.a_pre_i, q.act = p.a_pre ? p.a_act : PIC_ACT_NONE;
  q.K = p.J, q.N = p.K;
  if (dtype == PIC_DTYPE_F32) return backward_x<float>(q, s);
  if (dtype == PIC_DTYPE_F16) return backward_x<__half>(q, s);
  return backward_x<__nv_bfloat16>(q, s);
}

int few_dw(const GroupProduct& p, void* db, long long db_group, int dtype, Chain& s) {
  FewParams q = params(p);
  q.dy = p.a, q.lddy = p.a_i, q.pre = p.a_pre, q.ldpre = p.a_pre_i, q.act = p.a_pre ? p.a_act : PIC_ACT_NONE;
  q.x = p.b, q.ldx = p.b_k;
  q.K = p.J, q.N = p.I;
  q.z = db, q.ldz = db_group;
  if (dtype == PIC_DTYPE_F32) return backward_w<float>(q, s);
  if (dtype == PIC_DTYPE_F16) return backward_w<__half>(q, s);
  return backward_w<__nv_bfloat16>(q, s);
}

}  // namespace grp
}  // namespace pic
