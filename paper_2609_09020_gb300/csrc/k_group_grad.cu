// k_group_grad.cu -- the elementwise part of the grouped layers' gradient: dz = dy
// act'(z), and its column sums over each group's rows.  As k_linear_grad.cu, bound by
// memory: a thread takes 16 bytes of neighbouring columns of every so many-th row of a
// run of rows of one group; the block adds its threads' sums in shared memory, and a
// second kernel the sums of a group's runs in order.  Measured: bf16 8192 x 4096 GELU with dz
// 45 us for 201 MB, 4.5 TB/s (GELU' is some 20 instructions an element).
#include "group.cuh"

namespace pic {
namespace grp {
namespace {

using lin::Piece16;
using lin::to_f32;

constexpr int kThreads = 256;
constexpr int kUnroll = 4;
constexpr int kSms = 152;

struct Share {
  int tx;    // threads across columns
  int run;   // rows of a run
  bool on16;  // rows of dy and z start, and end, on 16-byte boundaries
  long long col_blocks, items;  // items: runs, at most
};

Share share(const GroupGradAct& g, int elem) {
  const auto on16 = [&](const void* p, long long ld) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * elem % 16 == 0;
  };
  Share s;
  const int v = 16 / elem;
  s.on16 = on16(g.dy, g.lddy) && (g.act == PIC_ACT_NONE || on16(g.pre, g.ldpre)) && g.J % v == 0;
  const long long across = (g.J + v - 1) / v;
  s.tx = 1;
  while (s.tx < across && s.tx < 32) s.tx *= 2;
  s.col_blocks = (across + s.tx - 1) / s.tx;
  const int ty = kThreads / s.tx;
  // some eight blocks for each SM, but runs long enough that their sums cost little
  long long run = g.rows * s.col_blocks / (8 * kSms);
  const long long least = static_cast<long long>(ty) * kUnroll;
  run = (run + least - 1) / least * least;
  s.run = static_cast<int>(run < least ? least : run);
  s.items = g.rows / s.run + g.groups;
  return s;
}

// Where the first kernel leaves its table of runs for the second, behind the sums.
__host__ __device__ inline int* table_of(const GroupGradAct& g, const Share& s) {
  return reinterpret_cast<int*>(g.parts + s.items * g.J);
}

template <typename T, bool ON16>
__global__ void __launch_bounds__(kThreads, ON16 ? 4 : 3) grad_act_kernel(const GroupGradAct g, const Share s) {
  constexpr int V = 16 / sizeof(T);
  __shared__ GroupTable table;
  __shared__ float sums[kThreads * V];
  make_table(table, g.offsets, g.groups, g.rows, s.run, 1, g.status);
  wait_for_earlier();
  const int tx = threadIdx.x % s.tx, ty = threadIdx.x / s.tx, rows = kThreads / s.tx, width = s.tx * V;
  const long long work = table.tiles[g.groups] * s.col_blocks;
  if (g.db && g.rows > s.run && blockIdx.x == 0)
    for (int i = threadIdx.x; i <= g.groups; i += kThreads) table_of(g, s)[i] = table.tiles[i];
  for (long long w = blockIdx.x; w < work; w += gridDim.x) {
    const int item = static_cast<int>(w / s.col_blocks), at = table.find(item, g.groups);
    const long long col_block = w % s.col_blocks, j = (col_block * s.tx + tx) * V;
    const int part = item - table.tiles[at];
    const long long i0 = table.start[at] + static_cast<long long>(part) * s.run,
                    i1 = min(static_cast<long long>(table.start[at + 1]), i0 + s.run);
    float sum[V] = {};
    if (j < g.J) {
      const T* dy = static_cast<const T*>(g.dy) + j;
      const T* pre = static_cast<const T*>(g.pre) + j;
      T* dz = static_cast<T*>(g.dz) + j;
      const auto row = [&](const uint32_t (&a)[4], const uint32_t (&z)[4], long long r) {
        float d[V];
#pragma unroll
        for (int e = 0; e < V; ++e) d[e] = to_f32(reinterpret_cast<const T*>(a)[e]);
        if (g.act != PIC_ACT_NONE) {
          const T* v = reinterpret_cast<const T*>(z);
#pragma unroll
          for (int e = 0; e < V; e += 2) {
            const float2 f = lin::act_grad2<sizeof(T) == 4>(make_float2(d[e], d[e + 1]),
                                                            make_float2(to_f32(v[e]), to_f32(v[e + 1])), g.act);
            d[e] = f.x;
            d[e + 1] = f.y;
          }
        }
        uint32_t out[4];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          sum[e] += d[e];
          reinterpret_cast<T*>(out)[e] = lin::from_f32<T>(d[e]);
        }
        if (g.dz) *reinterpret_cast<uint4*>(dz + r * g.lddz) = make_uint4(out[0], out[1], out[2], out[3]);
      };
      constexpr int kRows = ON16 ? kUnroll : kUnroll / 2;
      const int bytes = static_cast<int>(min(static_cast<long long>(V), g.J - j) * sizeof(T));
      for (long long i = i0 + ty; i < i1; i += rows * kRows) {
        Piece16<ON16> a[kRows], z[kRows];
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
          const long long r = i + u * rows;
          a[u].load(reinterpret_cast<const char*>(dy + r * g.lddy), r < i1 ? bytes : 0);
          if (g.act != PIC_ACT_NONE) z[u].load(reinterpret_cast<const char*>(pre + r * g.ldpre), r < i1 ? bytes : 0);
        }
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
          const long long r = i + u * rows;
          if (r >= i1) break;
          uint32_t v[4], x[4] = {};
          a[u].template get<T>(static_cast<int>(reinterpret_cast<uintptr_t>(dy + r * g.lddy) & 15), v);
          if (!ON16) lin::keep_bytes<T>(v, bytes);
          if (g.act != PIC_ACT_NONE) {
            z[u].template get<T>(static_cast<int>(reinterpret_cast<uintptr_t>(pre + r * g.ldpre) & 15), x);
            if (!ON16) lin::keep_bytes<T>(x, bytes);
          }
          row(v, x, r);
        }
      }
    }
    if (!g.db) continue;
#pragma unroll
    for (int e = 0; e < V; ++e) sums[ty * width + tx * V + e] = sum[e];
    __syncthreads();
    for (int c = threadIdx.x; c < width; c += kThreads) {
      const long long col = col_block * width + c;
      if (col >= g.J) break;
      float t = 0.0f;
      for (int r = 0; r < rows; ++r) t += sums[r * width + c];
      if (table.tiles[at + 1] - table.tiles[at] == 1)
        static_cast<T*>(g.db)[at * g.db_group + col] = lin::from_f32<T>(t);
      else
        g.parts[item * g.J + col] = t;
    }
    __syncthreads();
  }
}

// A block takes 64 columns of a group that has several runs, four threads a column.
// `tiles`: the first kernel's table of runs.
template <typename T>
__global__ void __launch_bounds__(256) sum_parts_kernel(const GroupGradAct g, const int* tiles) {
  __shared__ float sums[4][64];
  wait_for_earlier();
  const int at = blockIdx.y, tx = threadIdx.x % 64, ty = threadIdx.x / 64;
  const int p0 = __ldcg(tiles + at), p1 = __ldcg(tiles + at + 1);
  if (p1 - p0 < 2) return;
  const long long j = blockIdx.x * 64LL + tx;
  float sum = 0.0f;
  if (j < g.J) {
#pragma unroll 8
    for (int p = p0 + ty; p < p1; p += 4) sum += __ldcg(g.parts + p * g.J + j);
  }
  sums[ty][tx] = sum;
  __syncthreads();
  if (ty == 0 && j < g.J) {
#pragma unroll
    for (int r = 1; r < 4; ++r) sum += sums[r][tx];
    static_cast<T*>(g.db)[at * g.db_group + j] = lin::from_f32<T>(sum);
  }
}

template <typename T>
int run(GroupGradAct g, Chain& chain) {
  const Share s = share(g, sizeof(T));
  const long long most = s.items * s.col_blocks, slots = (s.on16 ? 4 : 3) * kSms;
  const unsigned blocks = static_cast<unsigned>(most < slots ? most : slots);
  const int rc = chain.launch(s.on16 ? grad_act_kernel<T, true> : grad_act_kernel<T, false>, dim3(blocks), kThreads, 0, g, s);
  if (rc != PIC_OK || !g.db || g.rows <= s.run) return rc;
  return chain.launch(sum_parts_kernel<T>, dim3(static_cast<unsigned>((g.J + 63) / 64), g.groups), 256, 0, g,
                      static_cast<const int*>(table_of(g, s)));
}

}  // namespace

long long grad_act_workspace(const GroupGradAct& g, int dtype) {
  const Share s = share(g, dtype == PIC_DTYPE_F32 ? 4 : 2);
  return g.db && g.rows > s.run ? (s.items * g.J + g.groups + 1) * 4 : 0;
}

int grad_act(const GroupGradAct& g, int dtype, Chain& s) {
  if (dtype == PIC_DTYPE_F32) return run<float>(g, s);
  if (dtype == PIC_DTYPE_F16) return run<__half>(g, s);
  return run<__nv_bfloat16>(g, s);
}

}  // namespace grp
}  // namespace pic
