// k_group_planes.cu -- large grouped products of fp32 matrices on the tensor cores, as
// k_linear_planes.cu's: operands are cut into three planes of bfloat16 pieces (cut3.cuh)
// once, in the workspace, and a pair of CTAs computes tiles of 256 rows x 128 columns
// with six MMAs for every 16 of K, whose sums the epilogue takes over into registers
// after every 128 of K and adds there to nearest.
//
// In the planes each group's rows begin on a multiple of 64 (kAlign), and the rows from
// its last to the next such multiple are zeros; so are the rows of a group's weights from
// its last to the next multiple of 64.  A sum over a group's rows, or over its weights'
// rows, is then one over whole slices of 64 with nothing of a neighbour's in them, not
// even a NaN.  A tile's rows behind the group's are loaded and not stored.
//
// Blocks of 128 x 128 that have an infinite or NaN value are marked, and an epilogue warp
// sums a takeover's K again with FP32 FMAs, from the matrices as they were, where a block
// that its rows or columns meet there is marked.
//
// Measured: the gradient of 16 groups of 256 -> 512 with 4096 rows 82 us (by FP32 FMAs 143):
// six launches (with cold caches dz and db 17 us, the cut 18, the products 29 and 30, parts
// 12), whose 100 or so tiles are less than two rounds; 16000 x 300 -> 1000 91 us (435).
#include "cut3.cuh"
#include "group.cuh"
#include "k_linear_planes.cuh"

namespace pic {
namespace grp {
namespace {

using lin::cut_a;
using lin::cut_b;
using lin::kPieces;
using lin::kPlBlock;
using lin::kPlCols;
using lin::kPlRows;
using lin::kSlice;

constexpr int kSms = 152;
constexpr int kAlign = 64;
constexpr int kEpi = 8;
constexpr int kThreads = 64 + 32 * kEpi;
constexpr int kTakeover = 2;  // slices
constexpr int kHalf = 32;     // K of a stage, half a slice
constexpr int kABytes = 128 * 2 * kHalf, kBBytes = kPlCols / 2 * 2 * kHalf;  // one plane of one CTA
constexpr int kBlock = kHalf * 128;  // 64 rows of an operand that lies along them
constexpr int kStageBytes = kPieces * (kABytes + kBBytes);
constexpr int kStages = 5;
constexpr int kBufs = 4;
constexpr int kBars = 2 * kStages + 2 * kBufs + 1;
constexpr int kOffPanels = kStages * kStageBytes;
constexpr int kOffTable = kOffPanels + kEpi * lin::kTurnBytes;
constexpr int kOffTiles = kOffTable + static_cast<int>(sizeof(GroupTable));  // tiles before each group's
constexpr int kOffBars = (kOffTiles + 4 * (kMaxGroups + 1) + 15) / 16 * 16;
constexpr int kSmem = kOffBars + kBars * 8 + 16 + 1024;
constexpr int kTmemCols = kBufs * kPlCols;
static_assert(kSmem <= 227 * 1024, "shared memory of an SM");

// An operand's matrix as it was, and the marks of the blocks of its planes.
struct Source {
  const float* m;
  long long ld, group;  // group: of weights, from one matrix to the next
  const int* marks;
  int col_blocks;
};

struct GpParams {
  long long rows, I, J, K;
  long long tiles_i, tiles_j;  // sums: of a group
  int groups;
  const long long* offsets;
  int sums;       // over the groups' rows; else by rows
  int b_mn;       // by rows: the weights lie along j
  int w_rows;     // by rows: of a group's weights in the planes
  int chunk;      // sums: rows of a part, a multiple of 128
  float* parts;
  Source a, b;
  const float* bias;
  long long bias_group;
  float* y;
  long long ldy, y_group;
  float* pre;
  long long ldpre;
  int act;
  Waits waits;
};
struct GpMaps {
  CUtensorMap a, b;
};

// Whether a block of rows [r0, r1) and columns [c0, c1) of the planes is marked.
__device__ __forceinline__ bool marked(const Source& o, long long r0, long long r1, long long c0, long long c1,
                                       long long row_blocks, int lane) {
  const long long ra = r0 / kPlBlock, rb = min((r1 - 1) / kPlBlock, row_blocks - 1);
  const int ca = static_cast<int>(c0 / kPlBlock), cb = static_cast<int>(min((c1 - 1) / kPlBlock, o.col_blocks - 1LL));
  bool bad = false;
  for (long long r = ra; r <= rb; ++r)
    for (int c = ca + lane; c <= cb; c += 32) bad |= o.marks[r * o.col_blocks + c] != 0;
  return __any_sync(0xffffffffu, bad);
}

struct Item {
  int g, first, len, at;  // the group, its rows, and where they begin in the planes
  long long ti, tj;
  int k0, k1;             // slices
  int item;
  bool whole;
};

__device__ __forceinline__ Item item_of(const GpParams& q, const GroupTable& t, const int* tiles, long long w) {
  Item m;
  const auto find = [&](int n) {
    int lo = 0, hi = q.groups - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (tiles[mid + 1] <= n)
        lo = mid + 1;
      else
        hi = mid;
    }
    return lo;
  };
  if (q.sums) {
    const long long per = q.tiles_i * q.tiles_j;
    m.item = static_cast<int>(w / per);
    m.g = find(m.item);
    lin::tile_place<kPlRows>(w % per, q.tiles_i, q.tiles_j, m.ti, m.tj);
  } else {
    long long rt;
    lin::tile_place<kPlRows>(w, tiles[q.groups], q.tiles_j, rt, m.tj);
    m.g = find(static_cast<int>(rt));
    m.ti = rt - tiles[m.g];
  }
  m.first = t.start[m.g], m.len = t.rows(m.g), m.at = t.tiles[m.g] * kAlign;
  m.k0 = 0, m.k1 = static_cast<int>((q.K + kSlice - 1) / kSlice);
  if (q.sums) {
    m.whole = m.len <= q.chunk;
    m.k0 = (m.item - tiles[m.g]) * (q.chunk / kSlice);
    m.k1 = min((m.len + kSlice - 1) / kSlice, m.k0 + q.chunk / kSlice);
  }
  return m;
}

// Which blocks of the planes the operands' slices [c0, c1) of a tile are in.
__device__ __forceinline__ bool marked_in(const GpParams& q, const Item& m, uint32_t rank, int c0, int c1, long long all_rows,
                                          int lane) {
  const long long row_blocks = (all_rows + kPlBlock - 1) / kPlBlock;
  const long long i = m.ti * kPlRows + rank * 128, j = m.tj * kPlCols, ka = c0 * 64LL, kb = c1 * 64LL;
  if (q.sums)
    return marked(q.a, m.at + ka, m.at + kb, i, i + 128, row_blocks, lane) ||
           marked(q.b, m.at + ka, m.at + kb, j, j + kPlCols, row_blocks, lane);
  const long long w0 = static_cast<long long>(m.g) * q.w_rows, w_blocks = (static_cast<long long>(q.groups) * q.w_rows + kPlBlock - 1) / kPlBlock;
  return marked(q.a, m.at + i, m.at + i + 128, ka, kb, row_blocks, lane) ||
         (q.b_mn ? marked(q.b, w0 + ka, w0 + kb, j, j + kPlCols, w_blocks, lane)
                 : marked(q.b, w0 + j, w0 + j + kPlCols, ka, kb, w_blocks, lane));
}

// The takeovers of an item of which some are marked: those from memory again.  A function
// of its own, so that it takes no registers from the usual path.
struct TakeMarked {
  Item m;
  uint32_t rank, tmem, bar_acc, lead_free;
  long long row, col0, all_rows;
  int lane;
  bool withhold;
  volatile int* abort_flag;
};
__device__ __noinline__ bool take_marked(float* out, const GpParams& q, const TakeMarked& k, int buf, uint32_t phase) {
  float v[64] = {};
  const Item& m = k.m;
  for (int c0 = m.k0; c0 < m.k1; c0 += kTakeover) {
    if (!__all_sync(0xffffffffu, lin::wait_bounded(k.bar_acc + 8 * buf, phase, k.abort_flag, q.waits))) return false;
    tc::tc_fence_after();
    const int c1 = min(m.k1, c0 + kTakeover);
    if (marked_in(q, m, k.rank, c0, c1, k.all_rows, k.lane)) {
      const float* a = q.a.m + m.first * q.a.ld;
      if (q.sums)
        lin::sum_again(v, a, 1, q.a.ld, q.b.m + m.first * q.b.ld, 1, q.b.ld, k.row, q.I, k.col0, q.J, c0 * 64LL,
                       min(static_cast<long long>(m.len), c1 * 64LL));
      else
        lin::sum_again(v, a, q.a.ld, 1, q.b.m + m.g * q.b.group, q.b_mn ? 1 : q.b.ld, q.b_mn ? q.b.ld : 1, k.row,
                       static_cast<long long>(m.len), k.col0, q.J, c0 * 64LL, min(q.K, c1 * 64LL));
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t r[32];
        tc::tmem_ld32_wait(k.tmem + buf * kPlCols + 32 * h, r);
#pragma unroll
        for (int c = 0; c < 32; ++c) v[32 * h + c] += __uint_as_float(r[c]);
      }
    }
    tc::tc_fence_before();
    __syncwarp();
    if (k.lane == 0 && !k.withhold) tc::mbar_arrive_cluster(k.lead_free + 8 * buf);
    if (++buf == kBufs) buf = 0, phase ^= 1;
  }
#pragma unroll
  for (int c = 0; c < 64; ++c) out[c] = v[c];
  return true;
}

__global__ void __launch_bounds__(kThreads, 1) planes_kernel(const __grid_constant__ GpParams q, const __grid_constant__ GpMaps maps) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = tc::smem_addr(smem_raw);
  uint8_t* smem = smem_raw + ((1024 - (raw & 1023)) & 1023);
  const uint32_t base = tc::smem_addr(smem);
  GroupTable& table = *reinterpret_cast<GroupTable*>(smem + kOffTable);
  int* tiles = reinterpret_cast<int*>(smem + kOffTiles);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = tc::cluster_rank();
  const uint32_t bars = base + kOffBars;
  const uint32_t bar_full = bars, bar_empty = bars + 8 * kStages, bar_acc = bar_empty + 8 * kStages,
                 bar_free = bar_acc + 8 * kBufs, bar_drain = bar_free + 8 * kBufs;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + kOffBars + 8 * kBars);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kOffBars + 8 * kBars + 4);

  if (threadIdx.x == 0) {
    tc::prefetch_map(&maps.a);
    tc::prefetch_map(&maps.b);
    for (int s = 0; s < kStages; ++s) {
      tc::mbar_init(bar_full + 8 * s, 1);
      tc::mbar_init(bar_empty + 8 * s, 1);
    }
    for (int b = 0; b < kBufs; ++b) {
      tc::mbar_init(bar_acc + 8 * b, 1);
      tc::mbar_init(bar_free + 8 * b, kEpi * 2);
    }
    tc::mbar_init(bar_drain, 1);
    *abort_flag = 0;
    tc::fence_mbar_init();
  }
  if (warp == 1) tc::tmem_alloc_cg<2>(tc::smem_addr(tmem_slot), kTmemCols);
  // first tiles (items) of the groups, then where they begin in the planes
  make_table(table, q.offsets, q.groups, q.rows, q.sums ? q.chunk : kPlRows, q.sums ? 1 : 0, q.waits.status);
  for (int g = threadIdx.x; g <= q.groups; g += kThreads) tiles[g] = table.tiles[g];
  __syncthreads();
  make_table(table, q.offsets, q.groups, q.rows, kAlign, 0, q.waits.status);
  tc::tc_fence_before();
  __syncthreads();
  tc::cluster_sync();
  tc::tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  wait_for_earlier();
  auto wait = [&](uint32_t bar, uint32_t parity) { return lin::wait_bounded(bar, parity, abort_flag, q.waits); };
  const long long first = blockIdx.x / 2, step = gridDim.x / 2;
  const long long work = tiles[q.groups] * (q.sums ? q.tiles_i * q.tiles_j : q.tiles_j);
  const bool a_mn = q.sums, b_mn = q.sums || q.b_mn;
  // one plane is kABytes (kBBytes) of rows along K (64 bytes each); of an operand
  // along its rows each block of 64 rows has its three planes of kBlock bytes
  const int a_plane = a_mn ? kBlock : kABytes, b_plane = b_mn ? kBlock : kBBytes;

  int s = 0;
  uint32_t phase = 0;
  bool ok = true;
  if (warp == 0) {
    if (tc::elect_one()) {
      const uint32_t lead_full = tc::map_rank(bar_full, 0);
      for (long long w = first; w < work && ok; w += step) {
        const Item m = item_of(q, table, tiles, w);
        const int i0 = static_cast<int>(m.ti * kPlRows + rank * 128), j0 = static_cast<int>(m.tj * kPlCols + rank * 64);
        const int w0 = q.sums ? 0 : m.g * q.w_rows;
        for (int kh = 2 * m.k0; kh < 2 * m.k1; ++kh) {
          if (!(ok = wait(bar_empty + 8 * s, phase ^ 1))) break;
          if (rank == 0) tc::mbar_arrive_expect_tx(bar_full + 8 * s, 2 * kStageBytes);
          const uint32_t sa = base + s * kStageBytes, sb = sa + kPieces * kABytes, bar = lead_full + 8 * s;
          const int k = kh * kHalf;
          if (q.sums) {
            tc::tma_load_planes_pair(sa, &maps.a, i0, m.at + k, bar);
            tc::tma_load_planes_pair(sa + kPieces * kBlock, &maps.a, i0 + 64, m.at + k, bar);
            tc::tma_load_planes_pair(sb, &maps.b, j0, m.at + k, bar);
          } else {
            tc::tma_load_planes_pair(sa, &maps.a, k, m.at + i0, bar);
            if (q.b_mn)
              tc::tma_load_planes_pair(sb, &maps.b, j0, w0 + k, bar);
            else
              tc::tma_load_planes_pair(sb, &maps.b, k, w0 + j0, bar);
          }
          if (++s == kStages) s = 0, phase ^= 1;
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0 && tc::elect_one()) {
      const uint32_t idesc = tc::idesc_16(256, kPlCols, true, a_mn, b_mn);
      const uint32_t a_step = a_mn ? 2048 : 32, b_step = b_mn ? 2048 : 32;
      int buf = 0;
      uint32_t free_phase = 0;
      for (long long w = first; w < work && ok; w += step) {
        const Item m = item_of(q, table, tiles, w);
        for (int c0 = m.k0; c0 < m.k1 && ok; c0 += kTakeover) {
          if (!(ok = wait(bar_free + 8 * buf, free_phase ^ 1))) break;
          tc::tc_fence_after();
          const uint32_t d = tmem + buf * kPlCols;
          const int h0 = 2 * c0, h1 = 2 * min(m.k1, c0 + kTakeover);
          for (int kh = h0; kh < h1 && ok; kh += 2) {
            // a slice's two stages: the products of small pieces of both, then hi hi of both
            const int s2 = s + 1 == kStages ? 0 : s + 1;
            const uint32_t phase2 = s2 == 0 ? phase ^ 1 : phase;
            const auto products = [&](int stage, int t0, int t1, bool begin) {
              const uint32_t sa = base + stage * kStageBytes, sb = sa + kPieces * kABytes;
#pragma unroll
              for (int t = t0; t < t1; ++t)
#pragma unroll
                for (int kk = 0; kk < kHalf / 16; ++kk) {
                  const uint32_t a = sa + cut_a(t) * a_plane + kk * a_step, b = sb + cut_b(t) * b_plane + kk * b_step;
                  tc::mma_16<2>(d, a_mn ? tc::smem_desc_sw128(a, kPieces * kBlock, 1024) : tc::smem_desc_sw64(a),
                                b_mn ? tc::smem_desc_sw128(b, kPieces * kBlock, 1024) : tc::smem_desc_sw64(b), idesc,
                                (!begin || t > t0 || kk > 0) ? 1u : 0u);
                }
            };
            if (!(ok = wait(bar_full + 8 * s, phase))) break;
            tc::tc_fence_after();
            products(s, 0, 5, kh == h0);
            if (!(ok = wait(bar_full + 8 * s2, phase2))) break;
            tc::tc_fence_after();
            products(s2, 0, 5, false);
            products(s, 5, 6, false);
            tc::mma_commit_cg<2>(bar_empty + 8 * s);
            products(s2, 5, 6, false);
            tc::mma_commit_cg<2>(bar_empty + 8 * s2);
            s = s2 + 1, phase = phase2;
            if (s == kStages) s = 0, phase ^= 1;
          }
          if (!ok) break;
          tc::mma_commit_cg<2>(bar_acc + 8 * buf);
          if (++buf == kBufs) buf = 0, free_phase ^= 1;
        }
      }
    }
    __syncwarp();
  } else {
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    float* turn = reinterpret_cast<float*>(smem + kOffPanels + (warp - 2) * lin::kTurnBytes);
    const uint32_t lead_free = tc::map_rank(bar_free, 0);
    const long long all_rows = table.tiles[q.groups] * static_cast<long long>(kAlign);
    int buf = 0;
    for (long long w = first; w < work && ok; w += step) {
      const Item m = item_of(q, table, tiles, w);
      const long long row0 = m.ti * kPlRows + rank * 128 + quarter * 32, col0 = m.tj * kPlCols + half * 64;
      float v[64];
      const bool withhold = q.waits.test_fault && w == 0 && rank == 0 && warp == 2;
      if (m.k0 >= m.k1) {  // a group without rows
#pragma unroll
        for (int c = 0; c < 64; ++c) v[c] = 0.0f;
      } else if (!marked_in(q, m, rank, m.k0, m.k1, all_rows, lane)) {
        for (int c0 = m.k0; c0 < m.k1; c0 += kTakeover) {
          ok = __all_sync(0xffffffffu, wait(bar_acc + 8 * buf, phase));
          if (!ok) break;
          tc::tc_fence_after();
          const uint32_t d = tmem + buf * kPlCols + half * 64 + (static_cast<uint32_t>(quarter * 32) << 16);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t r[32];
            tc::tmem_ld32_wait(d + 32 * h, r);
#pragma unroll
            for (int c = 0; c < 32; ++c)
              v[32 * h + c] = c0 == m.k0 ? __uint_as_float(r[c]) : v[32 * h + c] + __uint_as_float(r[c]);
          }
          tc::tc_fence_before();
          __syncwarp();
          if (lane == 0 && !withhold) tc::mbar_arrive_cluster(lead_free + 8 * buf);
          if (++buf == kBufs) buf = 0, phase ^= 1;
        }
      } else {
        float u[64];
        const TakeMarked k{m, rank, tmem + half * 64 + (static_cast<uint32_t>(quarter * 32) << 16), bar_acc, lead_free,
                           row0 + lane, col0, all_rows, lane, withhold, abort_flag};
        ok = take_marked(u, q, k, buf, phase);
        buf += (m.k1 - m.k0 + kTakeover - 1) / kTakeover;
        phase ^= buf / kBufs & 1, buf %= kBufs;
#pragma unroll
        for (int c = 0; c < 64; ++c) v[c] = u[c];
      }
      if (!ok) break;
      if (q.sums && !m.whole) {
        float4* out = reinterpret_cast<float4*>(q.parts) +
                      (((part_slot(table, m.g, m.item, q.chunk, lane) * q.tiles_i + m.ti) * q.tiles_j + m.tj) * 2 + rank) * 2 * (128 * 16) +
                      half * (128 * 16) + quarter * (32 * 16) + lane;
#pragma unroll
        for (int c = 0; c < 16; ++c) out[c * 32] = make_float4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
        continue;
      }
      lin::Product p{};
      p.I = q.sums ? q.I : m.len, p.J = q.J;
      if (row0 >= p.I || col0 >= p.J) continue;
      p.bias = q.bias ? q.bias + m.g * q.bias_group : nullptr;
      p.y = q.sums ? q.y + m.g * q.y_group : q.y + m.first * q.ldy, p.ldy = q.ldy;
      p.pre = q.pre ? q.pre + m.first * q.ldpre : nullptr, p.ldpre = q.ldpre;
      p.act = q.act;
      lin::finish_rows(v, p, turn, lane, row0, col0);
    }
    __syncwarp();
  }
  tc::tc_fence_before();
  __syncthreads();
  if (*abort_flag) {  // as in k_linear_tc.cuh
    if (warp == 0 && rank == 0 && tc::elect_one()) lin::drain_loads(bar_full, kStages, s, phase, q.waits);
    if (warp == 1 && rank == 0 && tc::elect_one()) lin::drain_mmas<2>(bar_drain, q.waits);
    __nanosleep(200000);
    __syncthreads();
  }
  tc::cluster_sync();
  tc::tc_fence_after();
  if (warp == 1) tc::tmem_dealloc_cg<2>(tmem, kTmemCols);
}

// The planes and marks of a matrix: of rows by group (offsets not null), or of weights,
// `rows` in `padded` rows of each of `groups`.  A block of threads takes 128 x 128.
struct Cut {
  const float* m;
  long long ld, group;
  long long rows, cols;
  int padded, groups;
  const long long* offsets;
  uint16_t* planes;
  long long plane, ld_out;  // elements of a plane
  int* marks;
};
struct Cuts {
  Cut m[3];
};
// The y-th row of blocks takes the y-th matrix.
__global__ void __launch_bounds__(256) cut_kernel(const __grid_constant__ Cuts cuts, int* status) {
  __shared__ GroupTable table;
  const Cut& q = cuts.m[blockIdx.y];
  const bool grouped = q.offsets != nullptr;
  if (grouped) make_table(table, q.offsets, q.groups, q.rows, kAlign, 0, status);
  wait_for_earlier();
  const long long all = grouped ? table.tiles[q.groups] * static_cast<long long>(kAlign) : static_cast<long long>(q.groups) * q.padded;
  const unsigned col_blocks = static_cast<unsigned>((q.cols + kPlBlock - 1) / kPlBlock);
  const long long work = (all + kPlBlock - 1) / kPlBlock * col_blocks;
  const bool vec = reinterpret_cast<uintptr_t>(q.m) % 16 == 0 && q.ld % 4 == 0 && (grouped || q.group % 4 == 0);
  for (long long w = blockIdx.x; w < work; w += gridDim.x) {
    const long long r0 = w / col_blocks * kPlBlock, c0 = w % col_blocks * static_cast<long long>(kPlBlock);
    const long long col = c0 + threadIdx.x % 32 * 4;
    // the group and its place of each 64 rows
    const float* from[2];
    long long left[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const long long r = r0 + kAlign * h;
      left[h] = 0, from[h] = q.m;
      if (r >= all) continue;
      if (grouped) {
        const int g = table.find(static_cast<int>(r / kAlign), q.groups);
        const long long in = r - table.tiles[g] * static_cast<long long>(kAlign);
        left[h] = table.rows(g) - in, from[h] = q.m + (table.start[g] + in) * q.ld;
      } else {
        const long long g = r / q.padded, in = r - g * q.padded;
        left[h] = q.rows - in, from[h] = q.m + g * q.group + in * q.ld;
      }
    }
    uint32_t largest = 0;
#pragma unroll 4
    for (int u = 0; u < kPlBlock / 8; ++u) {
      const int in = threadIdx.x / 32 + u * 8, h = u >= kAlign / 8, at = in - kAlign * h;
      if (r0 + in >= all || col >= q.cols) continue;
      uint32_t v[4] = {0, 0, 0, 0};
      if (at < left[h]) {
        const float* p = from[h] + at * q.ld + col;
        if (vec && col + 4 <= q.cols) {
          const uint4 x = __ldg(reinterpret_cast<const uint4*>(p));
          v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = col + i < q.cols ? __ldg(reinterpret_cast<const uint32_t*>(p) + i) : 0u;
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) largest = max(largest, v[i] & 0x7fffffffu);
      uint32_t h0, m0, l0, h1, m1, l1;
      lin::cut3(v[0], v[1], h0, m0, l0);
      lin::cut3(v[2], v[3], h1, m1, l1);
      // rows are a multiple of eight places: the four are there
      uint16_t* o = q.planes + (r0 + in) * q.ld_out + col;
      *reinterpret_cast<uint2*>(o) = make_uint2(h0, h1);
      *reinterpret_cast<uint2*>(o + q.plane) = make_uint2(m0, m1);
      *reinterpret_cast<uint2*>(o + 2 * q.plane) = make_uint2(l0, l1);
    }
    const int bad = __syncthreads_or(largest >= lin::kCutLimit);
    if (threadIdx.x == 0) q.marks[w] = bad;
  }
}

long long round_up(long long v, long long to) { return (v + to - 1) / to * to; }

// An operand's planes in the workspace.
struct Planes {
  long long rows, cols, ld;  // rows: at most
  long long bytes, mark_bytes;
};
Planes planes_of(long long rows, long long cols) {
  Planes p{rows, cols, round_up(cols, cols < 64 ? 8 : 64), 0, 0};  // wide rows on 128-byte lines
  p.bytes = round_up(3 * rows * p.ld * 2, 256);
  p.mark_bytes = round_up((rows + kPlBlock - 1) / kPlBlock * ((cols + kPlBlock - 1) / kPlBlock) * 4, 256);
  return p;
}

struct Plan {
  Planes a, b;
  long long tiles_i, tiles_j, work;
  int chunk;
  long long part_bytes;
  double time;  // estimated, us
};
Plan plan(const GroupProduct& p) {
  Plan r{};
  const double each = static_cast<double>(p.rows) / p.groups;
  const auto up = [](double a, double b) { return static_cast<double>(static_cast<long long>((a + b - 1) / b)); };
  const long long padded = round_up(p.rows, kAlign) + static_cast<long long>(p.groups) * kAlign;
  r.tiles_j = (p.J + kPlCols - 1) / kPlCols;
  double slices, tiles;
  if (p.by_rows) {
    r.a = planes_of(padded, p.K);
    const long long w_rows = p.b_k == 1 ? p.J : p.K, w_cols = p.b_k == 1 ? p.K : p.J;
    r.b = planes_of(p.groups * round_up(w_rows, kAlign), w_cols);
    r.work = ((p.rows + kPlRows - 1) / kPlRows + p.groups) * r.tiles_j;
    slices = up(static_cast<double>(p.K), kSlice);
    tiles = p.groups * up(each, kPlRows) * r.tiles_j;
    r.time = 0;
  } else {
    r.a = planes_of(padded, p.I);
    r.b = planes_of(padded, p.J);
    r.tiles_i = (p.I + kPlRows - 1) / kPlRows;
    // parts of a group's rows where there are few tiles
    tiles = static_cast<double>(p.groups) * r.tiles_i * r.tiles_j;
    double best = 1e30;
    for (int want = 1; want <= 128; want = want < 8 ? want + 1 : want + want / 8) {
      const long long chunk = round_up(static_cast<long long>(each / want) + 1, 128);
      if (want > 1 && chunk < 256) break;
      const double parts = up(each, static_cast<double>(chunk)), rounds = up(tiles * parts, kSms / 2);
      const double t = rounds * up(static_cast<double>(chunk), kSlice) * 0.95 +
                       (parts > 1 ? 3.0 + tiles * parts * kPlRows * kPlCols * 4 / 2.6e6 : 0.0);
      if (t < best) best = t, r.chunk = static_cast<int>(want == 1 ? (1 << 30) : chunk);
    }
    r.work = (p.rows / r.chunk + p.groups) * r.tiles_i * r.tiles_j;
    const long long slots = p.rows <= r.chunk ? 0 : min(p.rows / r.chunk + p.groups, 2 * (p.rows / r.chunk));
    r.part_bytes = round_up(slots * r.tiles_i * r.tiles_j * kPlRows * kPlCols * 4, 256);
    r.time = best;
    slices = 0;
  }
  if (p.by_rows) r.time = up(tiles, kSms / 2) * slices * 0.95;
  // the cut: 10 bytes of traffic an element
  const double elements = static_cast<double>(p.rows) * r.a.cols + (p.by_rows ? static_cast<double>(r.b.rows) * r.b.cols : static_cast<double>(p.rows) * r.b.cols);
  r.time += 14.0 + elements * 10.0 / 5e6;
  return r;
}

}  // namespace

// (k_group_any.cu's kernel, measured: 16 of K take from 1.3 us with few tiles of 64 x 64 to 4
// with four on each SM)
bool planes_takes(const GroupProduct& p, int dtype) {
  if (dtype != PIC_DTYPE_F32 || p.rows == 0) return false;
  // rows of the planes are counted in 32 bits
  const long long w_rows = p.by_rows ? p.groups * round_up(p.b_k == 1 ? p.J : p.K, kAlign) : 0;
  if (w_rows > 0x7fffffffLL - kPlRows || p.rows + static_cast<long long>(p.groups) * kAlign > 0x7fffffffLL - kPlRows) return false;
  const double each = static_cast<double>(p.rows) / p.groups;
  const auto up = [](double a, double b) { return static_cast<double>(static_cast<long long>((a + b - 1) / b)); };
  const double k = p.by_rows ? static_cast<double>(p.K) : each;
  const double tiles = p.groups * (p.by_rows ? up(each, 64) : up(static_cast<double>(p.I), 64)) * up(static_cast<double>(p.J), 64);
  const double full = tiles / (4 * kSms);
  const double any = 4.0 + up(k, 16) * (full <= 1 ? 1.0 + 3.0 * full : 4.0 * up(full, 1));
  return plan(p).time < any;
}

namespace {

int blocks_of(long long cols) { return static_cast<int>((cols + kPlBlock - 1) / kPlBlock); }

// The planes and marks of an operand, and the job of making them.
struct Made {
  Planes l;
  char *planes, *marks;
  Cut cut;
};
// grouped: of rows by group; else of p's weights.
Made made(const GroupProduct& p, const Planes& l, bool grouped, const void* m, long long ld, long long group, lin::Arena& ws) {
  Made o{l, static_cast<char*>(ws.take(l.bytes)), static_cast<char*>(ws.take(l.mark_bytes)), {}};
  const long long rows = p.b_k == 1 ? p.J : p.K;  // of a group's weights
  o.cut = {static_cast<const float*>(m), ld, group, grouped ? p.rows : rows, l.cols, static_cast<int>(round_up(rows, kAlign)), p.groups,
           grouped ? p.offsets : nullptr, reinterpret_cast<uint16_t*>(o.planes), l.rows * l.ld, l.ld, reinterpret_cast<int*>(o.marks)};
  return o;
}
Made made_a(const GroupProduct& p, const Plan& r, lin::Arena& ws) { return made(p, r.a, true, p.a, p.a_i, 0, ws); }
Made made_b(const GroupProduct& p, const Plan& r, lin::Arena& ws) {
  return made(p, r.b, !p.by_rows, p.b, p.by_rows && p.b_k == 1 ? p.b_j : p.b_k, p.b_group, ws);
}
int cut_all(const Made* const* m, int n, int* status, Chain& s) {
  Cuts c{};
  long long most = 1;
  for (int i = 0; i < n; ++i) {
    c.m[i] = m[i]->cut;
    const long long want = (m[i]->l.rows + kPlBlock - 1) / kPlBlock * blocks_of(m[i]->l.cols);
    if (want > most) most = want;
  }
  return s.launch(cut_kernel, dim3(static_cast<unsigned>(most < 6 * kSms ? most : 6 * kSms), n), 256, 0, c, status);
}

int multiply(const GroupProduct& p, const Plan& r, const Made& a, const Made& b, float* parts, const Waits& waits, Chain& s) {
  GpParams q{};
  GpMaps maps;
  q.rows = p.rows, q.I = p.I, q.J = p.J, q.K = p.K;
  q.tiles_i = r.tiles_i, q.tiles_j = r.tiles_j;
  q.groups = p.groups, q.offsets = p.offsets;
  q.sums = !p.by_rows;
  q.b_mn = p.by_rows && p.b_k != 1;
  q.w_rows = b.cut.padded;
  q.chunk = r.chunk;
  q.parts = parts;
  const auto source = [](const Made& o) { return Source{o.cut.m, o.cut.ld, o.cut.group, o.cut.marks, blocks_of(o.l.cols)}; };
  q.a = source(a), q.b = source(b);
  q.bias = static_cast<const float*>(p.bias), q.bias_group = p.bias_group;
  q.y = static_cast<float*>(p.y), q.ldy = p.ldy, q.y_group = p.y_group;
  q.pre = static_cast<float*>(p.pre), q.ldpre = p.ldpre, q.act = p.act;
  q.waits = waits;
  // 32 of K: along K a box of the CTA's rows, else blocks of 64 rows
  if (!(q.sums ? lin::encode_planes(&maps.a, a.planes, a.l.rows, a.l.cols, a.l.ld, 64, 32)
               : lin::encode_planes(&maps.a, a.planes, a.l.rows, a.l.cols, a.l.ld, 32, 128)) ||
      !(q.sums || q.b_mn ? lin::encode_planes(&maps.b, b.planes, b.l.rows, b.l.cols, b.l.ld, 64, 32)
                         : lin::encode_planes(&maps.b, b.planes, b.l.rows, b.l.cols, b.l.ld, 32, 64)))
    return PIC_ERR_CUDA;
  const void* fn = reinterpret_cast<const void*>(planes_kernel);
  if (lin::allow_smem(fn, 54, kSmem) != PIC_OK) return PIC_ERR_CUDA;
  const long long want = 2 * r.work;
  void* args[] = {&q, &maps};
  if (s.launch(fn, dim3(static_cast<unsigned>(want < kSms ? want : kSms)), kThreads, kSmem, 2, args) != PIC_OK) return PIC_ERR_CUDA;
  if (r.part_bytes == 0) return PIC_OK;
  const JoinParams j{p.offsets, p.rows, p.I, p.J, r.tiles_i, r.tiles_j, p.groups, r.chunk, kPlCols,
                     reinterpret_cast<const float4*>(q.parts), p.y, p.ldy, p.y_group, waits.status};
  return join_parts(j, kPlRows, PIC_DTYPE_F32, s);
}

}  // namespace

int planes_product(const GroupProduct& p, lin::Arena& ws, bool launch, const Waits& waits, Chain& s) {
  const Plan r = plan(p);
  const Made a = made_a(p, r, ws), b = made_b(p, r, ws);
  float* parts = static_cast<float*>(ws.take(r.part_bytes));
  if (!launch) return PIC_OK;
  const Made* both[] = {&a, &b};
  const int rc = cut_all(both, 2, waits.status, s);
  return rc == PIC_OK ? multiply(p, r, a, b, parts, waits, s) : rc;
}

int planes_gradients(const GroupProduct& dx, const GroupProduct& dw, lin::Arena& ws, bool launch, const Waits& waits, Chain& s) {
  const Plan rx = plan(dx), rw = plan(dw);
  // the same planes of dz serve both
  const Made dz = made_a(dx, rx, ws), w = made_b(dx, rx, ws), x = made_b(dw, rw, ws);
  float* parts = static_cast<float*>(ws.take(rw.part_bytes));
  if (!launch) return PIC_OK;
  const Made* all[] = {&dz, &w, &x};
  int rc = cut_all(all, 3, waits.status, s);
  if (rc == PIC_OK) rc = multiply(dx, rx, dz, w, nullptr, waits, s);
  return rc == PIC_OK ? multiply(dw, rw, dz, x, parts, waits, s) : rc;
}

}  // namespace grp
}  // namespace pic
