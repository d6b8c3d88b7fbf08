// k_group_tc.cu -- host side of the grouped products on the tensor cores: tile
// shapes, parts, tensor maps; and the small kernels around them, which lay out
// matrices that TMA cannot read, make the groups' maps and join parts.
#include "k_group_tc.cuh"

namespace pic {
namespace grp {
namespace {

constexpr int kSms = 152;

long long round_up(long long v, long long to) { return (v + to - 1) / to * to; }

// Rows that start on 16-byte boundaries, from ones that do not: a thread puts eight
// elements together from the aligned 16-byte pieces that hold them.
struct Pad {
  const uint16_t* src;
  long long ld, group;   // elements from row to row, from matrix to matrix
  long long rows, count;  // of a matrix; matrices
  int cols;
  uint4* dst;            // [count][rows][ld_out / 8]
  int ld_out;
};
__global__ void __launch_bounds__(256) pad_kernel(const Pad q) {
  wait_for_earlier();
  const int chunks = (q.cols + 7) / 8;
  const long long all = q.rows * q.count * chunks;
  for (long long e = blockIdx.x * 256LL + threadIdx.x; e < all; e += gridDim.x * 256LL) {
    const long long r = e / chunks;
    const int c = static_cast<int>(e - r * chunks);
    const uint16_t* p = q.src + r / q.rows * q.group + r % q.rows * q.ld + c * 8;
    const int bytes = min(8, q.cols - c * 8) * 2;
    lin::Piece16<false> v;
    v.load(reinterpret_cast<const char*>(p), bytes);
    uint32_t w[4];
    v.get<uint16_t>(static_cast<int>(reinterpret_cast<uintptr_t>(p) & 15), w);
    lin::keep_bytes<uint16_t>(w, bytes);
    q.dst[r * (q.ld_out / 8) + c] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// The groups' tensor maps: those of the whole matrices, cut off behind each group's last
// row.  Their base stays the matrix's, and a group's first row is a coordinate: a map that
// was encoded for more than 128 KB may be used by the copy engine as if that much were
// mapped from its base on, and behind a later row it need not be (with the group's first
// row as the base, sums over a last small group faulted where memory ended behind them).
struct MakeMaps {
  const long long* offsets;
  long long rows;
  CUtensorMap* out;  // [groups][2]
};
__global__ void __launch_bounds__(32) maps_kernel(const MakeMaps q, const __grid_constant__ GtMaps maps) {
  __shared__ __align__(128) uint32_t sm[2][32];
  const int g = blockIdx.x, lane = threadIdx.x;
  wait_for_earlier();
  // an offset counts as the largest so far, within [0, rows]
  long long first = 0;
  for (int i = lane; i <= g; i += 32) first = max(first, q.offsets[i]);
#pragma unroll
  for (int d = 16; d > 0; d /= 2) first = max(first, __shfl_xor_sync(0xffffffffu, first, d));
  first = min(first, q.rows);
  const long long last = min(max(first, q.offsets[g + 1]), q.rows);
  if (last <= first) return;
  sm[0][lane] = reinterpret_cast<const uint32_t*>(&maps.a)[lane];
  sm[1][lane] = reinterpret_cast<const uint32_t*>(&maps.b)[lane];
  __syncwarp();
  if (lane < 2)
    asm volatile("tensormap.replace.tile.global_dim.shared::cta.b1024.b32 [%0], 1, %1;" ::"r"(tc::smem_addr(sm[lane])),
                 "r"(static_cast<uint32_t>(last))
                 : "memory");
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 2; ++i)
    asm volatile("tensormap.cp_fenceproxy.global.shared::cta.tensormap::generic.release.gpu.sync.aligned [%0], [%1], 128;" ::"l"(
                     reinterpret_cast<uint64_t>(q.out + 2 * g + i)),
                 "r"(tc::smem_addr(sm[i]))
                 : "memory");
}

// (group.cuh)
template <typename T, int ROWS>
__global__ void __launch_bounds__(256) join_kernel(const JoinParams q) {
  __shared__ GroupTable table;
  make_table(table, q.offsets, q.groups, q.rows, q.chunk, 1, q.status);
  wait_for_earlier();
  const int g = blockIdx.y;
  const int parts = table.tiles[g + 1] - table.tiles[g];
  if (parts < 2) return;
  const long long slot = part_slot(table, g, table.tiles[g], q.chunk, threadIdx.x & 31);
  const int per_tile = ROWS * q.bn / 4;
  const long long tile = blockIdx.x / (per_tile / 256);
  const long long ti = tile / q.tiles_j, tj = tile % q.tiles_j;
  const lin::JoinItem m = lin::join_place<ROWS>(static_cast<int>(blockIdx.x % (per_tile / 256)) * 256 + threadIdx.x, q.bn, ti, tj);
  if (m.i >= q.I || m.j >= q.J) return;
  const long long step = q.tiles_i * q.tiles_j * per_tile;
  const float4* at = q.parts + slot * step + tile * per_tile + m.at;
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
  for (int s = 0; s < parts; ++s) {
    const float4 f = __ldcg(at + s * step);
    v.x += f.x, v.y += f.y, v.z += f.z, v.w += f.w;
  }
  lin::Product p{};
  p.I = q.I, p.J = q.J;
  p.y = static_cast<T*>(q.y) + g * q.y_group, p.ldy = q.ldy;
  p.act = PIC_ACT_NONE;
  lin::finish_item<T>(p, m, v);
}

// A matrix, or several, as TMA reads them.
struct Operand {
  const void* m;
  long long rows, cols, ld, count, group;
  bool pad;
  long long bytes;  // of the workspace
};
Operand operand(const void* m, long long rows, long long cols, long long ld, long long count, long long group) {
  Operand o{m, rows, cols, ld, count, count == 1 ? rows * ld : group, false, 0};
  o.pad = reinterpret_cast<uintptr_t>(m) % 16 != 0 || ld % 8 != 0 || ld * 2 >= (1LL << 40) || o.group % 8 != 0 ||
          o.group * 2 >= (1LL << 40);
  if (o.pad) {
    o.ld = round_up(cols, 64);  // rows on 128-byte lines
    o.group = rows * o.ld;
    o.bytes = round_up(count * o.group * 2, 256);
  }
  return o;
}

struct Plan {
  TcMode mode;
  int bn, cg, chunk;
  long long tiles_i, tiles_j, work;  // work: at most
  Operand a, b;
  long long map_bytes, part_bytes;
};

// Times of tiles as measured for one product (k_linear_tc.cu), in microseconds: launch,
// first loads and last epilogue; 64 of K of a tile; a tile's epilogue.
struct ShapeCost {
  int bn, cg, slots;
  double fixed, slice, tile;
};
constexpr ShapeCost kShapes[] = {{64, 1, 2 * kSms, 4.2, 0.20, 3.0}, {128, 1, kSms, 4.5, 0.19, 2.2}, {256, 2, kSms / 2, 6.8, 0.26, 3.4}};

// Tile shapes, and for sums the parts, with the least estimated time if all groups have as
// many rows.
Plan plan(const GroupProduct& p) {
  Plan r{};
  const double each = static_cast<double>(p.rows) / p.groups;
  const auto ceil_div = [](double a, double b) { return static_cast<double>(static_cast<long long>((a + b - 1) / b)); };
  double best = 1e30;
  if (p.by_rows) {
    r.a = operand(p.a, p.rows, p.K, p.a_i, 1, 0);
    r.b = p.b_k == 1 ? operand(p.b, p.J, p.K, p.b_j, p.groups, p.b_group) : operand(p.b, p.K, p.J, p.b_k, p.groups, p.b_group);
    const double slices = ceil_div(static_cast<double>(p.K), kSlice);
    r.mode = each <= 48 ? kTurned : kRows;
    if (r.mode == kTurned) {
      r.bn = each <= 8 ? 16 : each <= 20 ? 32 : 64, r.cg = 1;
      r.tiles_i = (p.J + 127) / 128, r.tiles_j = 0;
      r.work = ((p.rows + r.bn - 1) / r.bn + p.groups) * r.tiles_i;
    } else {
      for (const ShapeCost& h : kShapes) {
        const double tiles = p.groups * ceil_div(each, 128.0 * h.cg) * ceil_div(static_cast<double>(p.J), h.bn);
        const double rounds = ceil_div(tiles, h.slots);
        const double one = slices * h.slice * (h.bn == 64 && tiles > kSms ? 1.5 : 1.0);
        const double t = h.fixed + rounds * (rounds > 1 && one < h.tile ? h.tile : one);
        if (t < best) best = t, r.bn = h.bn, r.cg = h.cg;
      }
      r.tiles_j = (p.J + r.bn - 1) / r.bn;
      r.work = ((p.rows + 128 * r.cg - 1) / (128 * r.cg) + p.groups) * r.tiles_j;
    }
    return r;
  }
  r.mode = kSums;
  r.a = operand(p.a, p.rows, p.I, p.a_i, 1, 0);
  r.b = operand(p.b, p.rows, p.J, p.b_k, 1, 0);
  r.map_bytes = round_up(p.groups * 2LL * sizeof(CUtensorMap), 256);
  for (const ShapeCost& h : kShapes) {
    const long long ti = (p.I + 128 * h.cg - 1) / (128 * h.cg), tj = (p.J + h.bn - 1) / h.bn;
    for (int want = 1; want <= 256; want = want < 8 ? want + 1 : want + want / 8) {
      const long long even = round_up(static_cast<long long>(each / want) + 1, kSlice);
      if (want > 1 && even < 256) break;
      const long long chunk = even < kTcMostK ? even : kTcMostK;
      const double parts = ceil_div(each, static_cast<double>(chunk));
      const double tiles = p.groups * static_cast<double>(ti * tj) * parts, rounds = ceil_div(tiles, h.slots);
      const double one = static_cast<double>(chunk) / kSlice * h.slice * (h.bn == 64 && tiles > kSms ? 1.5 : 1.0);
      double t = h.fixed + rounds * (rounds > 1 && one < h.tile ? h.tile : one);
      if (parts > 1) t += 3.0 + 4.0 * 128 * h.cg * h.bn * tiles / 2.6e6;
      if (t < best) {
        best = t, r.bn = h.bn, r.cg = h.cg;
        // groups somewhat larger than others are not cut where none has to be
        r.chunk = static_cast<int>(want == 1 ? kTcMostK : chunk);
      }
    }
  }
  r.tiles_i = (p.I + 128 * r.cg - 1) / (128 * r.cg), r.tiles_j = (p.J + r.bn - 1) / r.bn;
  r.work = (p.rows / r.chunk + p.groups) * r.tiles_i * r.tiles_j;
  // parts: a group of n > 1 has more than (n - 1) chunk rows, so all of them are at most
  // twice the chunks in all rows, and no more than there are pieces
  const long long slots = p.rows <= r.chunk ? 0 : min(p.rows / r.chunk + p.groups, 2 * (p.rows / r.chunk));
  r.part_bytes = round_up(slots * r.tiles_i * r.tiles_j * 128 * r.cg * r.bn * 4, 256);
  return r;
}

int pad(const Operand& o, long long ld, long long group, void* to, Chain& s) {
  const Pad q{static_cast<const uint16_t*>(o.m), ld, group, o.rows, o.count, static_cast<int>(o.cols),
              static_cast<uint4*>(to), static_cast<int>(o.ld)};
  const long long blocks = (o.rows * o.count * ((o.cols + 7) / 8) + 255) / 256;
  return s.launch(pad_kernel, dim3(static_cast<unsigned>(blocks < 16 * kSms ? blocks : 16 * kSms)), 256, 0, q);
}

template <typename T>
int join(JoinParams q, int rows, Chain& s) {
  const dim3 grid(static_cast<unsigned>(q.tiles_i * q.tiles_j * rows * q.bn / 4 / 256), q.groups);
  return s.launch(rows == 128 ? join_kernel<T, 128> : join_kernel<T, 256>, grid, 256, 0, q);
}

}  // namespace

int join_parts(const JoinParams& q, int rows, int dtype, Chain& s) {
  if (dtype == PIC_DTYPE_F32) return join<float>(q, rows, s);
  if (dtype == PIC_DTYPE_F16) return join<__half>(q, rows, s);
  return join<__nv_bfloat16>(q, rows, s);
}

bool tc_takes(const GroupProduct& p, int dtype) {
  if (dtype == PIC_DTYPE_F32) return false;
  return p.by_rows ? p.K <= kTcMostK : p.rows > 0;
}

long long tc_workspace(const GroupProduct& p, int) {
  const Plan r = plan(p);
  return r.a.bytes + r.b.bytes + r.map_bytes + r.part_bytes;
}

int tc_product(const GroupProduct& p, int dtype, void* ws, const Waits& waits, Chain& s) {
  const Plan r = plan(p);
  char* w = static_cast<char*>(ws);
  Operand a = r.a, b = r.b;
  if (a.pad) {
    if (pad(a, p.a_i, 0, w, s) != PIC_OK) return PIC_ERR_CUDA;
    a.m = w;
  }
  if (b.pad) {
    if (pad(b, p.by_rows && p.b_k == 1 ? p.b_j : p.b_k, p.b_group, w + a.bytes, s) != PIC_OK) return PIC_ERR_CUDA;
    b.m = w + a.bytes;
  }
  GtParams q{};
  GtMaps maps{};
  q.rows = p.rows, q.I = p.I, q.J = p.J, q.K = p.K;
  q.tiles_i = r.tiles_i, q.tiles_j = r.tiles_j;
  q.groups = p.groups, q.offsets = p.offsets;
  q.b_mn = p.by_rows && p.b_k != 1;
  q.chunk = r.chunk;
  q.maps = reinterpret_cast<CUtensorMap*>(w + a.bytes + b.bytes);
  q.parts = reinterpret_cast<float*>(w + a.bytes + b.bytes + r.map_bytes);
  q.bias = p.bias, q.bias_group = p.bias_group;
  q.y = p.y, q.ldy = p.ldy, q.y_group = p.y_group, q.pre = p.pre, q.ldpre = p.ldpre, q.act = p.act;
  q.waits = waits;
  const auto fits = [&](const void* m, long long ld) {
    return reinterpret_cast<uintptr_t>(m) % 16 == 0 && ld % 8 == 0 && ld * 2 < (1LL << 40);
  };
  bool ok;
  if (p.by_rows) {
    if (r.mode == kTurned) {
      ok = lin::encode_many(&maps.a, b.m, b.rows, b.cols, b.ld, b.count, b.group, q.b_mn ? 64 : 128, dtype) &&
           lin::encode(&maps.b, a.m, a.rows, a.cols, a.ld, r.bn, dtype);
    } else {
      ok = lin::encode(&maps.a, a.m, a.rows, a.cols, a.ld, 128, dtype) &&
           lin::encode_many(&maps.b, b.m, b.rows, b.cols, b.ld, b.count, b.group, q.b_mn ? 64 : r.bn / r.cg, dtype);
      // a TMA store ends on a 16-byte boundary of the row
      q.store_tma = p.J % 8 == 0 && fits(p.y, p.ldy) && (!p.pre || fits(p.pre, p.ldpre));
      if (q.store_tma) ok = ok && lin::encode(&maps.y, p.y, p.rows, p.J, p.ldy, 32, dtype);
      if (q.store_tma && p.pre) ok = ok && lin::encode(&maps.pre, p.pre, p.rows, p.J, p.ldpre, 32, dtype);
    }
  } else {
    ok = lin::encode(&maps.a, a.m, a.rows, a.cols, a.ld, 64, dtype) && lin::encode(&maps.b, b.m, b.rows, b.cols, b.ld, 64, dtype);
    q.store_tma = p.J % 8 == 0 && fits(p.y, p.ldy) && (p.groups == 1 || fits(p.y, p.y_group));
    if (q.store_tma)
      ok = ok && lin::encode_many(&maps.y, p.y, p.I, p.J, p.ldy, p.groups, p.groups == 1 ? p.I * p.ldy : p.y_group, 32, dtype);
  }
  if (!ok) return PIC_ERR_CUDA;
  if (!p.by_rows && p.rows > 0) {
    const MakeMaps mk{p.offsets, p.rows, const_cast<CUtensorMap*>(q.maps)};
    if (s.launch(maps_kernel, dim3(p.groups), 32, 0, mk, maps) != PIC_OK) return PIC_ERR_CUDA;
  }
  const GtKernel k = dtype == PIC_DTYPE_BF16 ? group_kernel_bf16(r.mode, r.bn) : group_kernel_f16(r.mode, r.bn);
  if (lin::allow_smem(k.fn, k.slot, k.smem) != PIC_OK) return PIC_ERR_CUDA;
  const long long slots = static_cast<long long>(kSms) * k.ctas, want = r.work * r.cg;
  void* args[] = {&q, &maps};
  if (s.launch(k.fn, dim3(static_cast<unsigned>(want < slots ? want : slots)), k.threads, k.smem, r.cg, args) != PIC_OK) return PIC_ERR_CUDA;
  if (!p.by_rows && r.part_bytes > 0) {
    const JoinParams j{p.offsets, p.rows, p.I, p.J, r.tiles_i, r.tiles_j, p.groups, r.chunk, r.bn,
                       reinterpret_cast<const float4*>(q.parts), p.y, p.ldy, p.y_group, waits.status};
    return join_parts(j, 128 * r.cg, dtype, s);
  }
  return PIC_OK;
}

}  // namespace grp
}  // namespace pic
