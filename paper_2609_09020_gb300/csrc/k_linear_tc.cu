// k_linear_tc.cu -- host side of the linear layer's tensor-core products: tile
// shapes, cuts along K, tensor maps; and the two small kernels around them,
// which lay out matrices that TMA cannot read and join parts.
#include <atomic>

#include <cuda.h>
#include <cudaTypedefs.h>

#include "k_linear_planes.cuh"
#include "k_linear_reg.cuh"

namespace pic {
namespace lin {
namespace {

constexpr int kSms = 152;

// Up to two matrices whose rows start on 16-byte boundaries, from ones whose do
// not: a thread puts eight elements together from the aligned words that hold
// them, of four rows at a time.  Bound by memory: it reads and writes each element
// once.
struct Repack {
  const uint16_t* src[2];
  uint4* dst[2];
  long long ld[2], rows[2];
  int cols[2], ld_out[2];  // ld_out: chunks of eight elements from row to row
  int tx[2];               // threads along a row, a power of two
  unsigned blocks0;        // blocks that work on the first matrix
};
constexpr int kRepackRows = 4;

__global__ void __launch_bounds__(256) repack_kernel(const Repack q) {
  const int m = blockIdx.x < q.blocks0 ? 0 : 1;
  const unsigned block = m ? blockIdx.x - q.blocks0 : blockIdx.x, blocks = m ? gridDim.x - q.blocks0 : q.blocks0;
  const long long ld = q.ld[m], rows = q.rows[m];
  const int cols = q.cols[m], chunks = (cols + 7) / 8, tx = q.tx[m], ty = 256 / tx;
  const int x = threadIdx.x & (tx - 1), y = threadIdx.x / tx;
  for (long long r0 = static_cast<long long>(block) * ty * kRepackRows; r0 < rows;
       r0 += static_cast<long long>(blocks) * ty * kRepackRows)
    for (int chunk = x; chunk < chunks; chunk += tx) {
      const int c = chunk * 8;
      uint32_t h[kRepackRows][5];
      bool odd[kRepackRows];
#pragma unroll
      for (int u = 0; u < kRepackRows; ++u) {
        const long long r = r0 + u * ty + y;
        const uint16_t* p = q.src[m] + r * ld + c;
        odd[u] = (reinterpret_cast<uintptr_t>(p) & 2) != 0;
        // the words' last half belongs to the element after the eight
        const bool words = r < rows && c + 8 + (odd[u] && r + 1 == rows ? 1 : 0) <= cols;
        if (words || r >= rows) {
          const uint32_t* v = reinterpret_cast<const uint32_t*>(p - (odd[u] ? 1 : 0));
#pragma unroll
          for (int i = 0; i < 4; ++i) h[u][i] = load_if(v + i, words);
          h[u][4] = load_if(v + 4, words && odd[u]);
        } else {
          odd[u] = false;
          uint32_t e[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) e[i] = load_if(p + i, c + i < cols);
#pragma unroll
          for (int i = 0; i < 4; ++i) h[u][i] = e[2 * i] | e[2 * i + 1] << 16;
          h[u][4] = 0;
        }
      }
#pragma unroll
      for (int u = 0; u < kRepackRows; ++u) {
        const long long r = r0 + u * ty + y;
        if (r >= rows) continue;
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = odd[u] ? __funnelshift_r(h[u][i], h[u][i + 1], 16) : h[u][i];
        q.dst[m][r * q.ld_out[m] + chunk] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
}

struct JoinParams {
  Product p;
  const float4* parts;
  long long tiles_i, tiles_j;
  int splits, rows, bn;  // rows and columns of a tile
};

// A thread finishes an item (four columns of a row), where there are few parts.
template <typename T, int ROWS>
__global__ void __launch_bounds__(256) join_few_kernel(const JoinParams q) {
  const int per_tile = ROWS * q.bn / 4;
  const long long tile = blockIdx.x / (per_tile / 256);
  long long ti, tj;
  tile_place<ROWS>(tile, q.tiles_i, q.tiles_j, ti, tj);
  const JoinItem m = join_place<ROWS>(static_cast<int>(blockIdx.x % (per_tile / 256)) * 256 + threadIdx.x, q.bn, ti, tj);
  if (m.i >= q.p.I || m.j >= q.p.J) return;
  const float4* parts = q.parts + tile * q.splits * per_tile + m.at;
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
  for (int s = 0; s < q.splits; ++s) {
    const float4 f = __ldcg(parts + static_cast<long long>(s) * per_tile);
    v.x += f.x, v.y += f.y, v.z += f.z, v.w += f.w;
  }
  finish_item<T>(q.p, m, v);
}

// A block finishes 32 items, where there are many parts: its warps add every
// eighth, then the first warp the warps' sums.
template <typename T, int ROWS>
__global__ void __launch_bounds__(256) join_kernel(const JoinParams q) {
  __shared__ float4 sums[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int per_tile = ROWS * q.bn / 4;
  const long long tile = blockIdx.x / (per_tile / 32);
  long long ti, tj;
  tile_place<ROWS>(tile, q.tiles_i, q.tiles_j, ti, tj);
  const JoinItem m = join_place<ROWS>(static_cast<int>(blockIdx.x % (per_tile / 32)) * 32 + lane, q.bn, ti, tj);
  const bool inside = m.i < q.p.I && m.j < q.p.J;
  const float4* parts = q.parts + tile * q.splits * per_tile + m.at;
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (inside) {
#pragma unroll 4
    for (int s = warp; s < q.splits; s += 8) {
      const float4 f = __ldcg(parts + static_cast<long long>(s) * per_tile);
      v.x += f.x, v.y += f.y, v.z += f.z, v.w += f.w;
    }
  }
  sums[warp][lane] = v;
  __syncthreads();
  if (warp > 0 || !inside) return;
#pragma unroll
  for (int w = 1; w < 8; ++w) {
    const float4 f = sums[w][lane];
    v.x += f.x, v.y += f.y, v.z += f.z, v.w += f.w;
  }
  finish_item<T>(q.p, m, v);
}

struct Operand {
  long long rows, cols, ld;  // as stored: cols contiguous
  bool mn, repack;
  long long ld_packed;
};

Operand operand(const void* m, long long s_row, long long s_k, long long rows, long long K, bool fp32) {
  Operand o{};
  o.mn = s_k != 1;
  o.rows = o.mn ? K : rows;
  o.cols = o.mn ? rows : K;
  o.ld = o.mn ? s_k : s_row;
  o.ld_packed = (o.cols + 63) / 64 * 64;  // rows on 128-byte lines
  if (o.rows == 1) o.ld = o.ld_packed;  // not used
  if (fp32) return o;
  o.repack = reinterpret_cast<uintptr_t>(m) % 16 != 0 || o.ld % 8 != 0 || o.ld * 2 >= (1LL << 40);
  return o;
}

struct Plan {
  Operand a, b;
  bool reg;     // fp32 operands through registers
  bool planes;  // fp32 operands cut into planes first
  int cg, bn;
  long long tiles_i, tiles_j;
  int k_blocks, part_blocks, splits;
  long long a_bytes, b_bytes, part_bytes, carry_bytes;
};

long long round256(long long v) { return (v + 255) / 256 * 256; }

long long planes_bytes(const Operand& o) { return round256(3 * o.rows * o.ld_packed * 2); }
long long mark_cols(const Operand& o) { return (o.cols + kPlBlock - 1) / kPlBlock; }
long long marks_bytes(const Operand& o) { return round256((o.rows + kPlBlock - 1) / kPlBlock * mark_cols(o) * 4); }

// What a tile shape costs, in microseconds, as measured on products of 64..4096
// rows, K of 256..16384 and 256..4096 columns (bf16; fp32 for the last two).
struct ShapeCost {
  int bn, cg;
  int slots;         // CTAs or pairs that run at once
  double fixed;      // launch, first loads, last epilogue
  double slice;      // 64 of K of a tile
  double tile;       // a tile's epilogue, which the next one's slices hide
};
constexpr ShapeCost kShape64{64, 1, 2 * kSms, 4.2, 0.20, 3.0};
constexpr ShapeCost kShape128{128, 1, kSms, 4.5, 0.19, 2.2};
constexpr ShapeCost kShape256{256, 2, kSms / 2, 6.8, 0.26, 3.4};
constexpr ShapeCost kShapeReg{kRegCols, 1, kSms, 6.0, 1.7, 4.0};
constexpr ShapeCost kShapePlanes{kPlCols, 2, kSms / 2, 8.0, 0.95, 3.4};

// The shape and the number of parts of K with the least estimated time, parts at
// least `least` slices long: rounds of tiles, and for parts the second kernel, which
// costs 2 us and their fp32 traffic at 2.6 TB/s.  For instance, in us (measured):
// 1024 x 1024 -> 1024 128/1 7.6 (7.7), 1024 x 4096 -> 1024 128/1 16.7 (16.5) and
// 128/4 19.0 (19.0), 512 x 16384 -> 512 128/8 15.8 (15.2), 64/8 (20), 256/8 (19.3).
// Rows that are not whole 128-byte lines make slices of 64 and 128 columns half as
// slow again (720 x 12632 -> 496 128/4 25.9 (25.7), 256/8 21.9 (21.2)).
// The estimate is returned.
double choose(Plan& r, const Product& p, const ShapeCost* shapes, int n_shapes, int least, bool lines) {
  double best = 1e30;
  for (int c = 0; c < n_shapes; ++c) {
    const ShapeCost& h = shapes[c];
    const int rows = 128 * h.cg;
    const long long ti = (p.I + rows - 1) / rows, tj = (p.J + h.bn - 1) / h.bn, tiles = ti * tj;
    double slice = h.slice;
    if (!lines) slice *= h.bn == 256 ? 1.25 : 1.75;
    for (int want = 1; want <= 2 * kSms; want = want < 8 ? want + 1 : want + want / 8) {
      if (want > 1 && (tiles * want > h.slots || r.k_blocks / want < least)) break;
      const int part = (r.k_blocks + want - 1) / want;
      const int splits = (r.k_blocks + part - 1) / part;
      const long long work = tiles * splits, rounds = (work + h.slots - 1) / h.slots;
      const bool shared = h.slots > kSms && work > kSms;  // two CTAs on an SM
      const double each = part * slice * (shared ? 1.5 : 1.0);
      double t = h.fixed + (rounds > 1 && each < h.tile ? rounds * h.tile : rounds * each);
      if (splits > 1) t += 2.0 + 4.0 * rows * h.bn * static_cast<double>(work) / 2.6e6;
      if (t < best) {
        best = t;
        r.bn = h.bn, r.cg = h.cg, r.tiles_i = ti, r.tiles_j = tj;
        r.part_blocks = part, r.splits = splits;
      }
    }
  }
  return best;
}

// fp32: operands cut into planes first, or on the way, again for every tile.  The
// first costs 4 us and 10 bytes of traffic an element at 5 TB/s; the second takes
// longer for rows off 16-byte boundaries.  us, planes / on the way: 200 x 4096 -> 8192
// 137 / 229, 4000 x 2686 -> 221 58 / 87, 200 x 500 -> 8192 25 / 46; 100 x 4096 -> 2048 45
// / 34, 500 x 500 -> 150 20 / 14, 16000 x 512 -> 16 32 / 18.
void choose_fp32(Plan& r, const Product& p, bool rows16) {
  Plan other = r;
  ShapeCost reg = kShapeReg;
  if (!rows16) reg.slice *= 1.15;
  const double on_the_way = choose(r, p, &reg, 1, 4, true);
  r.reg = true;
  if (p.swapped) return;
  const double elements = static_cast<double>(p.K) * static_cast<double>(p.I + p.J);
  const double first = choose(other, p, &kShapePlanes, 1, 4, true) + 4.0 + elements * 10.0 / 5e6;
  if (first < on_the_way) {
    r = other;
    r.planes = true;
  }
  r.reg = !r.planes;
}

// fp32 with no more rows than the smaller side of a tile through registers: w takes the
// larger one where fewer tiles are less time, which is where there are many (us, 12 x
// 4096 -> 8192 70 instead of 105, 48 x 2048 -> 8192 35 instead of 51).  Columns of y a
// row apart cost a little: 33 x 2048 -> 512 14.8 instead of 13.5.
Product oriented(const Product& p, int dtype) {
  if (dtype != PIC_DTYPE_F32 || p.I > kRegCols || p.J <= kRegRows) return p;
  Product q = p;
  q.a = p.b, q.a_i = p.b_j, q.a_k = p.b_k, q.I = p.J;
  q.b = p.a, q.b_j = p.a_i, q.b_k = p.a_k, q.J = p.I;
  q.swapped = 1;
  Plan r{};
  r.k_blocks = static_cast<int>((p.K + kSlice - 1) / kSlice);
  return choose(r, q, &kShapeReg, 1, 4, true) + 1.5 < choose(r, p, &kShapeReg, 1, 4, true) ? q : p;
}

// CTAs of a launch: persistent, two on an SM for tiles of 64 columns of 16-bit types.
long long ctas(const Plan& r) {
  const long long want = r.tiles_i * r.tiles_j * r.splits * r.cg, most = r.bn == 64 && !r.reg ? 2 * kSms : kSms;
  return want < most ? want : most;
}

Plan plan(const Product& p, int dtype) {
  Plan r{};
  const bool fp32 = dtype == PIC_DTYPE_F32;
  r.a = operand(p.a, p.a_i, p.a_k, p.I, p.K, fp32);
  r.b = operand(p.b, p.b_j, p.b_k, p.J, p.K, fp32);
  r.k_blocks = static_cast<int>((p.K + kSlice - 1) / kSlice);
  if (fp32) {
    const auto rows16 = [](const void* m, const Operand& o) { return reinterpret_cast<uintptr_t>(m) % 16 == 0 && o.ld % 4 == 0; };
    choose_fp32(r, p, rows16(p.a, r.a) && rows16(p.b, r.b));
  } else {
    const ShapeCost shapes[] = {kShape64, kShape128, kShape256};
    const auto lines = [](const Operand& o) { return o.repack || o.ld % 64 == 0; };
    choose(r, p, shapes, 3, 4, lines(r.a) && lines(r.b));
  }
  const int rows = 128 * r.cg;
  if (r.a.repack) r.a_bytes = round256(r.a.rows * r.a.ld_packed * 2);
  if (r.b.repack) r.b_bytes = round256(r.b.rows * r.b.ld_packed * 2);
  if (r.planes) {
    r.a_bytes = planes_bytes(r.a) + marks_bytes(r.a);
    r.b_bytes = planes_bytes(r.b) + marks_bytes(r.b);
  }
  if (r.splits > 1) r.part_bytes = r.tiles_i * r.tiles_j * r.splits * rows * r.bn * 4;
  if (!fp32 && r.part_blocks > kTcTakeover) r.carry_bytes = ctas(r) * 128 * r.bn * 4;
  return r;
}

PFN_cuTensorMapEncodeTiled_v12000 encoder() {
  static const PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q = cudaDriverEntryPointSymbolNotFound;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      f = nullptr;
    }
    return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
  }();
  return fn;
}

// The three planes of a matrix, in boxes of box_cols columns (64, 128-byte swizzled,
// or 32, 64-byte swizzled), box_rows rows and all planes.
bool encode_planes(CUtensorMap* map, const void* m, long long rows, long long cols, long long ld, int box_cols, int box_rows) {
  const PFN_cuTensorMapEncodeTiled_v12000 enc = encoder();
  if (!enc) return false;
  const cuuint64_t dim[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows), 3};
  const cuuint64_t stride[2] = {static_cast<cuuint64_t>(ld * 2), static_cast<cuuint64_t>(rows * ld * 2)};
  const cuuint32_t box[3] = {static_cast<cuuint32_t>(box_cols), static_cast<cuuint32_t>(box_rows), 3};
  const cuuint32_t elem[3] = {1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(m), dim, stride, box, elem,
             CU_TENSOR_MAP_INTERLEAVE_NONE, box_cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The operands where TMA can read them: as they are, or laid out in the workspace.
void lay_out(const Product& p, const Plan& r, char* w, const void** a, const void** b, cudaStream_t s) {
  Repack q{};
  unsigned blocks[2] = {0, 0};
  int n = 0;
  const auto add = [&](const void* m, const Operand& o, char* at) {
    if (!o.repack) return m;
    q.src[n] = static_cast<const uint16_t*>(m);
    q.dst[n] = reinterpret_cast<uint4*>(at);
    q.ld[n] = o.ld, q.rows[n] = o.rows;
    q.cols[n] = static_cast<int>(o.cols);
    q.ld_out[n] = static_cast<int>(o.ld_packed / 8);
    q.tx[n] = 1;
    while (q.tx[n] < (o.cols + 7) / 8 && q.tx[n] < 256) q.tx[n] *= 2;
    const long long per_block = 256 / q.tx[n] * kRepackRows, want = (o.rows + per_block - 1) / per_block;
    blocks[n++] = static_cast<unsigned>(want < 16 * kSms ? want : 16 * kSms);
    return static_cast<const void*>(at);
  };
  *a = add(p.a, r.a, w);
  *b = add(p.b, r.b, w + r.a_bytes);
  q.blocks0 = blocks[0];
  if (n > 0) repack_kernel<<<blocks[0] + blocks[1], 256, 0, s>>>(q);
}

template <typename T>
int join(const JoinParams& q, cudaStream_t s) {
  const long long items = q.tiles_i * q.tiles_j * q.rows * q.bn / 4;
  if (q.splits <= 16) {
    const unsigned blocks = static_cast<unsigned>(items / 256);
    if (q.rows == 128)
      join_few_kernel<T, 128><<<blocks, 256, 0, s>>>(q);
    else
      join_few_kernel<T, 256><<<blocks, 256, 0, s>>>(q);
  } else {
    const unsigned blocks = static_cast<unsigned>(items / 32);
    if (q.rows == 128)
      join_kernel<T, 128><<<blocks, 256, 0, s>>>(q);
    else
      join_kernel<T, 256><<<blocks, 256, 0, s>>>(q);
  }
  return cudaGetLastError() == cudaSuccess ? PIC_OK : PIC_ERR_CUDA;
}

}  // namespace

bool encode(CUtensorMap* map, const void* m, long long rows, long long cols, long long ld, int box_rows, int dtype) {
  const PFN_cuTensorMapEncodeTiled_v12000 enc = encoder();
  if (!enc) return false;
  const unsigned e = dtype == PIC_DTYPE_F32 ? 4 : 2;
  const CUtensorMapDataType type = dtype == PIC_DTYPE_F32   ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : dtype == PIC_DTYPE_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                            : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  const cuuint64_t dim[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
  const cuuint64_t stride[1] = {static_cast<cuuint64_t>(ld * e)};
  const cuuint32_t box[2] = {128u / e, static_cast<cuuint32_t>(box_rows)};
  const cuuint32_t elem[2] = {1, 1};
  return enc(map, type, 2, const_cast<void*>(m), dim, stride, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int allow_smem(const void* fn, int slot, int smem) {
  static std::atomic<uint64_t> done[kSmemSlots];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return PIC_ERR_CUDA;
  const uint64_t bit = 1ull << (dev & 63);
  if (done[slot].load(std::memory_order_acquire) & bit) return PIC_OK;
  if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return PIC_ERR_CUDA;
  done[slot].fetch_or(bit, std::memory_order_release);
  return PIC_OK;
}

long long tc_workspace(const Product& p, int dtype) {
  const Plan r = plan(oriented(p, dtype), dtype);
  return r.a_bytes + r.b_bytes + r.part_bytes + r.carry_bytes;
}

int tc_product(const Product& given, int dtype, void* ws, const Waits& waits, cudaStream_t s) {
  const Product p = oriented(given, dtype);
  const Plan r = plan(p, dtype);
  const long long elem = dtype == PIC_DTYPE_F32 ? 4 : 2;
  char* w = static_cast<char*>(ws);
  const void *a, *b;
  lay_out(p, r, w, &a, &b, s);

  TcParams q{};
  TcMaps maps;
  RegOperands o{};
  PlOperands pl{};
  q.p = p;
  q.tiles_i = r.tiles_i, q.tiles_j = r.tiles_j;
  q.splits = r.splits, q.k_blocks = r.k_blocks, q.part_blocks = r.part_blocks;
  q.work = r.tiles_i * r.tiles_j * r.splits;
  q.a_mn = r.a.mn, q.b_mn = r.b.mn;
  q.parts = r.splits > 1 ? reinterpret_cast<float*>(w + r.a_bytes + r.b_bytes) : nullptr;
  q.carry = r.carry_bytes ? reinterpret_cast<float*>(w + r.a_bytes + r.b_bytes + r.part_bytes) : nullptr;
  q.waits = waits;
  const auto fits = [&](const void* m, long long ld, long long rows) {
    return reinterpret_cast<uintptr_t>(m) % 16 == 0 && ((ld * elem % 16 == 0 && ld * elem < (1LL << 40)) || rows == 1);
  };
  // a TMA store ends on a 16-byte boundary of the row: columns that do not would
  // have their neighbours overwritten
  q.store_tma = !q.parts && elem == 2 && p.J * elem % 16 == 0 && fits(p.y, p.ldy, p.I) && (!p.pre || fits(p.pre, p.ldpre, p.I));
  const auto out_ld = [&](long long ld) { return p.I == 1 ? (p.J + 7) / 8 * 8 : ld; };
  bool ok = true;
  if (r.reg) {
    o.a = p.a, o.b = p.b;
    o.lda = r.a.ld, o.ldb = r.b.ld;
    const auto vec = [&](const void* m, const Operand& x) {
      return reinterpret_cast<uintptr_t>(m) % (4 * elem) == 0 && (x.ld % 4 == 0 || x.rows == 1);
    };
    o.vec_a = vec(p.a, r.a), o.vec_b = vec(p.b, r.b);
  } else if (r.planes) {
    CutMatrix m[2];
    const auto add = [&](CutMatrix& c, const void* from, const Operand& x, char* at, PlOperand& out, CUtensorMap* map, int tile) {
      c = {static_cast<const float*>(from), x.ld, x.rows, x.cols, at, x.ld_packed, reinterpret_cast<int*>(at + planes_bytes(x))};
      out = {c.m, x.ld, c.marks, static_cast<int>(mark_cols(x))};
      // 32 of K: along K a box of the CTA's rows, else blocks of 64 rows
      return x.mn ? encode_planes(map, at, x.rows, x.cols, x.ld_packed, 64, 32)
                  : encode_planes(map, at, x.rows, x.cols, x.ld_packed, 32, tile);
    };
    ok = add(m[0], p.a, r.a, w, pl.a, &maps.a, 128) &&
         add(m[1], p.b, r.b, w + r.a_bytes, pl.b, &maps.b, 64) && cut_planes(m, s) == PIC_OK;
  } else {
    // of an operand that lies along its rows a box is 64 of them by 64 of K
    ok = encode(&maps.a, a, r.a.rows, r.a.cols, r.a.repack ? r.a.ld_packed : r.a.ld, r.a.mn ? 64 : 128, dtype) &&
         encode(&maps.b, b, r.b.rows, r.b.cols, r.b.repack ? r.b.ld_packed : r.b.ld, r.b.mn ? 64 : r.bn / r.cg, dtype);
  }
  if (q.store_tma) ok = ok && encode(&maps.y, p.y, p.I, p.J, out_ld(p.ldy), 32, dtype);
  if (q.store_tma && p.pre) ok = ok && encode(&maps.pre, p.pre, p.I, p.J, out_ld(p.ldpre), 32, dtype);
  if (!ok) return PIC_ERR_CUDA;

  const void* fn;
  int slot, smem, threads;
  if (r.reg) {
    const RegKernel k = reg_kernel_info();
    fn = k.fn, threads = k.threads, smem = k.smem;
    slot = 6;
  } else if (r.planes) {
    const PlKernel k = planes_kernel_info();
    fn = k.fn, threads = k.threads, smem = k.smem;
    slot = 7;
  } else {
    const bool long_parts = r.carry_bytes > 0;
    fn = dtype == PIC_DTYPE_BF16 ? tc_kernel_bf16(r.bn, long_parts) : tc_kernel_f16(r.bn, long_parts);
    const int shape = r.bn == 256 ? 2 : r.bn == 128 ? 1 : 0;
    slot = shape + (dtype == PIC_DTYPE_BF16 ? 3 : 0) + (long_parts ? 20 : 0);
    smem = shape == 2 ? TcShape<2, 256>::kSmem : shape == 1 ? TcShape<1, 128>::kSmem : TcShape<1, 64>::kSmem;
    threads = shape == 2 ? TcShape<2, 256>::kThreads : shape == 1 ? TcShape<1, 128>::kThreads : TcShape<1, 64>::kThreads;
  }
  if (allow_smem(fn, slot, smem) != PIC_OK) return PIC_ERR_CUDA;
  void* args[] = {&q, &maps, r.planes ? static_cast<void*>(&pl) : &o};  // 16-bit kernels take the first two
  if (launch_kernel(fn, ctas(r), threads, smem, r.cg, args, s) != PIC_OK) return PIC_ERR_CUDA;
  if (q.parts) {
    const JoinParams j{p, reinterpret_cast<const float4*>(q.parts), r.tiles_i, r.tiles_j, r.splits, 128 * r.cg, r.bn};
    if (dtype == PIC_DTYPE_F32) return join<float>(j, s);
    return dtype == PIC_DTYPE_BF16 ? join<__nv_bfloat16>(j, s) : join<__half>(j, s);
  }
  return PIC_OK;
}

}  // namespace lin
}  // namespace pic
