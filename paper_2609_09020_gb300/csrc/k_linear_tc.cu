// k_linear_tc.cu -- host side of the linear layer's tensor-core products: tile
// shapes, cuts along K, tensor maps; and the two small kernels around them,
// which lay out matrices that TMA cannot read and join parts.
#include <atomic>

#include <cuda.h>
#include <cudaTypedefs.h>

#include "k_linear_tc.cuh"

namespace pic {
namespace lin {
namespace {

constexpr int kSms = 152;

// A matrix whose rows start on 16-byte boundaries, from one whose do not.
__global__ void __launch_bounds__(256) repack_kernel(const uint16_t* src, long long ld, long long rows, int cols,
                                                     uint16_t* dst, int ld_out) {
  const long long n = rows * ld_out;
  for (long long e = blockIdx.x * 256LL + threadIdx.x; e < n; e += gridDim.x * 256LL) {
    const long long r = e / ld_out;
    const int c = static_cast<int>(e % ld_out);
    if (c < cols) dst[e] = src[r * ld + c];
  }
}

struct JoinParams {
  Product p;
  const float4* parts;
  long long tiles_i, tiles_j;
  int splits, rows, bn;  // rows and columns of a tile
};

// A thread adds the parts of four columns of a row, in order, and runs the epilogue.
template <typename T, int ROWS>
__global__ void __launch_bounds__(256) join_kernel(const JoinParams q) {
  const Product& p = q.p;
  const long long per_tile = static_cast<long long>(ROWS) * q.bn / 4;
  const long long n = q.tiles_i * q.tiles_j * per_tile;
  for (long long e = blockIdx.x * 256LL + threadIdx.x; e < n; e += gridDim.x * 256LL) {
    const long long tile = e / per_tile;
    const int in = static_cast<int>(e % per_tile);
    // [rank][panel][quarter][16][32 lanes]
    const int lane = in & 31, c4 = in >> 5 & 15, quarter = in >> 9 & 3, rest = in >> 11;
    const int panel = rest % (q.bn / 64), rank = rest / (q.bn / 64);
    long long ti, tj;
    tile_place<ROWS>(tile, q.tiles_i, q.tiles_j, ti, tj);
    const long long i = ti * ROWS + rank * 128 + quarter * 32 + lane, j = tj * q.bn + panel * 64 + c4 * 4;
    if (i >= p.I || j >= p.J) continue;
    float v[4] = {};
    for (int s = 0; s < q.splits; ++s) {
      const float4 f = q.parts[(tile * q.splits + s) * per_tile + in];
      v[0] += f.x, v[1] += f.y, v[2] += f.z, v[3] += f.w;
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      if (j + c >= p.J) break;
      float z = v[c];
      if (p.bias) z += to_f32(static_cast<const T*>(p.bias)[j + c]);
      if (p.pre) static_cast<T*>(p.pre)[i * p.ldpre + j + c] = from_f32<T>(z);
      z = act_value<false>(z, p.act);
      if (p.residual) z += to_f32(static_cast<const T*>(p.residual)[i * p.ldr + j + c]);
      static_cast<T*>(p.y)[i * p.ldy + j + c] = from_f32<T>(z);
    }
  }
}

struct Operand {
  long long rows, cols, ld;  // as stored: cols contiguous
  bool mn, repack;
  long long ld_packed;
};

Operand operand(const void* m, long long s_row, long long s_k, long long rows, long long K) {
  Operand o;
  o.mn = s_k != 1;
  o.rows = o.mn ? K : rows;
  o.cols = o.mn ? rows : K;
  o.ld = o.mn ? s_k : s_row;
  o.ld_packed = (o.cols + 7) / 8 * 8;
  if (o.rows == 1) o.ld = o.ld_packed;  // not used
  o.repack = reinterpret_cast<uintptr_t>(m) % 16 != 0 || o.ld % 8 != 0 || o.ld * 2 >= (1LL << 40);
  return o;
}

struct Plan {
  Operand a, b;
  int cg, bn;
  long long tiles_i, tiles_j;
  int k_blocks, part_blocks, splits;
  long long a_bytes, b_bytes, part_bytes;
};

long long round256(long long v) { return (v + 255) / 256 * 256; }

Plan plan(const Product& p) {
  Plan r{};
  r.a = operand(p.a, p.a_i, p.a_k, p.I, p.K);
  r.b = operand(p.b, p.b_j, p.b_k, p.J, p.K);
  const long long big = ((p.I + 255) / 256) * ((p.J + 255) / 256);
  r.bn = p.J <= 64 ? 64 : p.J <= 128 || big < kSms / 2 ? 128 : 256;
  r.cg = r.bn == 256 ? 2 : 1;
  const int rows = 128 * r.cg;
  r.tiles_i = (p.I + rows - 1) / rows;
  r.tiles_j = (p.J + r.bn - 1) / r.bn;
  r.k_blocks = static_cast<int>((p.K + kSlice - 1) / kSlice);
  const int splits = split_count(r.tiles_i * r.tiles_j, r.k_blocks, 4, kSms);
  r.part_blocks = (r.k_blocks + splits - 1) / splits;
  r.splits = (r.k_blocks + r.part_blocks - 1) / r.part_blocks;
  if (r.a.repack) r.a_bytes = round256(r.a.rows * r.a.ld_packed * 2);
  if (r.b.repack) r.b_bytes = round256(r.b.rows * r.b.ld_packed * 2);
  if (r.splits > 1) r.part_bytes = r.tiles_i * r.tiles_j * r.splits * rows * r.bn * 4;
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

// A [rows][cols] matrix of 16-bit values in boxes of 64 columns and box_rows
// rows, 128-byte swizzled.
bool encode(CUtensorMap* map, const void* m, long long rows, long long cols, long long ld, int box_rows, bool bf16) {
  const PFN_cuTensorMapEncodeTiled_v12000 enc = encoder();
  if (!enc) return false;
  const cuuint64_t dim[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
  const cuuint64_t stride[1] = {static_cast<cuuint64_t>(ld * 2)};
  const cuuint32_t box[2] = {64, static_cast<cuuint32_t>(box_rows)};
  const cuuint32_t elem[2] = {1, 1};
  return enc(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void*>(m), dim,
             stride, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

const void* repacked(const void* m, const Operand& o, void* ws, cudaStream_t s) {
  if (!o.repack) return m;
  long long b = (o.rows * o.ld_packed + 1023) / 1024;
  if (b > 16 * kSms) b = 16 * kSms;
  repack_kernel<<<static_cast<unsigned>(b), 256, 0, s>>>(static_cast<const uint16_t*>(m), o.ld, o.rows,
                                                         static_cast<int>(o.cols), static_cast<uint16_t*>(ws),
                                                         static_cast<int>(o.ld_packed));
  return ws;
}

template <int CG, int BN>
int smem_of() {
  return TcShape<CG, BN>::kSmem;
}

// The kernel's shared-memory attribute, set once per device.
int set_up(const void* fn, int slot, int smem) {
  static std::atomic<uint64_t> done[6];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return PIC_ERR_CUDA;
  const uint64_t bit = 1ull << (dev & 63);
  if (done[slot].load(std::memory_order_acquire) & bit) return PIC_OK;
  if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return PIC_ERR_CUDA;
  done[slot].fetch_or(bit, std::memory_order_release);
  return PIC_OK;
}

template <typename T>
int join(const JoinParams& q, cudaStream_t s) {
  long long b = (q.tiles_i * q.tiles_j * q.rows * q.bn / 4 + 255) / 256;
  if (b > 16 * kSms) b = 16 * kSms;
  if (q.rows == 128)
    join_kernel<T, 128><<<static_cast<unsigned>(b), 256, 0, s>>>(q);
  else
    join_kernel<T, 256><<<static_cast<unsigned>(b), 256, 0, s>>>(q);
  return cudaGetLastError() == cudaSuccess ? PIC_OK : PIC_ERR_CUDA;
}

}  // namespace

long long tc_workspace(const Product& p) {
  const Plan r = plan(p);
  return r.a_bytes + r.b_bytes + r.part_bytes;
}

int tc_product(const Product& p, int dtype, void* ws, int* status, unsigned spin_limit, cudaStream_t s) {
  const Plan r = plan(p);
  const bool bf16 = dtype == PIC_DTYPE_BF16;
  char* w = static_cast<char*>(ws);
  const void* a = repacked(p.a, r.a, w, s);
  const void* b = repacked(p.b, r.b, w + r.a_bytes, s);
  float* parts = r.splits > 1 ? reinterpret_cast<float*>(w + r.a_bytes + r.b_bytes) : nullptr;

  TcParams q{};
  TcMaps maps;
  q.p = p;
  q.tiles_i = r.tiles_i, q.tiles_j = r.tiles_j;
  q.splits = r.splits, q.k_blocks = r.k_blocks, q.part_blocks = r.part_blocks;
  q.work = r.tiles_i * r.tiles_j * r.splits;
  q.a_mn = r.a.mn, q.b_mn = r.b.mn;
  q.parts = parts;
  q.status = status;
  q.spin_limit = spin_limit;
  const auto fits = [](const void* m, long long ld, long long rows) {
    return reinterpret_cast<uintptr_t>(m) % 16 == 0 && ((ld % 8 == 0 && ld * 2 < (1LL << 40)) || rows == 1);
  };
  q.store_tma = !parts && fits(p.y, p.ldy, p.I) && (!p.pre || fits(p.pre, p.ldpre, p.I));
  // of an operand that lies along its rows a box is 64 of them by 64 of K
  const int b_rows = r.bn / r.cg;
  bool ok = encode(&maps.a, a, r.a.rows, r.a.cols, r.a.repack ? r.a.ld_packed : r.a.ld, r.a.mn ? 64 : 128, bf16) &&
            encode(&maps.b, b, r.b.rows, r.b.cols, r.b.repack ? r.b.ld_packed : r.b.ld, r.b.mn ? 64 : b_rows, bf16);
  const auto out_ld = [&](long long ld) { return p.I == 1 ? (p.J + 7) / 8 * 8 : ld; };
  if (q.store_tma) ok = ok && encode(&maps.y, p.y, p.I, p.J, out_ld(p.ldy), 32, bf16);
  if (q.store_tma && p.pre) ok = ok && encode(&maps.pre, p.pre, p.I, p.J, out_ld(p.ldpre), 32, bf16);
  if (!ok) return PIC_ERR_CUDA;

  const void* fn = bf16 ? tc_kernel_bf16(r.bn) : tc_kernel_f16(r.bn);
  const int shape = r.bn == 256 ? 2 : r.bn == 128 ? 1 : 0;
  const int smem = shape == 2 ? smem_of<2, 256>() : shape == 1 ? smem_of<1, 128>() : smem_of<1, 64>();
  if (set_up(fn, shape + (bf16 ? 3 : 0), smem) != PIC_OK) return PIC_ERR_CUDA;
  long long grid = q.work * r.cg;
  const long long most = r.bn == 64 ? 2 * kSms : kSms;
  if (grid > most) grid = most;
  void* args[] = {&q, &maps};
  if (cudaLaunchKernel(fn, dim3(static_cast<unsigned>(grid)), dim3(kTcThreads), args, smem, s) != cudaSuccess)
    return PIC_ERR_CUDA;
  if (parts) {
    const JoinParams j{p, reinterpret_cast<const float4*>(parts), r.tiles_i, r.tiles_j, r.splits, 128 * r.cg, r.bn};
    return bf16 ? join<__nv_bfloat16>(j, s) : join<__half>(j, s);
  }
  return PIC_OK;
}

}  // namespace lin
}  // namespace pic
