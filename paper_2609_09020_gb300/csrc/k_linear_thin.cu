// k_linear_thin.cu -- launches of the thin products (k_linear_thin.cuh).
#include <algorithm>
#include <atomic>

#include "k_linear_thin.cuh"

namespace pic {
namespace lin {
namespace {

constexpr int kSms = 152, kSmemSm = 227 * 1024;

// How rows of J columns of a matrix (if there is one) are written or read.
int mode_of(const void* m, long long ld, const Product& p, int elem) {
  if (!m) return kThinVector;
  const bool on16 = reinterpret_cast<uintptr_t>(m) % 16 == 0;
  if (on16 && ld * elem % 16 == 0 && p.J * elem % 16 == 0) return kThinVector;
  return on16 && ld == p.J ? kThinRun : kThinElements;
}

// A kernel's shared memory allowed once per device.
int allow(const void* fn, int slot) {
  static std::atomic<uint64_t> done[3 * 2 * 16];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return PIC_ERR_CUDA;
  const uint64_t bit = 1ull << (dev & 63);
  if (done[slot].load(std::memory_order_acquire) & bit) return PIC_OK;
  if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemSm - 2048) != cudaSuccess) return PIC_ERR_CUDA;
  done[slot].fetch_or(bit, std::memory_order_release);
  return PIC_OK;
}

}  // namespace

// Not 16-bit rows of exactly two slices of K of the tiled kernel, many of them and,
// like those of y, on 16-byte boundaries: nothing of its loads is wasted there.  us, here / tiled: fp16
// 200000 x 128 -> 128 28.6 / 22.1, -> 64 16.6 / 12.8; but 120 -> 64 17.0 / 24.8, 64 ->
// 128 18.8 / 20.4, 64 -> 64 11.5 / 12.4, 16 -> 128 15.2 / 31.5; 20000 x 128 -> 128 7.9
// / 7.3, -> 64 5.3 / 5.6; 300 x 64 -> 64 3.3 / 5.0.  fp32 200000 x 128 -> 128 96.9 /
// 156, 64 -> 64 31.8 / 55.9, 20000 x 64 -> 64 7.3 / 12.2; the one shape behind is up to
// 2000 rows of 128 -> 128, 11.5 / 9.7.
bool thin_takes(const Product& p, int dtype) {
  if (p.a_k != 1 || p.b_k != 1 || p.a_pre || p.K > kThinMost || p.J > kThinMost) return false;
  return dtype == PIC_DTYPE_F32 || p.K != kThinMost || p.J <= 32 || p.I < 65536 || p.a_i % 8 != 0 || p.J % 8 != 0 ||
         p.ldy % 8 != 0 || (reinterpret_cast<uintptr_t>(p.a) | reinterpret_cast<uintptr_t>(p.y)) % 16 != 0;
}

int thin_product(const Product& p, int dtype, cudaStream_t s) {
  const int elem = dtype == PIC_DTYPE_F32 ? 4 : 2;
  const int columns = static_cast<int>(p.J);
  ThinParams q{};
  q.p = p;
  q.y_mode = mode_of(p.y, p.ldy, p, elem);
  q.pre_mode = mode_of(p.pre, p.ldpre, p, elem);
  q.res_mode = mode_of(p.residual, p.ldr, p, elem);
  const bool x16 = reinterpret_cast<uintptr_t>(p.a) % 16 == 0 && p.a_i * elem % 16 == 0;
  const bool fast = x16 && q.y_mode == kThinVector && q.pre_mode == kThinVector && q.res_mode == kThinVector;
  const ThinKernel k = dtype == PIC_DTYPE_F32   ? thin_kernel_f32(columns, fast)
                       : dtype == PIC_DTYPE_F16 ? thin_kernel_f16(columns, fast)
                                                : thin_kernel_bf16(columns, fast);
  q.steps = static_cast<int>((p.K * elem + 127) / 128);
  q.pieces = static_cast<int>((p.K * elem + 63) / 64);
  q.ragged = p.K * elem % 16 != 0;
  q.w16 = reinterpret_cast<uintptr_t>(p.b) % 16 == 0 && p.b_j * elem % 16 == 0;
  const bool panels = q.y_mode != kThinVector || q.pre_mode != kThinVector || q.res_mode != kThinVector;
  q.panel_at = q.steps * k.step_bytes;
  q.panel_bytes = panels ? kThinRows * columns * elem : 0;
  q.tiles = (p.I + kThinRows - 1) / kThinRows;
  const int smem = q.panel_at + kThinWarps * q.panel_bytes;
  const int slot = (dtype * 2 + fast) * 16 + k.tiles - 1;
  if (smem > 46 * 1024 && allow(k.fn, slot) != PIC_OK) return PIC_ERR_CUDA;
  const long long ctas = std::min(k.ctas, kSmemSm / (smem + 2048));
  const long long grid = std::min(kSms * ctas, q.tiles);
  void* args[] = {&q};
  return launch_kernel(k.fn, grid, kThinThreads, smem, 1, args, s);
}

}  // namespace lin
}  // namespace pic
