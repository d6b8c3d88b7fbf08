// k_linear_thin.cuh -- products of at most 128 columns over at most 128 of K: a
// layer of a synthesis net over the pixels of an image.  y and x are all that
// there is to move, a few hundred bytes a row against some thousand operations, so
// the kernel is a stream: a warp takes 16 rows at a time, by itself, from memory
// straight into the fragments of warp-level MMAs (m16n8k16) and from their
// accumulators straight back.  The weights, in the order of the fragments, are in
// shared memory.  (Tiles of 128 rows through TMA, tensor memory and panels cost a
// CTA some 3 us each for 14 KB, and rows off 16-byte boundaries a copy before.)
// Measured, of the copy rate of 6.7 TB/s: fp16 393216 x 64 -> 64 ReLU keeping z 27.3
// us, 83 %; 632029 x 40 -> 64 keeping z 37 us, 86 %; 1034578 x 40 -> 16 22 us, 79 %;
// bf16 581299 x 32 -> 64 with residual 36 us, 77 %.  Off boundaries the shifts and
// panels bind, 660 instructions of a warp for 16 rows: 1365121 x 40 -> 44 GELU 81 us,
// 42 %.  fp32 is bound by its MMAs: 200000 x 64 -> 64 32 us, 49 %.
//
// Which of K's elements a lane holds in which fragment is free as long as both
// operands agree, and so is which column a fragment's column is.  So a lane has 16
// bytes in a row of x in each load, four lanes the row's next 64 bytes; and a lane
// ends up with neighbouring columns of y (16 bytes, 8 for the last 16 columns of a
// 16-bit type).  Rows of x off 16-byte boundaries: the two aligned pieces that
// have the 16 bytes, shifted (a piece that has an element of the row is in the
// row's allocation).  Rows of y, pre and the residual off them: if they lie end to
// end the warp's 16 rows are a run on a boundary, turned in shared memory; else
// element by element.
//
// fp32 values are cut into three bfloat16 pieces (cut3.cuh) in registers, with six
// MMAs for every 16 of K, which start from zero, and whose results are added to the
// sums to nearest (error of 27 of K 5.5e-8, of 128 7.4e-8; with pieces by
// truncation and sums inside the MMAs 2.6e-7); rows with an infinite or NaN value, or any if a weight is
// one, are computed again with FP32 FMAs.
//
// While a step (128 bytes of each row) is multiplied, the next, of this tile or the
// warp's next, is on its way.
#pragma once

#include "cut3.cuh"
#include "linear.cuh"
#include "linear_ptx.cuh"

namespace pic {
namespace lin {

constexpr int kThinMost = 128;  // columns, and K
constexpr int kThinThreads = 256, kThinWarps = kThinThreads / 32, kThinRows = 16;

// Rows of y, pre or the residual: 16 bytes of each lane's straight, or through a panel
// in shared memory: the warp's 16 rows one run of memory on a boundary, or not.
enum ThinMode { kThinVector = 0, kThinRun = 1, kThinElements = 2 };

struct ThinParams {
  Product p;
  int steps, pieces;        // of 128 and 64 bytes along K
  int ragged;               // K ends inside 16 bytes
  int w16;                  // rows of the weights start on 16-byte boundaries
  int y_mode, pre_mode, res_mode;  // a FAST kernel's are kThinVector
  int panel_at, panel_bytes;  // a warp's panel, where a mode needs it
  long long tiles;
};

// Groups of neighbouring columns: 32 of a 16-bit type (the last may have 16), 16 of fp32.
template <typename T, int NT>
struct ThinShape {
  static constexpr int kElem = static_cast<int>(sizeof(T));
  static constexpr bool kWide = kElem == 4;
  static constexpr int kGroup = kWide ? 2 : 4;  // MMA columns of 8 in a group
  static constexpr int kGroups = (NT + kGroup - 1) / kGroup;
  static constexpr int kPiece = 16 / kElem;  // elements of a load
  // a lane's weights for a piece and 8 columns: 8 of a 16-bit type, or 3 x 4 pieces of bfloat16
  static constexpr int kWords = kWide ? 6 : 4;
  static constexpr int kStepBytes = 2 * NT * 32 * kWords * 4;
  __host__ __device__ static constexpr int in_group(int g) { return NT - g * kGroup < kGroup ? NT - g * kGroup : kGroup; }
  // first column of lane group t in group g, and what MMA column nn of MMA tile j is
  __device__ static int column(int g, int t) { return g * kGroup * 8 + 2 * in_group(g) * t; }
  __device__ static int column_of(int j, int nn) {
    const int g = j / kGroup;
    return column(g, nn / 2) + 2 * (j - g * kGroup) + nn % 2;
  }
};

template <typename T>
__device__ __forceinline__ void thin_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  if constexpr (sizeof(T) == 2 && !std::is_same<T, __nv_bfloat16>::value)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The sums of a lane's places, on the FP32 cores.
template <int NT>
__device__ __noinline__ void thin_again(const Product& p, long long row, int t, float* u) {
  using S = ThinShape<float, NT>;
  const float *a = static_cast<const float*>(p.a), *b = static_cast<const float*>(p.b);
  for (int e = 0; e < NT * 4; ++e) {
    const long long i = row + (e & 2) * 4, j = S::column_of(e >> 2, 2 * t + (e & 1));
    float s = 0.0f;
    if (i < p.I && j < p.J)
      for (long long k = 0; k < p.K; ++k) s = fmaf(a[i * p.a_i + k], b[j * p.b_j + k], s);
    u[e] = s;
  }
}

// CTAs on an SM: what the registers of a kernel with NT x 8 columns leave room for
// (fp16 300000 x 128 -> 128 with one CTA 41 us, with two, which spill, 47; 581299 x 32
// -> 64 with residual two 36, three 41; the general kernel of 96 columns two 67, one 72).
template <typename T, int NT, bool FAST>
constexpr int thin_ctas() {
  if (sizeof(T) == 4) return NT <= 8 ? 2 : 1;
  if (NT <= 4) return FAST ? 4 : 2;
  return NT <= 8 || !FAST ? 2 : 1;
}

// FAST: rows of every matrix start and end on 16-byte boundaries (x's may end anywhere).
template <typename T, int NT, bool FAST>
__global__ void __launch_bounds__(kThinThreads, thin_ctas<T, NT, FAST>()) thin_kernel(const __grid_constant__ ThinParams q) {
  using S = ThinShape<T, NT>;
  constexpr int E = S::kElem;
  extern __shared__ __align__(16) uint8_t thin_smem[];
  __shared__ __align__(8) float bias[NT * 8];
  const Product& p = q.p;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int J = static_cast<int>(p.J), K = static_cast<int>(p.K);

  const long long first = warp * static_cast<long long>(gridDim.x) + blockIdx.x;  // few tiles: over all SMs
  const long long stride = gridDim.x * static_cast<long long>(kThinWarps);
  const char* a = static_cast<const char*>(p.a);
  const long long lda = p.a_i * E;
  const int k_bytes = K * E;
  uint8_t* panel = thin_smem + q.panel_at + warp * q.panel_bytes;
  // bytes of a tile's rows that lie end to end (a multiple of 16 but for the last tile's)
  const auto run_bytes = [&](long long tile) {
    return static_cast<int>(min(static_cast<long long>(kThinRows), p.I - tile * kThinRows)) * J * E;
  };

  Piece16<FAST> next[2][2];  // rows g and g + 8; the pieces of a step
  const auto fetch = [&](long long tile, int step) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const long long row = tile * kThinRows + g + 8 * h;
      const char* r = a + row * lda;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int at = step * 128 + c * 64 + t * 16;
        next[h][c].load(r + at, row < p.I ? k_bytes - at : 0);
      }
    }
  };
  // the residual of a tile: each lane's places, or 16 bytes here and there of a run
  uint32_t res[2][NT * E / 2];
  const auto fetch_residual = [&](long long tile) {
    const T* r = static_cast<const T*>(p.residual);
    if (FAST || q.res_mode == kThinVector) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const long long row = tile * kThinRows + g + 8 * h;
#pragma unroll
        for (int gi = 0; gi < S::kGroups; ++gi) {
          const int cols = 2 * S::in_group(gi), col = S::column(gi, t);
          const T* at = r + row * p.ldr + col;
          uint32_t* o = &res[h][gi * S::kGroup * E / 2];
          const bool there = row < p.I && col < J;
          if (cols * E == 16) {
            const uint4 w = load_if16(at, there);
            o[0] = w.x, o[1] = w.y, o[2] = w.z, o[3] = w.w;
          } else {
            o[0] = load_if(reinterpret_cast<const uint32_t*>(at), there);
            o[1] = load_if(reinterpret_cast<const uint32_t*>(at) + 1, there);
          }
        }
      }
    } else if (q.res_mode == kThinRun) {
      const int run = run_bytes(tile);
      const uint4* v = reinterpret_cast<const uint4*>(r + tile * kThinRows * p.J);
#pragma unroll
      for (int i = 0; i < NT * E / 4; ++i) {
        const uint4 w = load_if16(v + i * 32 + lane, (i * 32 + lane) * 16 < run);
        uint32_t* o = &res[0][0] + 4 * i;
        o[0] = w.x, o[1] = w.y, o[2] = w.z, o[3] = w.w;
      }
    }
  };
  if (first < q.tiles) {
    fetch(first, 0);
    if (p.residual) fetch_residual(first);
  }
  // the weights, zero outside, while the first rows are on their way
  uint32_t* frag = reinterpret_cast<uint32_t*>(thin_smem);
  bool bad_w = false;
  for (int e = threadIdx.x; e < q.steps * 2 * NT * 32; e += kThinThreads) {
    const int l = e & 31, j = e / 32 % NT, piece = e / 32 / NT;
    const int n = S::column_of(j, l >> 2), k0 = piece * (S::kPiece * 4) + (l & 3) * S::kPiece;
    const T* w = static_cast<const T*>(p.b) + n * p.b_j + k0;
    const int there = n < J ? K - k0 : 0;  // elements of the row from here on
    uint32_t v[4];
    if (q.w16) {
      const uint4 x = load_if16(w, there > 0);
      v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
      keep_bytes<T>(v, there * E);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (S::kWide) {
          v[i] = load_if(reinterpret_cast<const uint32_t*>(w) + i, i < there);
        } else {
          const uint16_t* u = reinterpret_cast<const uint16_t*>(w) + 2 * i;
          v[i] = load_if(u, 2 * i < there) | load_if(u + 1, 2 * i + 1 < there) << 16;
        }
      }
    }
    if constexpr (S::kWide) {
      uint32_t o[6];
#pragma unroll
      for (int i = 0; i < 4; ++i) bad_w |= (v[i] & 0x7fffffffu) >= kCutLimit;
      cut3(v[0], v[1], o[0], o[2], o[4]);
      cut3(v[2], v[3], o[1], o[3], o[5]);
      uint2* out = reinterpret_cast<uint2*>(frag) + ((piece * NT + j) * 3) * 32 + l;
#pragma unroll
      for (int i = 0; i < 3; ++i) out[i * 32] = make_uint2(o[2 * i], o[2 * i + 1]);
    } else {
      reinterpret_cast<uint4*>(frag)[e] = make_uint4(v[0], v[1], v[2], v[3]);
    }
  }
  for (int e = threadIdx.x; e < NT * 8; e += kThinThreads) {
    const int n = S::column_of(e / 8, e % 8);
    bias[e] = p.bias && n < p.J ? to_f32(static_cast<const T*>(p.bias)[n]) : 0.0f;
  }
  bad_w = __syncthreads_or(bad_w);

  const auto add_bias = [&](float (&acc)[NT][4]) {
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const float2 b = *reinterpret_cast<const float2*>(bias + j * 8 + 2 * t);
      acc[j][0] += b.x, acc[j][1] += b.y, acc[j][2] += b.x, acc[j][3] += b.y;
    }
  };
  for (long long tile = first; tile < q.tiles; tile += stride) {
    const long long row0 = tile * kThinRows, row = row0 + g;
    float acc[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[j][e] = 0.0f;
    // 16-bit types: sums begin with the bias (fp32 ones, in which the MMAs' truncations would show, end with it)
    if constexpr (!S::kWide) add_bias(acc);
    bool bad = bad_w;
    for (int step = 0; step < q.steps; ++step) {
      uint32_t x[2][2][4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int m = FAST ? 0 : static_cast<int>(reinterpret_cast<uintptr_t>(a + (row + 8 * h) * lda) & 15);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          next[h][c].template get<T>(m, x[h][c]);
          const int left = k_bytes - (step * 128 + c * 64 + t * 16);
          if (q.ragged && step == q.steps - 1) keep_bytes<T>(x[h][c], left);
        }
      }
      const bool last = step + 1 == q.steps;
      const long long next_tile = last ? tile + stride : tile;
      if (next_tile < q.tiles) fetch(next_tile, last ? 0 : step + 1);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        if (step * 2 + c >= q.pieces) break;
        if constexpr (S::kWide) {
          uint32_t y[2][6];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < 4; ++i) bad |= (x[h][c][i] & 0x7fffffffu) >= kCutLimit;
            cut3(x[h][c][0], x[h][c][1], y[h][0], y[h][2], y[h][4]);
            cut3(x[h][c][2], x[h][c][3], y[h][1], y[h][3], y[h][5]);
          }
          const uint2* b = reinterpret_cast<const uint2*>(frag) + (step * 2 + c) * NT * 3 * 32 + lane;
#pragma unroll
          for (int j = 0; j < NT; j += 2) {
            uint2 w[2][3];
#pragma unroll
            for (int i = 0; i < 6; ++i) w[i / 3][i % 3] = b[(j * 3 + i) * 32];
            float part[2][4] = {};  // an MMA truncates when it adds: 16 of K alone, and those rounded to the sums
#pragma unroll
            for (int k = 0; k < 6; ++k)
#pragma unroll
              for (int jj = 0; jj < 2; ++jj)
                thin_mma<T>(part[jj], y[0][2 * cut_a(k)], y[1][2 * cut_a(k)], y[0][2 * cut_a(k) + 1],
                            y[1][2 * cut_a(k) + 1], w[jj][cut_b(k)].x, w[jj][cut_b(k)].y);
#pragma unroll
            for (int jj = 0; jj < 2; ++jj)
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[j + jj][e] += part[jj][e];
          }
        } else {
          const uint4* b = reinterpret_cast<const uint4*>(frag) + (step * 2 + c) * NT * 32 + lane;
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            const uint4 w = b[j * 32];
            thin_mma<T>(acc[j], x[0][c][0], x[1][c][0], x[0][c][1], x[1][c][1], w.x, w.y);
            thin_mma<T>(acc[j], x[0][c][2], x[1][c][2], x[0][c][3], x[1][c][3], w.z, w.w);
          }
        }
      }
    }
    if constexpr (S::kWide) {
      if (__any_sync(0xffffffffu, bad)) {
        float u[NT * 4];
        thin_again<NT>(p, row, t, u);
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[j][e] = u[4 * j + e];
      }
    }
    if constexpr (S::kWide) add_bias(acc);
    const int rows = static_cast<int>(min(static_cast<long long>(kThinRows), p.I - row0));
    // this lane's places of the 16 rows, rounded
    const auto put = [&](void* out, long long ld, int mode) {
      const bool straight = FAST || mode == kThinVector;
      if (!straight) __syncwarp();
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int gi = 0; gi < S::kGroups; ++gi) {
          const int cols = 2 * S::in_group(gi), col = S::column(gi, t);
          uint32_t w[4];
#pragma unroll
          for (int i = 0; i < cols / 2; ++i) {
            const float u = acc[gi * S::kGroup + i][2 * h], v = acc[gi * S::kGroup + i][2 * h + 1];
            if constexpr (S::kWide)
              w[2 * i] = __float_as_uint(u), w[2 * i + 1] = __float_as_uint(v);
            else
              w[i] = pack2_of<T>(u, v);
          }
          if (straight) {
            if (g + 8 * h >= rows || col >= J) continue;
            T* o = static_cast<T*>(out) + (row + 8 * h) * ld + col;
            if (cols * E == 16)
              *reinterpret_cast<uint4*>(o) = make_uint4(w[0], w[1], w[2], w[3]);
            else
              *reinterpret_cast<uint2*>(o) = make_uint2(w[0], w[1]);
            continue;
          }
          uint8_t* o = panel + ((g + 8 * h) * J + col) * E;
          if (S::kWide || J % 2 == 0) {
#pragma unroll
            for (int i = 0; i < cols * E / 4; ++i)
              if (col + i * (4 / E) < J) reinterpret_cast<uint32_t*>(o)[i] = w[i];
          } else {
#pragma unroll
            for (int i = 0; i < cols; ++i)
              if (col + i < J) reinterpret_cast<uint16_t*>(o)[i] = static_cast<uint16_t>(w[i / 2] >> (i % 2 * 16));
          }
        }
      if (straight) return;
      __syncwarp();
      T* o = static_cast<T*>(out) + row0 * ld;
      if (mode == kThinRun) {
        const int run = run_bytes(tile), whole = run / 16;
        for (int i = lane; i < whole; i += 32) reinterpret_cast<uint4*>(o)[i] = reinterpret_cast<const uint4*>(panel)[i];
        for (int i = whole * (16 / E) + lane; i < run / E; i += 32) o[i] = reinterpret_cast<const T*>(panel)[i];
      } else {
        for (int r = 0; r < rows; ++r)
          for (int c = lane; c < J; c += 32) o[r * ld + c] = reinterpret_cast<const T*>(panel)[r * J + c];
      }
    };
    if (p.pre) put(p.pre, p.ldpre, q.pre_mode);
    if (p.act == PIC_ACT_RELU) {
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][e] = relu_nan(acc[j][e]);
    } else if (p.act == PIC_ACT_GELU) {
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float2 y = gelu2<S::kWide>(make_float2(acc[j][2 * h], acc[j][2 * h + 1]));
          acc[j][2 * h] = y.x, acc[j][2 * h + 1] = y.y;
        }
    }
    if (p.residual) {
      if (FAST || q.res_mode == kThinVector) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            if constexpr (S::kWide) {
              acc[j][2 * h] += __uint_as_float(res[h][2 * j]);
              acc[j][2 * h + 1] += __uint_as_float(res[h][2 * j + 1]);
            } else {
              const float2 f = unpack2_of<T>(res[h][j]);
              acc[j][2 * h] += f.x, acc[j][2 * h + 1] += f.y;
            }
          }
      } else {
        __syncwarp();
        if (q.res_mode == kThinRun) {
#pragma unroll
          for (int i = 0; i < NT * E / 4; ++i) {
            const uint32_t* o = &res[0][0] + 4 * i;
            if ((i * 32 + lane) * 16 < run_bytes(tile))
              reinterpret_cast<uint4*>(panel)[i * 32 + lane] = make_uint4(o[0], o[1], o[2], o[3]);
          }
        } else {
          const T* r = static_cast<const T*>(p.residual) + row0 * p.ldr;
          using Bits = std::conditional_t<S::kWide, uint32_t, uint16_t>;
          for (int e0 = lane; e0 < rows * J; e0 += 32 * 8) {  // eight loads under way together
            uint32_t v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              const int e = e0 + 32 * u;
              v[u] = load_if(reinterpret_cast<const Bits*>(r + e / J * p.ldr + e % J), e < rows * J);
            }
#pragma unroll
            for (int u = 0; u < 8; ++u)
              if (e0 + 32 * u < rows * J) reinterpret_cast<Bits*>(panel)[e0 + 32 * u] = static_cast<Bits>(v[u]);
          }
        }
        __syncwarp();
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int col = S::column_of(j, 2 * t + e);
              if (col < J) acc[j][2 * h + e] += to_f32(reinterpret_cast<const T*>(panel)[(g + 8 * h) * J + col]);
            }
      }
      if (tile + stride < q.tiles) fetch_residual(tile + stride);
    }
    put(p.y, p.ldy, q.y_mode);
  }
}

// The kernel for a type, by the number of 8-column tiles.
struct ThinKernel {
  const void* fn;
  int tiles, step_bytes, ctas;
};
template <typename T, int NT>
ThinKernel thin_kernel_at(bool fast) {
  return {fast ? reinterpret_cast<const void*>(thin_kernel<T, NT, true>) : reinterpret_cast<const void*>(thin_kernel<T, NT, false>),
          NT, ThinShape<T, NT>::kStepBytes, fast ? thin_ctas<T, NT, true>() : thin_ctas<T, NT, false>()};
}
template <typename T>
ThinKernel thin_kernel_of(int columns, bool fast) {
  if (columns <= 16) return thin_kernel_at<T, 2>(fast);
  if (columns <= 32) return thin_kernel_at<T, 4>(fast);
  if (columns <= 48) return thin_kernel_at<T, 6>(fast);
  if (columns <= 64) return thin_kernel_at<T, 8>(fast);
  if (columns <= 96) return thin_kernel_at<T, 12>(fast);
  return thin_kernel_at<T, 16>(fast);
}
ThinKernel thin_kernel_f32(int columns, bool fast);
ThinKernel thin_kernel_f16(int columns, bool fast);
ThinKernel thin_kernel_bf16(int columns, bool fast);

}  // namespace lin
}  // namespace pic
