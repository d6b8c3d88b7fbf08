// k_orth.cu -- orthogonalised updates (include/pic_orth.h): the handle, the norms,
// and the products on the FP32 cores.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "orth.cuh"

struct pic_orthogonalizer {
  int device;
  int n_pieces, n_square, n_full;
  char* room;  // all of it
  pic::orth::Matrix* matrices;
  pic::orth::Piece* pieces;
  pic::orth::Tile* square;  // tiles of A and b A + c A^2
  pic::orth::Tile* full;    // tiles of X
  double* parts;
  int* status;
};

namespace {

using namespace pic::orth;
using pic::lin::from_f32;
using pic::lin::to_f32;

constexpr int kThreads = 256;
constexpr int kPiece = 16384;  // elements
constexpr int kTile = 64, kDeep = 16;

template <typename F>
__device__ __forceinline__ void for_type(int dtype, F f) {
  if (dtype == PIC_DTYPE_F32)
    f(float{});
  else if (dtype == PIC_DTYPE_F16)
    f(__half{});
  else
    f(__nv_bfloat16{});
}

// The squares of a piece: a thread adds at most 64 in fp32, and where that sum leaves the
// range in which fp32 is good, again in fp64; the block's threads in order.
__global__ void __launch_bounds__(kThreads) squares_kernel(const Matrix* matrices, const Piece* pieces, double* parts) {
  __shared__ double sums[kThreads / 32];
  const Piece p = pieces[blockIdx.x];
  const Matrix& m = matrices[p.matrix];
  double sum = 0.0;
  for_type(m.dtype, [&](auto t) {
    using T = decltype(t);
    const T* g = static_cast<const T*>(m.grad) + p.row0 * m.ld_grad + p.col0;
    const int count = p.rows * p.cols;
    float s = 0.0f;
    for (int e = threadIdx.x; e < count; e += kThreads) {
      const float v = to_f32(g[e / p.cols * m.ld_grad + e % p.cols]);
      s = fmaf(v, v, s);
    }
    sum = s;
    if (!(s >= 1e-28f && s <= 1e37f)) {
      sum = 0.0;
      for (int e = threadIdx.x; e < count; e += kThreads) {
        const double v = to_f32(g[e / p.cols * m.ld_grad + e % p.cols]);
        sum = fma(v, v, sum);
      }
    }
  });
#pragma unroll
  for (int d = 16; d > 0; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kThreads / 32; ++w) sum += sums[w];
    parts[blockIdx.x] = sum;
  }
}

// X = G / (|G| + eps), a piece a block: by a power of two first, then by what is left, so
// that no finite norm leaves fp32's range on the way.
__global__ void __launch_bounds__(kThreads) scale_kernel(const Matrix* matrices, const Piece* pieces, const double* parts,
                                                         float eps, int last) {
  __shared__ float factors[2];
  const Piece p = pieces[blockIdx.x];
  const Matrix& m = matrices[p.matrix];
  if (threadIdx.x < 32) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < m.parts; i += 32) sum += parts[m.part0 + i];
#pragma unroll
    for (int d = 16; d > 0; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if (threadIdx.x == 0) {
      const double norm = sqrt(sum) + eps;
      int e = 0;
      if (norm > 0.0 && norm < 1e300) frexp(norm, &e);
      e = min(max(e, -126), 126);
      factors[0] = static_cast<float>(ldexp(1.0, -e));
      factors[1] = static_cast<float>(ldexp(1.0, e) / norm);
    }
  }
  __syncthreads();
  const float f0 = factors[0], f1 = factors[1];
  for_type(m.dtype, [&](auto t) {
    using T = decltype(t);
    const T* g = static_cast<const T*>(m.grad);
    T* out = static_cast<T*>(m.out);
    for (int e = threadIdx.x; e < p.rows * p.cols; e += kThreads) {
      const long long r = p.row0 + e / p.cols, c = p.col0 + e % p.cols;
      const float v = to_f32(g[r * m.ld_grad + c]) * f0 * f1;
      if (last)
        out[r * m.ld_out + c] = from_f32<T>(v);
      else
        m.x[0][r * m.ldx + c] = v;
    }
  });
}

// Tile (i, j) of a product: STAGE 0 A = X X^T (or X^T X), 1 B = b A + c A A, 2 X' = a X +
// B X (or X B).  `last`: X' goes to out.
template <int STAGE>
__global__ void __launch_bounds__(kThreads) product_kernel(const Matrix* matrices, const Tile* tiles, Coefficients co,
                                                           int from, int last) {
  __shared__ __align__(16) float sa[kDeep][kTile + 4], sb[kDeep][kTile + 4];
  const Tile t = tiles[blockIdx.x];
  const Matrix& m = matrices[t.matrix];
  const float* x = m.x[from];
  const float *pa, *pb;
  long long ai, ak, bj, bk;
  int I, J, K;
  if (STAGE == 0) {
    pa = pb = x, I = J = m.m, K = m.left ? m.cols : m.rows;
    ai = bj = m.left ? m.ldx : 1, ak = bk = m.left ? 1 : m.ldx;
  } else if (STAGE == 1) {
    pa = pb = m.a, I = J = K = m.m;
    ai = bj = m.lda, ak = bk = 1;
  } else {
    I = m.rows, J = m.cols, K = m.m;
    pa = m.left ? m.b : x, ai = m.left ? m.lda : m.ldx, ak = 1;
    pb = m.left ? x : m.b, bj = m.left ? 1 : m.lda, bk = m.left ? m.ldx : 1;
  }
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const long long i0 = t.i * kTile, j0 = t.j * kTile;
  float acc[4][4] = {};
  for (int k0 = 0; k0 < K; k0 += kDeep) {
    for (int e = threadIdx.x; e < kTile * kDeep; e += kThreads) {
      const int ka = ak == 1 ? e % kDeep : e / kTile, ia = ak == 1 ? e / kDeep : e % kTile;
      sa[ka][ia] = i0 + ia < I && k0 + ka < K ? pa[(i0 + ia) * ai + (k0 + ka) * ak] : 0.0f;
      const int kb = bk == 1 ? e % kDeep : e / kTile, jb = bk == 1 ? e / kDeep : e % kTile;
      sb[kb][jb] = j0 + jb < J && k0 + kb < K ? pb[(j0 + jb) * bj + (k0 + kb) * bk] : 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kDeep; ++k) {
      const float4 u = *reinterpret_cast<const float4*>(&sa[k][4 * ty]), v = *reinterpret_cast<const float4*>(&sb[k][4 * tx]);
      const float p[4] = {u.x, u.y, u.z, u.w}, q[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[r][c] = fmaf(p[r], q[c], acc[r][c]);
    }
    __syncthreads();
  }
  for (int r = 0; r < 4; ++r)
    for (int c = 0; c < 4; ++c) {
      const long long i = i0 + 4 * ty + r, j = j0 + 4 * tx + c;
      if (i >= I || j >= J) continue;
      if (STAGE == 0) {
        m.a[i * m.lda + j] = acc[r][c];
      } else if (STAGE == 1) {
        m.b[i * m.lda + j] = co.b * m.a[i * m.lda + j] + co.c * acc[r][c];
      } else {
        const float v = co.a * x[i * m.ldx + j] + acc[r][c];
        if (last)
          for_type(m.dtype, [&](auto t) {
            using T = decltype(t);
            static_cast<T*>(m.out)[i * m.ld_out + j] = from_f32<T>(v);
          });
        else
          m.x[from ^ 1][i * m.ldx + j] = v;
      }
    }
}

long long elem_bytes(int dtype) { return dtype == PIC_DTYPE_F32 ? 4 : 2; }

// What a matrix of the call covers.
struct Span {
  uintptr_t first, end, ld, width;
  int matrix;
  bool out;
};

// Whether two matrices have an element in common, taking rows for whole spans where
// they are not the same distance apart.
bool meet(const Span& a, const Span& b) {
  if (a.first >= b.end || b.first >= a.end) return false;
  if (a.ld != b.ld) return true;
  // b's first column, counted along a's rows
  const uintptr_t at = b.first >= a.first ? (b.first - a.first) % a.ld : (a.ld - (a.first - b.first) % a.ld) % a.ld;
  return !(at >= a.width && at + b.width <= a.ld);
}

bool outputs_disjoint(const std::vector<pic_orth_matrix>& list) {
  std::vector<Span> spans;
  for (size_t i = 0; i < list.size(); ++i) {
    const pic_orth_matrix& m = list[i];
    const uintptr_t e = elem_bytes(m.dtype);
    const auto add = [&](const void* p, long long ld, bool out) {
      const uintptr_t first = reinterpret_cast<uintptr_t>(p);
      spans.push_back({first, first + ((m.rows - 1) * ld + m.cols) * e, ld * e, m.cols * e, static_cast<int>(i), out});
    };
    add(m.out, m.ld_out, true);
    if (m.grad != m.out || m.ld_grad != m.ld_out) add(m.grad, m.ld_grad, false);
  }
  std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.first < b.first; });
  std::vector<Span> open;
  for (const Span& s : spans) {
    open.erase(std::remove_if(open.begin(), open.end(), [&](const Span& o) { return o.end <= s.first; }), open.end());
    for (const Span& o : open)
      if ((o.out || s.out) && meet(o, s)) return false;
    open.push_back(s);
  }
  return true;
}

// Whether the singular values that steps meet, from [0, 1], stay in [-2, 2], and b s^2 + c
// s^4 within 12: what X and b A + c A^2 are held in has room for no more.
bool steps_ok(int steps, double a, double b, double c) {
  double top = 1.0;
  for (int k = 0; k < steps; ++k) {
    const double s2 = top * top;
    if (std::fabs(b) * s2 + std::fabs(c) * s2 * s2 > 12.0) return false;
    // |a s + b s^3 + c s^5| is largest at the end or where its derivative is zero
    const auto f = [&](double s) { return std::fabs(s * (a + s * s * (b + c * s * s))); };
    double next = f(top);
    const double disc = 9 * b * b - 20 * a * c;
    if (c != 0.0 && disc >= 0.0) {
      for (const double sign : {-1.0, 1.0}) {
        const double r = (-3 * b + sign * std::sqrt(disc)) / (10 * c);
        if (r > 0.0 && r < s2) next = std::max(next, f(std::sqrt(r)));
      }
    } else if (c == 0.0 && b != 0.0) {
      const double r = -a / (3 * b);
      if (r > 0.0 && r < s2) next = std::max(next, f(std::sqrt(r)));
    }
    top = next;
    if (!(top <= 2.0)) return false;
  }
  return true;
}

}  // namespace

extern "C" {

int pic_orth_create(const pic_orth_matrix* matrices, int n, pic_orthogonalizer** out) {
  if (!out) return PIC_ERR_INVALID_ARG;
  *out = nullptr;
  if (n < 0 || (n > 0 && !matrices)) return PIC_ERR_INVALID_ARG;
  pic_orthogonalizer* h = nullptr;
  try {
    std::vector<pic_orth_matrix> list;
    for (int i = 0; i < n; ++i) {
      const pic_orth_matrix& m = matrices[i];
      constexpr long long most = 0x7fffffffLL - 256;
      if (m.dtype != PIC_DTYPE_F32 && m.dtype != PIC_DTYPE_F16 && m.dtype != PIC_DTYPE_BF16) return PIC_ERR_INVALID_ARG;
      if (m.rows < 0 || m.cols < 0 || m.rows > most || m.cols > most) return PIC_ERR_INVALID_ARG;
      if (m.rows == 0 || m.cols == 0) continue;
      const auto bad = [&](const void* p, long long ld) {
        return !p || reinterpret_cast<uintptr_t>(p) % elem_bytes(m.dtype) || ld < m.cols || ld > (1LL << 40);
      };
      if (bad(m.grad, m.ld_grad) || bad(m.out, m.ld_out)) return PIC_ERR_INVALID_ARG;
      list.push_back(m);
    }
    if (!outputs_disjoint(list)) return PIC_ERR_INVALID_ARG;
    const int rc = pic::lin::device_status();
    if (rc != PIC_OK) return rc;
    std::vector<Matrix> table;
    std::vector<Piece> pieces;
    std::vector<Tile> square, full;
    long long bytes = 0;
    const auto take = [&](long long b) {
      const long long at = bytes;
      bytes += (b + 255) / 256 * 256;
      return at;
    };
    std::vector<long long> at;
    for (const pic_orth_matrix& m : list) {
      const int id = static_cast<int>(table.size());
      Matrix t{};
      t.grad = m.grad, t.out = m.out, t.ld_grad = m.ld_grad, t.ld_out = m.ld_out;
      t.rows = static_cast<int>(m.rows), t.cols = static_cast<int>(m.cols), t.dtype = m.dtype;
      t.m = std::min(t.rows, t.cols), t.left = t.rows <= t.cols;
      t.ldx = (m.cols + 7) / 8 * 8, t.lda = (t.m + 7) / 8 * 8;
      t.part0 = static_cast<int>(pieces.size());
      const int cols = std::min(t.cols, kPiece), rows = kPiece / cols;
      for (long long r = 0; r < t.rows; r += rows)
        for (long long c = 0; c < t.cols; c += cols)
          pieces.push_back({id, static_cast<int>(r), static_cast<int>(std::min<long long>(rows, t.rows - r)),
                            static_cast<int>(c), static_cast<int>(std::min<long long>(cols, t.cols - c))});
      t.parts = static_cast<int>(pieces.size()) - t.part0;
      for (int i = 0; i * kTile < t.m; ++i)
        for (int j = 0; j * kTile < t.m; ++j) square.push_back({id, i, j});
      for (int i = 0; i * static_cast<long long>(kTile) < t.rows; ++i)
        for (int j = 0; j * static_cast<long long>(kTile) < t.cols; ++j) full.push_back({id, i, j});
      for (int i = 0; i < 2; ++i) at.push_back(take(t.rows * t.ldx * 4));
      for (int i = 0; i < 2; ++i) at.push_back(take(t.m * t.lda * 4));
      table.push_back(t);
    }
    const long long at_matrices = take(table.size() * sizeof(Matrix)), at_pieces = take(pieces.size() * sizeof(Piece)),
                    at_square = take(square.size() * sizeof(Tile)), at_full = take(full.size() * sizeof(Tile)),
                    at_parts = take(pieces.size() * sizeof(double)), at_status = take(4);
    h = new pic_orthogonalizer{};
    if (cudaGetDevice(&h->device) != cudaSuccess || cudaMalloc(&h->room, bytes) != cudaSuccess) {
      cudaGetLastError();
      pic_orth_destroy(h);
      return PIC_ERR_ALLOC;
    }
    for (size_t i = 0; i < table.size(); ++i) {
      float** p[4] = {&table[i].x[0], &table[i].x[1], &table[i].a, &table[i].b};
      for (int k = 0; k < 4; ++k) *p[k] = reinterpret_cast<float*>(h->room + at[4 * i + k]);
    }
    h->matrices = reinterpret_cast<Matrix*>(h->room + at_matrices);
    h->pieces = reinterpret_cast<Piece*>(h->room + at_pieces);
    h->square = reinterpret_cast<Tile*>(h->room + at_square);
    h->full = reinterpret_cast<Tile*>(h->room + at_full);
    h->parts = reinterpret_cast<double*>(h->room + at_parts);
    h->status = reinterpret_cast<int*>(h->room + at_status);
    h->n_pieces = static_cast<int>(pieces.size());
    h->n_square = static_cast<int>(square.size());
    h->n_full = static_cast<int>(full.size());
    const auto put = [](void* to, const auto& v) {
      return v.empty() || cudaMemcpy(to, v.data(), v.size() * sizeof(v[0]), cudaMemcpyHostToDevice) == cudaSuccess;
    };
    if (!put(h->matrices, table) || !put(h->pieces, pieces) || !put(h->square, square) || !put(h->full, full) ||
        cudaMemset(h->status, 0, 4) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) {
      cudaGetLastError();
      pic_orth_destroy(h);
      return PIC_ERR_CUDA;
    }
    *out = h;
    return PIC_OK;
  } catch (const std::bad_alloc&) {
    pic_orth_destroy(h);
    return PIC_ERR_ALLOC;
  } catch (...) {
    pic_orth_destroy(h);
    return PIC_ERR_INVALID_ARG;
  }
}

int pic_orth(pic_orthogonalizer* h, int steps, float a, float b, float c, float eps, void* stream) {
  if (!h || steps < 0 || steps > 64 || !(eps >= 0.0f) || !std::isfinite(eps)) return PIC_ERR_INVALID_ARG;
  if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c) || !steps_ok(steps, a, b, c)) return PIC_ERR_INVALID_ARG;
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) {
    cudaGetLastError();
    return PIC_ERR_CUDA;
  }
  if (dev != h->device) return PIC_ERR_INVALID_ARG;
  if (h->n_pieces == 0) return PIC_OK;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const Coefficients co{a, b, c, eps};
  squares_kernel<<<h->n_pieces, kThreads, 0, s>>>(h->matrices, h->pieces, h->parts);
  scale_kernel<<<h->n_pieces, kThreads, 0, s>>>(h->matrices, h->pieces, h->parts, eps, steps == 0);
  for (int k = 0; k < steps; ++k) {
    product_kernel<0><<<h->n_square, kThreads, 0, s>>>(h->matrices, h->square, co, k & 1, 0);
    product_kernel<1><<<h->n_square, kThreads, 0, s>>>(h->matrices, h->square, co, k & 1, 0);
    product_kernel<2><<<h->n_full, kThreads, 0, s>>>(h->matrices, h->full, co, k & 1, k + 1 == steps);
  }
  if (cudaGetLastError() != cudaSuccess) return PIC_ERR_CUDA;
  return PIC_OK;
}

int pic_orth_check(pic_orthogonalizer* h, void* stream) {
  if (!h) return PIC_ERR_INVALID_ARG;
  int flag = 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (cudaMemcpyAsync(&flag, h->status, sizeof(int), cudaMemcpyDeviceToHost, s) != cudaSuccess ||
      cudaStreamSynchronize(s) != cudaSuccess ||
      (flag && (cudaMemsetAsync(h->status, 0, sizeof(int), s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess))) {
    cudaGetLastError();
    return PIC_ERR_CUDA;
  }
  return flag ? PIC_ERR_TIMEOUT : PIC_OK;
}

void pic_orth_destroy(pic_orthogonalizer* h) {
  if (!h) return;
  cudaFree(h->room);
  delete h;
}

}  // extern "C"
