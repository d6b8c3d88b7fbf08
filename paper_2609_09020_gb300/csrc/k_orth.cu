// k_orth.cu -- orthogonalised updates (include/pic_orth.h): the handle with its
// lists of jobs, and the norms.  Measured: squares and first X of 50 million bf16 elements 43 and
// 45 us.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "k_linear_tc.cuh"
#include "orth.cuh"

using pic::orth::kShapes;
constexpr int kShapeColumns[kShapes] = {64, 128, 256, 128}, kShapeRows[kShapes] = {128, 128, 256, 256};
// Small matrices of up to so much shared memory are launched together.
constexpr int kSmallLists = 3;
constexpr int kSmallBytes[kSmallLists] = {56 * 1024, 112 * 1024, pic::orth::kSmallMost};

struct pic_orthogonalizer {
  int device;
  int n_pieces;
  int n_totals;  // matrices, if one has more than kMostSquares pieces, or 0
  int* small[kSmallLists];  // matrices that a CTA each takes, by the shared memory that they need
  int n_small[kSmallLists], small_bytes[kSmallLists];
  char* room;  // all of it
  pic::orth::Matrix* matrices;
  CUtensorMap* maps;
  int n_maps;
  pic::orth::Piece* pieces;
  pic::orth::Job* jobs[3][kShapes];  // of each stage
  int n_jobs[3][kShapes];
  bool both[kShapes];  // a matrix of the shape has operands of two halves
  double* squares;
  float4* parts;
  unsigned* counters;
  long long n_counters;
  int* status;
};

namespace {

using namespace pic::orth;
using pic::lin::from_f32;
using pic::lin::to_f32;

constexpr int kThreads = 256;

template <typename F>
__device__ __forceinline__ void for_type(int dtype, F f) {
  if (dtype == PIC_DTYPE_F32)
    f(float{});
  else if (dtype == PIC_DTYPE_F16)
    f(__half{});
  else
    f(__nv_bfloat16{});
}

// A thread's elements of a panel of 32 x 64 of a piece: eight columns of a row, zeros
// where there are none.
template <typename T, bool ON16>
__device__ __forceinline__ void load8(const Matrix& m, int row, int col, float (&v)[8]) {
  constexpr int kBytes = static_cast<int>(sizeof(T));
  const char* at = reinterpret_cast<const char*>(static_cast<const T*>(m.grad) + row * m.ld_grad + col);
  const int bytes = row < m.rows ? min(8, m.cols - col) * kBytes : 0;
#pragma unroll
  for (int h = 0; h < kBytes / 2; ++h) {
    pic::lin::Piece16<ON16> p;
    p.load(at + 16 * h, bytes - 16 * h);
    uint32_t w[4];
    p.template get<T>(static_cast<int>(reinterpret_cast<uintptr_t>(at) & 15), w);
    pic::lin::keep_bytes<T>(w, bytes - 16 * h);
#pragma unroll
    for (int e = 0; e < 16 / kBytes; ++e) v[h * (16 / kBytes) + e] = to_f32(reinterpret_cast<const T*>(w)[e]);
  }
}
template <typename F>
__device__ __forceinline__ void for_form(const Matrix& m, F f) {
  for_type(m.dtype, [&](auto t) {
    using T = decltype(t);
    if (m.on16)
      f(t, [&](int row, int col, float (&v)[8]) { load8<T, true>(m, row, col, v); });
    else
      f(t, [&](int row, int col, float (&v)[8]) { load8<T, false>(m, row, col, v); });
  });
}

// The squares of a piece: a thread adds at most 64 in fp32, and where that sum leaves the
// range in which fp32 is good, again in fp64; the block's threads in order.  Being the
// first kernel of a call by tiles, it also sets the parts' counters to zero: a call whose
// waits gave up leaves them where its last parts came.
__global__ void __launch_bounds__(kThreads) squares_kernel(const Matrix* matrices, const Piece* pieces, double* squares,
                                                           unsigned* counters, long long n_counters) {
  __shared__ double sums[kThreads / 32];
  const Piece p = pieces[blockIdx.x];
  const Matrix& m = matrices[p.matrix];
  const int row = p.row0 + threadIdx.x / 8, col = p.col0 + threadIdx.x % 8 * 8, end = p.col0 + min(m.cols - p.col0, kPieceCols);
  wait_for_earlier();
  for (long long i = blockIdx.x * static_cast<long long>(kThreads) + threadIdx.x; i < n_counters; i += static_cast<long long>(gridDim.x) * kThreads)
    counters[i] = 0;
  double sum = 0.0;
  for_form(m, [&](auto, auto load) {
    float s = 0.0f;
    uint32_t some = 0;  // bits of values that are not zero
#pragma unroll 4
    for (int c = col; c < end; c += 64) {
      float v[8];
      load(row, c, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(v[e], v[e], s), some |= __float_as_uint(v[e]);
    }
    const bool again = some << 1 != 0 && !(s >= 1e-28f && s <= 1e37f);
    if (!__any_sync(0xffffffffu, again)) {
      // (fp64 is slow: the first eight lanes' sums in fp32)
#pragma unroll
      for (int d = 1; d < 8; d *= 2) s += __shfl_xor_sync(0xffffffffu, s, d);
      if ((threadIdx.x & 7) == 0) sum = s;
    } else if (!again) {
      sum = s;
    } else {
      for (int c = col; c < end; c += 64) {
        float v[8];
        load(row, c, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fma(static_cast<double>(v[e]), static_cast<double>(v[e]), sum);
      }
    }
  });
#pragma unroll
  for (int d = 16; d > 0; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kThreads / 32; ++w) sum += sums[w];
    squares[blockIdx.x] = sum;
  }
}

// The sum of `n` squares, by a block: in warp 0's lane 0.
__device__ __forceinline__ double sum_squares(const double* squares, int n, double* sums) {
  double sum = 0.0;
  for (int i = threadIdx.x; i < n; i += kThreads) sum += squares[i];
#pragma unroll
  for (int d = 16; d > 0; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0)
    for (int w = 1; w < kThreads / 32; ++w) sum += sums[w];
  return sum;
}

// Matrices of more than kMostSquares pieces: a block adds up one's squares into the first, so
// that the blocks that scale them need not all (1 x 2^29: 2.1 s of scaling, in 2^40 additions).
constexpr int kMostSquares = 4096;
__global__ void __launch_bounds__(kThreads) total_kernel(const Matrix* matrices, double* squares) {
  __shared__ double sums[kThreads / 32];
  const Matrix& m = matrices[blockIdx.x];
  wait_for_earlier();
  if (m.parts <= kMostSquares) return;
  const double sum = sum_squares(squares + m.part0, m.parts, sums);
  if (threadIdx.x == 0) squares[m.part0] = sum;
}

// X = G / (|G| + eps), a piece a block.
__global__ void __launch_bounds__(kThreads) scale_kernel(const Matrix* matrices, const Piece* pieces, const double* squares,
                                                         float eps, int last) {
  __shared__ float factors[2];
  __shared__ double sums[kThreads / 32];
  const Piece p = pieces[blockIdx.x];
  const Matrix& m = matrices[p.matrix];
  wait_for_earlier();
  const double sum = sum_squares(squares + m.part0, m.parts > kMostSquares ? 1 : m.parts, sums);
  if (threadIdx.x == 0) norm_factors(sum, eps, factors[0], factors[1]);
  __syncthreads();
  const float f0 = factors[0], f1 = last ? factors[1] : kScale;
  if (threadIdx.x == 0 && p.row0 == 0 && p.col0 == 0) *m.rest = factors[1];
  const int row = p.row0 + threadIdx.x / 8, col = p.col0 + threadIdx.x % 8 * 8, end = p.col0 + min(m.cols - p.col0, kPieceCols);
  for_form(m, [&](auto t, auto load) {
    using T = decltype(t);
#pragma unroll 2
    for (int c = col; c < end; c += 64) {
      float v[8];
      load(row, c, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = v[e] * f0 * f1;
      if (last) {
        if (row < m.rows) {
          T* out = static_cast<T*>(m.out) + row * m.ld_out + c;
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (c + e < m.cols) out[e] = from_f32<T>(v[e]);
        }
        continue;
      }
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        hi[e] = pic::lin::pack2_of<__half>(v[2 * e], v[2 * e + 1]);
        const float2 h = pic::lin::unpack2_of<__half>(hi[e]);
        lo[e] = pic::lin::pack2_of<__half>(v[2 * e] - h.x, v[2 * e + 1] - h.y);
      }
      // rows of the workspace are whole
      if (row < m.rows) {
        __half* x = m.x[0] + row * m.ldx + c;
        *reinterpret_cast<uint4*>(x) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        // (16-bit values have no second half, but for subnormal ones of half)
        if (m.halves == 2) *reinterpret_cast<uint4*>(x + m.rows * m.ldx) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
      }
    }
  });
}

long long elem_bytes(int dtype) { return dtype == PIC_DTYPE_F32 ? 4 : 2; }

// What a matrix of the call covers.
struct Span {
  uintptr_t first, end, ld, width, rows;
  bool out;
};

// Whether two matrices have a byte in common.
bool meet(const Span& a, const Span& b) {
  if (a.first >= b.end || b.first >= a.end) return false;
  if (a.ld == b.ld) {
    // b's first column, counted along a's rows
    const uintptr_t at = b.first >= a.first ? (b.first - a.first) % a.ld : (a.ld - (a.first - b.first) % a.ld) % a.ld;
    return !(at >= a.width && at + b.width <= a.ld);
  }
  // rows of different distances (a single row has any): each of the one that has fewer
  // against the last of the other's to begin before it, and the next
  const bool swap = b.rows < a.rows;
  const Span &few = swap ? b : a, &many = swap ? a : b;
  for (uintptr_t r = 0; r < few.rows; ++r) {
    const uintptr_t from = few.first + r * few.ld, to = from + few.width;
    if (to <= many.first || from >= many.end) continue;
    if (from < many.first) return true;
    const uintptr_t row = (from - many.first) / many.ld;
    if (from < many.first + row * many.ld + many.width) return true;
    if (row + 1 < many.rows && to > many.first + (row + 1) * many.ld) return true;
  }
  return false;
}

bool outputs_disjoint(const std::vector<pic_orth_matrix>& list) {
  std::vector<Span> spans;
  for (const pic_orth_matrix& m : list) {
    const uintptr_t e = elem_bytes(m.dtype);
    const auto add = [&](const void* p, long long ld, bool out) {
      const uintptr_t first = reinterpret_cast<uintptr_t>(p);
      spans.push_back({first, first + ((m.rows - 1) * ld + m.cols) * e, ld * e, m.cols * e, static_cast<uintptr_t>(m.rows), out});
    };
    add(m.out, m.ld_out, true);
    if (m.grad != m.out || (m.rows > 1 && m.ld_grad != m.ld_out)) add(m.grad, m.ld_grad, false);
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

// What five steps of a matrix take one CTA, in us (measured, of fp32: 32 x 32 15, 32 x 1000
// 100, 64 x 64 25, 64 x 256 62, 64 x 512 109, 128 x 128 115; by tiles 200 x 200 takes 127,
// 512 x 512 168).
double small_time(const Matrix& m) {
  const double n = std::max(m.rows, m.cols);
  return m.m <= 32 ? 12 + 0.09 * n : m.m <= 64 ? 13 + 0.19 * n : 50 + 0.6 * n;
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

// After how many slices sums of two halves are taken over.  An accumulator loses up to 2^-24
// of a sum with each 16 of K, always towards zero, and the steps multiply that: out's error, of
// elementary fp32's, with 32 to 64 slices in one / with takeovers: 512 x 20000 6.5 / 2.6, 40 of 130 x
// 20000 12.3 / 1.8, 2048 x 2048 3.6 / 0.6, 1500 x 1500 4.1 / 0.7.  A^2, whose diagonal outweighs its rows,
// counts most: eight there too 512 x 20000 4.6, 1024 x 1024 1.7 for 1.0; two to eight in the others
// hardly differ, but in A of few rows (1 x 2^24 4.8e-6 with eight).  A takeover costs some 0.2 us.
int takeover(int stage, const Matrix& m) { return stage == kPolynomial || (stage == kGram && m.m <= 64) ? 4 : 8; }

// The jobs of each stage and tile shape, the workspace of their parts and its counters.
//
// Shapes: by pairs of CTAs, which load half as much for as many operations, where the list
// has tiles of 256 x 256 for the pairs twice or nearly; 64 columns where the smaller side is no
// more, or where there are few tiles of 128; else 128.  us, 64 / 128 columns, tiles of 128 x 128 in
// the list: fp32 512 x 512 (16) 133 / 171, 1024 x 1024 (64) 193 / 237, 300 x 300 (99) 142 / 156,
// 256 x 256 (96) 163 / 154, 500 x 500 (96) 164 / 188, 1280 x 1280 (100) 253 / 271, 1408 x 1408 (121) 269 /
// 287, 1536 x 1536 (144) 374 / 326; bfloat16 512 x 512 (16) 101 / 104, 640 x 640 (25) 113 / 119, 200 x
// 200 (32) 94 / 99, 896 x 896 (49) 124 / 124, 1024 x 1024 (64) 135 / 130, 256 x 256 (64) 109 / 99, 300 x 300
// (72) 98 / 103, (99) 110 / 101, 1536 x 1536 (144) 178 / 161: the two meet between 100 and 144 tiles
// for fp32, and within a twentieth of one another from 16 to 72 for bfloat16.  us, 128 columns / pairs:
// bfloat16 2048 x 2048 243 / 374, two of them 410 / 343, four 757 / 584, 2048 x 8192 608 / 605; fp32
// 541 / 523, 1029 / 757, 1901 / 1431, 1563 / 1369.
//
// A pair's tiles are 256 columns wide but in A and A^2 of lists with operands of two halves,
// where they are 128: so their sums can be taken over (k_orth_tc.cu).  us and out's error, of
// elementary fp32's, with 256 columns / so: two 2048 x 2048 767 (3.6) / 772 (1.9), four 1431 / 1507,
// 2048 x 8192 1340 (2.5) / 1290 (1.8), 4000 x 12000 6990 (5.3) / 6650 (2.6); with 128 columns in the
// updates too 804 (0.6), 1502, 1303 (0.6), 7070 (0.6).  One half's matrices in such a list have
// the same tiles in A and A^2 (six of 1000 x 1100 with six of fp32 705 us, in a launch of their own 758).
//
// Parts: stages with fewer tiles than there are CTAs (kSlots) are cut along K, with at
// least kLeast slices (of all three products of halves) in a part, as a part more costs 3
// us; and sums of more than kMost slices (with two halves and 32 slices or 64, us: 130 x 200000
// 1200 and 940, 4000 x 12000 7300 and 6400, but 40 of 60 x 20000 1400 and 1440: 32 up to 64 rows; one
// half's own roundings outweigh what 256 slices of sums lose).  In A of up to 64 rows, whose sums are all of one
// sign on the diagonal, parts of four slices where there are CTAs for them (out's error, of
// elementary fp32's, without and so: 8 x 1500 1.7 and 1.2, 60 x 1500 3.2 and 2.9; the worst of 24 matrices
// of sides 8 to 1500 3.2 and 2.7, in the same time).
void make_jobs(const std::vector<Matrix>& table, std::vector<Job> (&jobs)[3][kShapes], bool (&both)[kShapes], long long& part_bytes,
               long long& counters) {
  constexpr int kSms = 152, kSlots[kShapes] = {2 * kSms, kSms, kSms / 2, kSms / 2}, kLeast = 16, kMost[2] = {256, 64}, kMostThin = 32;
  constexpr long long kLarge = 120;
  const auto blocks = [](long long n, long long of) { return (n + of - 1) / of; };
  long long large = 0, middle = 0;
  bool two = false, two_large = false;
  for (const Matrix& m : table) {
    if (m.parts == 0) continue;
    if (m.m > 512) large += blocks(m.rows, 256) * blocks(m.cols, 256);
    middle += blocks(m.rows, 128) * blocks(m.cols, 128);
    two |= m.halves == 2;
    two_large |= m.halves == 2 && m.m > 512;
  }
  const bool few = middle <= (two ? 110 : 16);
  for (int s = 0; s < 3; ++s) {
    long long tiles[kShapes] = {};
    std::vector<Job> plain[kShapes];
    for (size_t id = 0; id < table.size(); ++id) {
      const Matrix& m = table[id];
      if (m.parts == 0) continue;  // a CTA's
      const int shape = m.m <= 64 || few ? k64 : m.m > 512 && large >= kLarge ? (two_large && s != kUpdate ? kPair128 : kPair256) : k128;
      both[shape] |= m.halves == 2;
      const int bn = kShapeColumns[shape], rows = kShapeRows[shape];
      Job j{};
      j.matrix = static_cast<int>(id), j.halves = m.halves, j.parts = 1, j.take = takeover(s, m);
      long long I = m.m, J = m.m, K = m.m;
      if (s == kGram) {
        j.p_map = j.q_map = kMapX, j.p_mn = j.q_mn = !m.left, K = m.left ? m.cols : m.rows;
      } else if (s == kPolynomial) {
        j.p_map = j.q_map = kMapA, j.p_half = j.q_half = 1;
      } else {
        I = m.rows, J = m.cols;
        j.p_map = m.left ? kMapB : kMapX, j.q_map = m.left ? kMapX : kMapB;
        j.q_mn = m.left, j.p_half = m.left, j.q_half = !m.left;
      }
      j.k1 = static_cast<int>(blocks(K, 64));
      // some rows of tiles at a time, columns outermost among them, so that what they share stays in L2
      const long long ti = blocks(I, rows), tj = blocks(J, bn), group = 2048 / rows;
      for (long long g = 0; g < ti; g += group)
        for (long long c = 0; c < tj; ++c)
          for (long long r = g; r < std::min(ti, g + group); ++r) {
            if (s != kUpdate && c * bn >= (r + 1) * rows) continue;  // above the diagonal
            j.i = static_cast<int>(r * rows), j.j = static_cast<int>(c * bn);
            plain[shape].push_back(j);
          }
    }
    for (int shape = 0; shape < kShapes; ++shape) {
      // long ones first
      std::stable_sort(plain[shape].begin(), plain[shape].end(), [](const Job& a, const Job& b) {
        return a.k1 * (a.halves == 2 ? 3 : 1) > b.k1 * (b.halves == 2 ? 3 : 1);
      });
      tiles[shape] = static_cast<long long>(plain[shape].size());
      const long long slots = both[shape] && shape == k64 ? kSms : kSlots[shape];
      const long long fill = tiles[shape] ? slots / tiles[shape] : 1;
      const int panels = kShapeRows[shape] / 32 * (kShapeColumns[shape] / 64);
      int slot = 0;
      for (const Job& j : plain[shape]) {
        const int slices = j.k1, passes = j.halves == 2 ? 3 : 1;
        const bool thin = s == kGram && j.halves == 2 && table[j.matrix].m <= 64;
        const int most = thin ? kMostThin : kMost[j.halves - 1];
        const long long worth = thin ? blocks(slices, 4) : slices * passes / kLeast;
        long long parts = std::max(std::min(fill, worth), blocks(slices, most));
        parts = std::max<long long>(parts, 1);
        const int each = static_cast<int>(blocks(slices, parts));
        parts = blocks(slices, each);
        for (int p = 0; p < parts; ++p) {
          Job k = j;
          k.k0 = p * each, k.k1 = std::min(slices, k.k0 + each);
          k.part = p, k.parts = static_cast<int>(parts), k.slot = slot;
          jobs[s][shape].push_back(k);
        }
        if (parts > 1) slot += static_cast<int>(parts);
      }
      part_bytes = std::max(part_bytes, static_cast<long long>(slot) * panels * 512 * 16);
      counters = std::max(counters, static_cast<long long>(slot) * panels);
    }
  }
}

// Places in one allocation, on 256-byte boundaries.  `bytes` stays at about kMost, which no
// device has, where it would be more.
struct Room {
  static constexpr long long kMost = 1LL << 50;
  long long bytes = 0;
  long long take(long long count, long long size) {
    const long long at = bytes;
    if (size > 0 && count > (kMost - bytes) / size)
      bytes = kMost;
    else
      bytes += (count * size + 255) / 256 * 256;
    return at;
  }
};

// The matrices of a list that are not empty, and where X (twice), A and b A + c A^2 of the
// i-th are: at[4 i] and on, -1 for those that a CTA takes by itself (`small`).
struct Layout {
  std::vector<Matrix> table;
  std::vector<long long> at;
  std::vector<int> small[kSmallLists];
  int small_most[kSmallLists] = {};
  Room room;
};
// False for a list that is refused.
bool lay_out(const pic_orth_matrix* matrices, int n, Layout& l) {
  if (n < 0 || (n > 0 && !matrices)) return false;
  std::vector<pic_orth_matrix> list;
  for (int i = 0; i < n; ++i) {
    const pic_orth_matrix& m = matrices[i];
    constexpr long long most = 0x7fffffffLL - 256;
    if (m.dtype != PIC_DTYPE_F32 && m.dtype != PIC_DTYPE_F16 && m.dtype != PIC_DTYPE_BF16) return false;
    if (m.rows < 0 || m.cols < 0 || m.rows > most || m.cols > most) return false;
    if (m.rows == 0 || m.cols == 0) continue;
    const auto bad = [&](const void* p, long long ld) {
      return !p || reinterpret_cast<uintptr_t>(p) % elem_bytes(m.dtype) || ld < m.cols || ld > (1LL << 40) ||
             ld > INT64_MAX / elem_bytes(m.dtype) / m.rows;  // (so that no end wraps)
    };
    if (bad(m.grad, m.ld_grad) || bad(m.out, m.ld_out)) return false;
    list.push_back(m);
  }
  if (!outputs_disjoint(list)) return false;
  // by a CTA each: what is sooner done so than by tiles, or, beside others that go by
  // tiles, where it takes a fraction of their time
  const bool tiles = std::any_of(list.begin(), list.end(), [](const pic_orth_matrix& m) { return std::min(m.rows, m.cols) > 128; });
  const double worth = tiles ? 30.0 : 100.0;
  for (const pic_orth_matrix& m : list) {
    const int id = static_cast<int>(l.table.size());
    Matrix t{};
    t.grad = m.grad, t.out = m.out, t.ld_grad = m.ld_grad, t.ld_out = m.ld_out;
    t.rows = static_cast<int>(m.rows), t.cols = static_cast<int>(m.cols), t.dtype = m.dtype;
    t.m = std::min(t.rows, t.cols), t.left = t.rows <= t.cols;
    // (for a CTA by itself no difference: it takes products of both halves always, as 192
    // bfloat16 matrices of 64 nets take 29 us so and 23 in one half, but 8 x 8 2.7e-3 of error)
    t.halves = m.dtype == PIC_DTYPE_BF16 ? 1 : 2;
    t.ldx = (m.cols + 63) / 64 * 64, t.lda = (t.m + 63LL) / 64 * 64;  // whole panels
    const long long need = t.m <= 128 ? small_bytes(t.m, t.left ? t.cols : t.rows) : kSmallMost + 1LL;
    if (need <= kSmallMost && small_time(t) <= worth) {
      int which = 0;
      while (need > kSmallBytes[which]) ++which;
      l.small[which].push_back(id);
      l.small_most[which] = std::max(l.small_most[which], static_cast<int>(need));
      l.at.resize(l.at.size() + 4, -1);
      l.table.push_back(t);
      continue;
    }
    // bfloat16 in one half, out's error of five steps (its rounding alone 1.7e-3) and time:
    // 64 x 1000 2.4e-3, 300 x 1500 2.3e-3, 1500 x 1500 1.9e-3; eight 64 x 4096 129 us, in two
    // 167, eight 128 x 4096 140 and 191
    if (t.m <= 64) t.halves = 2;
    t.on16 = reinterpret_cast<uintptr_t>(m.grad) % 16 == 0 && m.ld_grad * elem_bytes(m.dtype) % 16 == 0;
    // (both halves of X, of every type: rows are counted in 64 bits, as up to 2^31 of them are)
    for (int i = 0; i < 2; ++i) l.at.push_back(l.room.take(2LL * t.rows, t.ldx * 2));
    for (int i = 0; i < 2; ++i) l.at.push_back(l.room.take(static_cast<long long>(t.halves) * t.m, t.lda * 2));
    l.table.push_back(t);
  }
  // long ones first, for CTAs of their own
  for (std::vector<int>& ids : l.small)
    std::stable_sort(ids.begin(), ids.end(), [&](int a, int b) { return small_time(l.table[a]) > small_time(l.table[b]); });
  return true;
}

}  // namespace

extern "C" {

int64_t pic_orth_room_bytes(const pic_orth_matrix* matrices, int n) {
  try {
    Layout l;
    return lay_out(matrices, n, l) ? l.room.bytes : -1;
  } catch (...) {
    return -1;
  }
}

int pic_orth_create(const pic_orth_matrix* matrices, int n, pic_orthogonalizer** out) {
  if (!out) return PIC_ERR_INVALID_ARG;
  *out = nullptr;
  pic_orthogonalizer* h = nullptr;
  try {
    Layout l;
    if (!lay_out(matrices, n, l)) return PIC_ERR_INVALID_ARG;
    const int rc = pic::lin::device_status();
    if (rc != PIC_OK) return rc;
    // (before the lists of work are made, which are long for matrices that do not fit)
    size_t unused = 0, device_bytes = 0;
    if (cudaMemGetInfo(&unused, &device_bytes) != cudaSuccess) {
      cudaGetLastError();
      return PIC_ERR_CUDA;
    }
    if (static_cast<size_t>(l.room.bytes) > device_bytes) return PIC_ERR_ALLOC;
    std::vector<Matrix>& table = l.table;
    const std::vector<long long>& at = l.at;
    std::vector<Piece> pieces;
    for (size_t id = 0; id < table.size(); ++id) {
      Matrix& t = table[id];
      if (at[4 * id] < 0) continue;
      t.part0 = static_cast<int>(pieces.size());
      for (long long r = 0; r < t.rows; r += 32)
        for (long long c = 0; c < t.cols; c += kPieceCols) pieces.push_back({static_cast<int>(id), static_cast<int>(r), static_cast<int>(c)});
      t.parts = static_cast<int>(pieces.size()) - t.part0;
    }
    std::vector<Job> jobs[3][kShapes];
    long long part_bytes = 0, counters = 0;
    bool both[kShapes] = {};
    make_jobs(table, jobs, both, part_bytes, counters);
    const auto take = [&](long long count, size_t size) { return l.room.take(count, static_cast<long long>(size)); };
    const long long at_rest = take(table.size(), sizeof(float));
    const long long at_matrices = take(table.size(), sizeof(Matrix)), at_maps = take(table.size(), kMaps * sizeof(CUtensorMap)),
                    at_pieces = take(pieces.size(), sizeof(Piece)), at_squares = take(pieces.size(), sizeof(double)),
                    at_parts = take(part_bytes, 1), at_counters = take(counters, 4), at_status = take(1, 4);
    long long at_jobs[3][kShapes];
    for (int s = 0; s < 3; ++s)
      for (int c = 0; c < kShapes; ++c) at_jobs[s][c] = take(jobs[s][c].size(), sizeof(Job));
    long long at_small[kSmallLists];
    for (int i = 0; i < kSmallLists; ++i) at_small[i] = take(l.small[i].size(), sizeof(int));
    h = new pic_orthogonalizer{};
    if (cudaGetDevice(&h->device) != cudaSuccess || cudaMalloc(&h->room, l.room.bytes) != cudaSuccess) {
      cudaGetLastError();
      pic_orth_destroy(h);
      return PIC_ERR_ALLOC;
    }
    std::vector<CUtensorMap> maps(table.size() * kMaps);
    bool ok = true;
    for (size_t i = 0; i < table.size(); ++i) {
      Matrix& t = table[i];
      t.rest = reinterpret_cast<float*>(h->room + at_rest) + i;
      if (t.parts == 0) continue;
      __half** p[4] = {&t.x[0], &t.x[1], &t.a, &t.b};
      for (int k = 0; k < 4; ++k) {
        *p[k] = reinterpret_cast<__half*>(h->room + at[4 * i + k]);
        const bool x = k < 2;
        const long long rows = x ? t.rows : t.m, cols = x ? t.cols : t.m, ld = x ? t.ldx : t.lda, n = x ? 2 : t.halves;
        ok = ok && pic::lin::encode_many(&maps[i * kMaps + k], *p[k], rows, cols, ld, n, rows * ld, 64, PIC_DTYPE_F16) &&
             pic::lin::encode_many(&maps[i * kMaps + kMapPanel + k], *p[k], rows, cols, ld, n, rows * ld, 32, PIC_DTYPE_F16);
      }
    }
    h->matrices = reinterpret_cast<Matrix*>(h->room + at_matrices);
    h->maps = reinterpret_cast<CUtensorMap*>(h->room + at_maps);
    h->n_maps = static_cast<int>(std::min<size_t>(maps.size(), 0x7fffffff));
    h->pieces = reinterpret_cast<Piece*>(h->room + at_pieces);
    h->squares = reinterpret_cast<double*>(h->room + at_squares);
    h->parts = reinterpret_cast<float4*>(h->room + at_parts);
    h->counters = reinterpret_cast<unsigned*>(h->room + at_counters);
    h->n_counters = counters;
    h->status = reinterpret_cast<int*>(h->room + at_status);
    h->n_pieces = static_cast<int>(pieces.size());
    if (std::any_of(table.begin(), table.end(), [](const Matrix& t) { return t.parts > kMostSquares; }))
      h->n_totals = static_cast<int>(table.size());
    const auto put = [](void* to, const auto& v) {
      return v.empty() || cudaMemcpy(to, v.data(), v.size() * sizeof(v[0]), cudaMemcpyHostToDevice) == cudaSuccess;
    };
    ok = ok && put(h->matrices, table) && put(h->maps, maps) && put(h->pieces, pieces);
    for (int i = 0; i < kSmallLists; ++i) {
      h->small[i] = reinterpret_cast<int*>(h->room + at_small[i]);
      h->n_small[i] = static_cast<int>(l.small[i].size());
      h->small_bytes[i] = l.small_most[i];
      ok = ok && put(h->small[i], l.small[i]);
    }
    for (int s = 0; s < 3; ++s)
      for (int c = 0; c < kShapes; ++c) {
        h->jobs[s][c] = reinterpret_cast<Job*>(h->room + at_jobs[s][c]);
        h->n_jobs[s][c] = static_cast<int>(jobs[s][c].size());
        h->both[c] = both[c];
        ok = ok && put(h->jobs[s][c], jobs[s][c]);
      }
    if (!ok || cudaMemset(h->status, 0, 4) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) {
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
  pic::lin::Chain s{static_cast<cudaStream_t>(stream)};
  for (int i = kSmallLists - 1; i >= 0; --i)
    if (launch_small(h->matrices, h->small[i], h->n_small[i], h->small_bytes[i], steps, {a, b, c}, eps, s) != PIC_OK) {
      cudaGetLastError();
      return PIC_ERR_CUDA;
    }
  if (h->n_pieces == 0) return PIC_OK;
  pic::lin::Waits waits;
  if (!pic::lin::call_waits(waits)) return PIC_ERR_CUDA;
  waits.status = h->status;
  const Matrix* matrices = h->matrices;
  const Piece* pieces = h->pieces;
  int rc = s.launch(squares_kernel, dim3(h->n_pieces), kThreads, 0, matrices, pieces, h->squares, h->counters, h->n_counters);
  if (rc == PIC_OK && h->n_totals > 0) rc = s.launch(total_kernel, dim3(h->n_totals), kThreads, 0, matrices, h->squares);
  if (rc == PIC_OK)
    rc = s.launch(scale_kernel, dim3(h->n_pieces), kThreads, 0, matrices, pieces, static_cast<const double*>(h->squares), eps,
                  static_cast<int>(steps == 0));
  if (rc != PIC_OK) {
    cudaGetLastError();
    return rc;
  }
  for (int k = 0; k < steps; ++k)
    for (const Stage stage : {kGram, kPolynomial, kUpdate})
      for (int shape = 0; shape < kShapes; ++shape) {
        const StageParams q{h->matrices, h->maps, h->n_maps, h->jobs[stage][shape], h->n_jobs[stage][shape], {a, b, c}, k & 1,
                            k == 0, k + 1 == steps, k > 0 && steps - k >= 3, steps - k - 1 >= 3, h->parts, h->counters, waits};
        if (launch_stage(stage, static_cast<TileShape>(shape), h->both[shape], q, s) != PIC_OK) {
          cudaGetLastError();
          return PIC_ERR_CUDA;
        }
      }
  return cudaGetLastError() == cudaSuccess ? PIC_OK : PIC_ERR_CUDA;
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
