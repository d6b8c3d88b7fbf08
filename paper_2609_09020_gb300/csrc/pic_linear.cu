// pic_linear.cu -- the C ABI of include/pic_linear.h: checks of arguments, the
// choice of kernels and the workspace's layout.
#include <atomic>

#include "linear.cuh"

namespace pic {
namespace lin {
namespace {

// The words that a kernel sets: when one of its bounded waits gives up, and when a
// grouped call's offsets are not as they must be.  Their address on each device is
// looked up once.
__device__ int lin_status[2];

int* status_word() {
  static std::atomic<int*> known[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
  int* p = known[dev].load(std::memory_order_relaxed);
  if (!p) {
    void* v = nullptr;
    if (cudaGetSymbolAddress(&v, lin_status) != cudaSuccess) return nullptr;
    p = static_cast<int*>(v);
    known[dev].store(p, std::memory_order_relaxed);
  }
  return p;
}

// pic_linear_test_wait_fault's: nonzero only while a test makes a wait run out.
std::atomic<int> test_fault{0};
std::atomic<unsigned> test_spin_limit{0};

}  // namespace

// The device must be the one that the kernels are built for; looked up once
// per device (0: not yet, 1: it is, 2: it is not).
int device_status() {
  static std::atomic<int> known[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) {
    cudaGetLastError();
    return PIC_ERR_UNSUPPORTED;
  }
  if (dev < 0 || dev >= 64) return PIC_ERR_UNSUPPORTED;
  int k = known[dev].load(std::memory_order_relaxed);
  if (k == 0) {
    int major = 0, minor = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev) != cudaSuccess) {
      cudaGetLastError();
      return PIC_ERR_CUDA;
    }
    k = major == 10 && minor == 3 ? 1 : 2;
    known[dev].store(k, std::memory_order_relaxed);
  }
  return k == 1 ? PIC_OK : PIC_ERR_UNSUPPORTED;
}

// False if the status word has no address.
bool call_waits(Waits& w) {
  const unsigned limit = test_spin_limit.load(std::memory_order_relaxed);
  w = {status_word(), limit ? limit : pic::kWaitPolls, test_fault.load(std::memory_order_relaxed)};
  return w.status != nullptr;
}

int take_status(int word, cudaStream_t s) {
  int* status = status_word();
  int flag = 0;
  if (status) status += word;
  if (!status || cudaMemcpyAsync(&flag, status, sizeof(int), cudaMemcpyDeviceToHost, s) != cudaSuccess ||
      cudaStreamSynchronize(s) != cudaSuccess ||
      (flag && (cudaMemsetAsync(status, 0, sizeof(int), s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess))) {
    cudaGetLastError();
    return -1;
  }
  return flag;
}

}  // namespace lin
}  // namespace pic

namespace {

using pic::lin::Arena;
using pic::lin::GradAct;
using pic::lin::Product;

constexpr long long kMaxDim = 0x7fffffffLL - 256;

size_t elem_bytes(int dtype) { return dtype == PIC_DTYPE_F32 ? 4 : 2; }

bool type_ok(int dtype) { return dtype == PIC_DTYPE_F32 || dtype == PIC_DTYPE_F16 || dtype == PIC_DTYPE_BF16; }
bool act_ok(int act) { return act == PIC_ACT_NONE || act == PIC_ACT_RELU || act == PIC_ACT_GELU; }

bool aligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// A [rows][cols] matrix of the call: present, on its element's boundary, rows
// apart by at least a row and at most 2^40 elements.
bool matrix_ok(const void* p, long long ld, long long rows, long long cols, int dtype) {
  return (p || rows == 0) && aligned(p, elem_bytes(dtype)) && ld >= cols && ld <= (1LL << 40);
}

bool dims_ok(long long rows, long long in, long long out) {
  return rows >= 0 && in >= 1 && out >= 1 && rows <= kMaxDim && in <= kMaxDim && out <= kMaxDim;
}

bool args_ok(const pic_linear_args* a) {
  if (!a || !dims_ok(a->rows, a->in_features, a->out_features) || !type_ok(a->dtype) || !act_ok(a->act)) return false;
  const long long M = a->rows, K = a->in_features, N = a->out_features;
  if (!matrix_ok(a->x, a->ldx, M, K, a->dtype) || !matrix_ok(a->w, a->ldw, N, K, a->dtype) ||
      !matrix_ok(a->y, a->ldy, M, N, a->dtype))
    return false;
  if (a->bias && !aligned(a->bias, elem_bytes(a->dtype))) return false;
  if (a->residual && !matrix_ok(a->residual, a->ldr == 0 ? N : a->ldr, M, N, a->dtype)) return false;
  if (a->residual == a->y && a->residual && a->ldr != a->ldy) return false;
  return !a->pre || matrix_ok(a->pre, a->ldpre, M, N, a->dtype);
}

bool args_ok(const pic_linear_grad_args* a) {
  if (!a || !dims_ok(a->rows, a->in_features, a->out_features) || !type_ok(a->dtype) || !act_ok(a->act)) return false;
  const long long M = a->rows, K = a->in_features, N = a->out_features;
  if (!a->dx && !a->dw && !a->db) return false;
  if (!matrix_ok(a->dy, a->lddy, M, N, a->dtype)) return false;
  if (a->act != PIC_ACT_NONE && !matrix_ok(a->pre, a->ldpre, M, N, a->dtype)) return false;
  if (a->dw && (!matrix_ok(a->x, a->ldx, M, K, a->dtype) || !matrix_ok(a->dw, a->lddw, N, K, a->dtype))) return false;
  if (a->dx && (!matrix_ok(a->w, a->ldw, N, K, a->dtype) || !matrix_ok(a->dx, a->lddx, M, K, a->dtype))) return false;
  return !a->db || aligned(a->db, elem_bytes(a->dtype));
}

// Whether the kernels for few rows take a product (they need no workspace), its
// workspace bytes, and the product.
bool few(const Product& p, int dtype) {
  return dtype == PIC_DTYPE_F32 ? pic::lin::few32_takes(p) : pic::lin::few_takes(p);
}

long long product_workspace(const Product& p, int dtype) {
  return few(p, dtype) || pic::lin::thin_takes(p, dtype) ? 0 : pic::lin::tc_workspace(p, dtype);
}

int product(const Product& p, int dtype, void* ws, cudaStream_t s) {
  if (few(p, dtype))
    return dtype == PIC_DTYPE_F32 ? pic::lin::few32_product(p, s) : pic::lin::few_product(p, dtype, s);
  if (pic::lin::thin_takes(p, dtype)) return pic::lin::thin_product(p, dtype, s);
  pic::lin::Waits w;
  return pic::lin::call_waits(w) ? pic::lin::tc_product(p, dtype, ws, w, s) : PIC_ERR_CUDA;
}

Product forward_product(const pic_linear_args& a) {
  Product p{};
  p.a = a.x, p.a_i = a.ldx, p.a_k = 1;
  p.b = a.w, p.b_j = a.ldw, p.b_k = 1;
  p.I = a.rows, p.J = a.out_features, p.K = a.in_features;
  p.bias = a.bias, p.residual = a.residual, p.ldr = a.ldr;
  p.y = a.y, p.ldy = a.ldy, p.pre = a.pre, p.ldpre = a.ldpre, p.act = a.act;
  return p;
}

int forward(const pic_linear_args& a, Arena& ws, bool launch, cudaStream_t s) {
  if (a.rows == 0) return PIC_OK;
  const Product p = forward_product(a);
  void* w = ws.take(product_workspace(p, a.dtype));
  return launch ? product(p, a.dtype, w, s) : PIC_OK;
}

int zero_rows(void* p, long long ld, long long rows, long long cols, int dtype, cudaStream_t s) {
  const size_t e = elem_bytes(dtype);
  return cudaMemset2DAsync(p, ld * e, 0, cols * e, rows, s) == cudaSuccess ? PIC_OK : PIC_ERR_CUDA;
}

int backward(const pic_linear_grad_args& a, Arena& ws, bool launch, cudaStream_t s) {
  const long long M = a.rows, K = a.in_features, N = a.out_features;
  int rc = PIC_OK;
  if (M == 0) {
    if (!launch) return PIC_OK;
    if (a.dw) rc = zero_rows(a.dw, a.lddw, N, K, a.dtype, s);
    if (a.db && rc == PIC_OK) rc = zero_rows(a.db, N, 1, N, a.dtype, s);
    return rc;
  }
  if (N <= 128 && K <= 128) {
    const pic::lin::NarrowGrad g{a.dy, a.lddy, a.pre, a.ldpre, a.x, a.ldx, a.w, a.ldw, a.dx, a.lddx,
                                 a.dw, a.lddw, a.db, M, static_cast<int>(N), static_cast<int>(K), a.act};
    if (pic::lin::narrow_takes(g, a.dtype)) {
      void* w = ws.take(pic::lin::narrow_workspace(g, a.dtype));
      if (!launch) return PIC_OK;
      pic::lin::Waits wt;
      return pic::lin::call_waits(wt) ? pic::lin::narrow_grad(g, a.dtype, w, wt, s) : PIC_ERR_CUDA;
    }
  }
  const auto dx_product = [&](const void* dz, long long lddz) {
    Product p{};
    p.a = dz, p.a_i = lddz, p.a_k = 1;
    p.b = a.w, p.b_j = 1, p.b_k = a.ldw;
    p.I = M, p.J = K, p.K = N;
    p.y = a.dx, p.ldy = a.lddx, p.act = PIC_ACT_NONE;
    return p;
  };
  bool dx = a.dx != nullptr, dw = a.dw != nullptr, db = a.db != nullptr;
  // few rows: dw and db by an outer product, dx from the weights straight, each with dz made on the way
  if (M <= pic::lin::kFewRows) {
    if (dw || db) {
      const pic::lin::OuterGrad g{a.dy, a.lddy, a.pre, a.ldpre, a.x, a.ldx, a.dw, a.lddw, a.db, M, N, K, a.act};
      if (launch && (rc = pic::lin::outer_grad(g, a.dtype, s)) != PIC_OK) return rc;
      dw = db = false;
    }
    Product p = dx_product(a.dy, a.lddy);
    if (a.act != PIC_ACT_NONE) p.a_pre = a.pre, p.a_pre_i = a.ldpre, p.a_act = a.act;
    if (dx && few(p, a.dtype)) {
      if (launch && (rc = product(p, a.dtype, nullptr, s)) != PIC_OK) return rc;
      dx = false;
    }
  }
  // dz: dy itself where there is no activation
  const void* dz = a.dy;
  long long lddz = a.lddy;
  const bool own_dz = a.act != PIC_ACT_NONE && (dx || dw);
  if (own_dz) {
    lddz = (N + 63) / 64 * 64;  // rows of 16-bit values on 128-byte lines
    dz = ws.take(M * lddz * static_cast<long long>(elem_bytes(a.dtype)));
  }
  if (own_dz || db) {
    GradAct g{a.dy, a.lddy, a.pre, a.ldpre, own_dz ? const_cast<void*>(dz) : nullptr, lddz, db ? a.db : nullptr, nullptr, M, N, a.act};
    g.parts = static_cast<float*>(ws.take(pic::lin::grad_act_workspace(g, a.dtype)));
    if (launch && (rc = pic::lin::grad_act(g, a.dtype, s)) != PIC_OK) return rc;
  }
  if (dx) {
    const Product p = dx_product(dz, lddz);
    void* w = ws.take(product_workspace(p, a.dtype));
    if (launch && (rc = product(p, a.dtype, w, s)) != PIC_OK) return rc;
  }
  if (dw) {
    Product p{};
    p.a = dz, p.a_i = 1, p.a_k = lddz;
    p.b = a.x, p.b_j = 1, p.b_k = a.ldx;
    p.I = N, p.J = K, p.K = M;
    p.y = a.dw, p.ldy = a.lddw, p.act = PIC_ACT_NONE;
    void* w = ws.take(product_workspace(p, a.dtype));
    if (launch && (rc = product(p, a.dtype, w, s)) != PIC_OK) return rc;
  }
  return PIC_OK;
}

template <typename Args, typename F>
int64_t count_bytes(const Args* a, F f) {
  if (!args_ok(a)) return -1;
  Arena ws{nullptr};
  f(*a, ws, false, nullptr);
  return ws.used;
}

template <typename Args, typename F>
int run(const Args* a, F f, void* workspace, size_t bytes, void* stream) {
  const int64_t need = count_bytes(a, f);
  if (need < 0 || bytes < static_cast<size_t>(need)) return PIC_ERR_INVALID_ARG;
  if (need > 0 && (!workspace || !aligned(workspace, 256))) return PIC_ERR_INVALID_ARG;
  const int rc = pic::lin::device_status();
  if (rc != PIC_OK) return rc;
  Arena ws{static_cast<char*>(workspace)};
  const int r = f(*a, ws, true, static_cast<cudaStream_t>(stream));
  if (r == PIC_ERR_CUDA) cudaGetLastError();
  return r;
}

}  // namespace

extern "C" {

int64_t pic_linear_workspace_bytes(const pic_linear_args* a) { return count_bytes(a, forward); }

int pic_linear(const pic_linear_args* a, void* workspace, size_t workspace_bytes, void* stream) {
  return run(a, forward, workspace, workspace_bytes, stream);
}

int64_t pic_linear_backward_workspace_bytes(const pic_linear_grad_args* a) { return count_bytes(a, backward); }

int pic_linear_backward(const pic_linear_grad_args* a, void* workspace, size_t workspace_bytes, void* stream) {
  return run(a, backward, workspace, workspace_bytes, stream);
}

int pic_linear_check(void* stream) {
  const int flag = pic::lin::take_status(0, static_cast<cudaStream_t>(stream));
  if (flag < 0) return PIC_ERR_CUDA;
  return flag ? PIC_ERR_TIMEOUT : PIC_OK;
}

int pic_linear_test_wait_fault(int withhold_arrival, unsigned spin_limit) {
  if (withhold_arrival != 0 && withhold_arrival != 1) return PIC_ERR_INVALID_ARG;
  pic::lin::test_spin_limit.store(spin_limit, std::memory_order_relaxed);
  pic::lin::test_fault.store(withhold_arrival, std::memory_order_relaxed);
  return PIC_OK;
}

}  // extern "C"
