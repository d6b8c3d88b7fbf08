// pic_group.cu -- the C ABI of include/pic_group.h: checks of arguments and the
// choice of kernels.
#include "group.cuh"

namespace {

using pic::grp::Chain;
using pic::grp::GroupProduct;
using pic::grp::GroupGradAct;

constexpr long long kMaxDim = 0x7fffffffLL - 256;

bool aligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
size_t elem_bytes(int dtype) { return dtype == PIC_DTYPE_F32 ? 4 : 2; }

// A [rows][cols] matrix of the call, or [groups] of them, each `group` elements behind the one before.
// (No address space has one whose last row is 2^60 elements from its first; up to there nothing wraps.)
bool matrix_ok(const void* p, long long ld, long long rows, long long cols, int dtype) {
  return (p || rows == 0) && aligned(p, elem_bytes(dtype)) && ld >= cols && ld <= (1LL << 40) &&
         (rows <= 1 || ld <= (1LL << 60) / rows);
}
bool matrices_ok(const void* p, long long ld, long long group, int groups, long long rows, long long cols, int dtype) {
  if (!matrix_ok(p, ld, rows, cols, dtype)) return false;
  return groups == 1 || (group <= (1LL << 44) && group >= (rows - 1) * ld + cols);
}
bool vectors_ok(const void* p, long long group, int groups, long long n, int dtype) {
  return aligned(p, elem_bytes(dtype)) && (groups == 1 || (group >= n && group <= (1LL << 44)));
}

template <typename Args>
bool sizes_ok(const Args* a) {
  if (!a) return false;
  const auto dim = [](long long v, long long least) { return v >= least && v <= kMaxDim; };
  return dim(a->rows, 0) && dim(a->in_features, 1) && dim(a->out_features, 1) && a->groups >= 1 &&
         a->groups <= PIC_MAX_GROUPS && (a->dtype == PIC_DTYPE_F32 || a->dtype == PIC_DTYPE_F16 || a->dtype == PIC_DTYPE_BF16) &&
         (a->act == PIC_ACT_NONE || a->act == PIC_ACT_RELU || a->act == PIC_ACT_GELU) && a->offsets && aligned(a->offsets, 8);
}

bool args_ok(const pic_grouped_linear_args* a) {
  if (!sizes_ok(a)) return false;
  const long long M = a->rows, K = a->in_features, N = a->out_features;
  return matrix_ok(a->x, a->ldx, M, K, a->dtype) && matrices_ok(a->w, a->ldw, a->w_group, a->groups, N, K, a->dtype) &&
         (!a->bias || vectors_ok(a->bias, a->bias_group, a->groups, N, a->dtype)) && matrix_ok(a->y, a->ldy, M, N, a->dtype) &&
         (!a->pre || matrix_ok(a->pre, a->ldpre, M, N, a->dtype));
}

bool args_ok(const pic_grouped_linear_grad_args* a) {
  if (!sizes_ok(a) || (!a->dx && !a->dw && !a->db)) return false;
  const long long M = a->rows, K = a->in_features, N = a->out_features;
  if (!matrix_ok(a->dy, a->lddy, M, N, a->dtype)) return false;
  if (a->act != PIC_ACT_NONE && !matrix_ok(a->pre, a->ldpre, M, N, a->dtype)) return false;
  if (a->dw && (!matrix_ok(a->x, a->ldx, M, K, a->dtype) ||
                !matrices_ok(a->dw, a->lddw, a->dw_group, a->groups, N, K, a->dtype)))
    return false;
  if (a->dx && (!matrices_ok(a->w, a->ldw, a->w_group, a->groups, N, K, a->dtype) || !matrix_ok(a->dx, a->lddx, M, K, a->dtype)))
    return false;
  return !a->db || vectors_ok(a->db, a->db_group, a->groups, N, a->dtype);
}

const long long* offsets_of(const int64_t* o) { return reinterpret_cast<const long long*>(o); }

int product(const GroupProduct& p, int dtype, pic::lin::Arena& ws, bool launch, const pic::lin::Waits& w, Chain& s) {
  if (pic::grp::tc_takes(p, dtype)) {
    void* room = ws.take(pic::grp::tc_workspace(p, dtype));
    return launch ? pic::grp::tc_product(p, dtype, room, w, s) : PIC_OK;
  }
  if (pic::grp::planes_takes(p, dtype)) return pic::grp::planes_product(p, ws, launch, w, s);
  return launch ? pic::grp::any_product(p, dtype, s) : PIC_OK;
}

// Few rows in the groups: up to `most` on average.
bool few(long long rows, int groups, int most) { return rows <= static_cast<long long>(most) * groups; }

// The forward of 16-bit types whose weights TMA can read goes by tiles that read them at the
// memory's rate; others would be laid out first.
bool few_forward(const pic_grouped_linear_args& a) {
  if (a.dtype == PIC_DTYPE_F32) return few(a.rows, a.groups, 24);
  const bool tma = aligned(a.w, 16) && a.ldw % 8 == 0 && (a.groups == 1 || a.w_group % 8 == 0) && a.ldw < (1LL << 39) && a.w_group < (1LL << 39);
  return !tma && few(a.rows, a.groups, 8);
}
// The gradient of 16-bit types: a row or two on average, or weights, x or dw that TMA cannot
// read or write.
bool few_backward(const pic_grouped_linear_grad_args& a) {
  if (a.dtype == PIC_DTYPE_F32) return few(a.rows, a.groups, 24);
  const auto tma = [&](const void* m, long long ld, long long group) {
    return !m || (aligned(m, 16) && ld % 8 == 0 && (a.groups == 1 || group % 8 == 0));
  };
  const bool all = (!a.dx || tma(a.w, a.ldw, a.w_group)) && (!a.dw || (tma(a.x, a.ldx, 0) && tma(a.dw, a.lddw, a.dw_group)));
  return few(a.rows, a.groups, all ? 1 : 4);
}

int forward(const pic_grouped_linear_args& a, pic::lin::Arena& ws, bool launch, const pic::lin::Waits& w, Chain& s) {
  if (a.rows == 0) return PIC_OK;
  GroupProduct p{};
  p.by_rows = true;
  p.a = a.x, p.a_i = a.ldx;
  p.b = a.w, p.b_group = a.w_group, p.b_j = a.ldw, p.b_k = 1;
  p.rows = a.rows, p.J = a.out_features, p.K = a.in_features;
  p.groups = a.groups, p.offsets = offsets_of(a.offsets);
  p.bias = a.bias, p.bias_group = a.bias_group;
  p.y = a.y, p.ldy = a.ldy, p.pre = a.pre, p.ldpre = a.ldpre, p.act = a.act;
  p.status = w.status;
  pic::lin::Product t{};
  t.a = a.x, t.a_i = a.ldx, t.a_k = 1;
  t.b = a.w, t.b_j = a.ldw, t.b_k = 1;
  t.I = a.rows, t.J = a.out_features, t.K = a.in_features;
  t.bias = a.bias;
  t.y = a.y, t.ldy = a.ldy, t.pre = a.pre, t.ldpre = a.ldpre, t.act = a.act;
  if (pic::lin::thin_group_takes(t, a.dtype)) {
    const pic::lin::ThinGroups g{p.offsets, a.groups, a.w_group, a.bias_group, w.status};
    return launch ? pic::lin::thin_group_product(t, a.dtype, g, s.stream) : PIC_OK;
  }
  if (few_forward(a)) return launch ? pic::grp::few_forward(p, a.dtype, s) : PIC_OK;
  return product(p, a.dtype, ws, launch, w, s);
}

int backward(const pic_grouped_linear_grad_args& a, pic::lin::Arena& ws, bool launch, const pic::lin::Waits& w, Chain& s) {
  const long long M = a.rows, K = a.in_features, N = a.out_features;
  int rc = PIC_OK;
  if (N <= 128 && K <= 128) {
    const pic::lin::NarrowGroups n{{a.dy, a.lddy, a.pre, a.ldpre, a.x, a.ldx, a.w, a.ldw, a.dx, a.lddx, a.dw, a.lddw, a.db, M,
                                    static_cast<int>(N), static_cast<int>(K), a.act},
                                   offsets_of(a.offsets), a.groups, a.w_group, a.dw_group, a.db_group};
    if (pic::lin::narrow_group_takes(n.g, a.groups, a.dtype)) {
      void* room = ws.take(pic::lin::narrow_group_workspace(n.g, a.groups, a.dtype));
      return launch ? pic::lin::narrow_group_grad(n, a.dtype, room, w, s) : PIC_OK;
    }
  }
  if (M == 0 || few_backward(a)) {
    if (!launch) return PIC_OK;
    GroupProduct p{};
    p.a = a.dy, p.a_i = a.lddy;
    if (a.act != PIC_ACT_NONE) p.a_pre = a.pre, p.a_pre_i = a.ldpre, p.a_act = a.act;
    p.rows = M, p.groups = a.groups, p.offsets = offsets_of(a.offsets), p.status = w.status;
    if (a.dx && M > 0) {
      p.b = a.w, p.b_group = a.w_group, p.b_j = 1, p.b_k = a.ldw;
      p.J = K, p.K = N;
      p.y = a.dx, p.ldy = a.lddx;
      if ((rc = pic::grp::few_dx(p, a.dtype, s)) != PIC_OK) return rc;
    }
    if (a.dw || a.db) {
      p.b = a.x, p.b_group = 0, p.b_j = 1, p.b_k = a.ldx;
      p.I = N, p.J = K;
      p.y = a.dw, p.ldy = a.lddw, p.y_group = a.dw_group;
      rc = pic::grp::few_dw(p, a.db, a.db_group, a.dtype, s);
    }
    return rc;
  }
  // dz: dy itself where there is no activation
  const void* dz = a.dy;
  long long lddz = a.lddy;
  const bool own_dz = a.act != PIC_ACT_NONE && (a.dx || a.dw);
  if (own_dz) {
    lddz = (N + 63) / 64 * 64;  // rows of 16-bit values on 128-byte lines
    dz = ws.take(M * lddz * static_cast<long long>(elem_bytes(a.dtype)));
  }
  if ((own_dz && M > 0) || a.db) {
    GroupGradAct g{a.dy, a.lddy, a.pre, a.ldpre, own_dz ? const_cast<void*>(dz) : nullptr, lddz, a.db, a.db_group, nullptr,
                   M, N, a.groups, a.act, offsets_of(a.offsets), w.status};
    g.parts = static_cast<float*>(ws.take(pic::grp::grad_act_workspace(g, a.dtype)));
    if (launch && (rc = pic::grp::grad_act(g, a.dtype, s)) != PIC_OK) return rc;
  }
  GroupProduct x{};
  x.a = dz, x.a_i = lddz;
  x.rows = M, x.groups = a.groups, x.offsets = offsets_of(a.offsets);
  x.act = PIC_ACT_NONE;
  x.status = w.status;
  GroupProduct v = x;
  x.by_rows = true;
  x.b = a.w, x.b_group = a.w_group, x.b_j = 1, x.b_k = a.ldw;
  x.J = K, x.K = N;
  x.y = a.dx, x.ldy = a.lddx;
  v.b = a.x, v.b_j = 1, v.b_k = a.ldx;
  v.I = N, v.J = K;
  v.y = a.dw, v.ldy = a.lddw, v.y_group = a.dw_group;
  if (a.dx && a.dw && pic::grp::planes_takes(x, a.dtype) && pic::grp::planes_takes(v, a.dtype))
    return pic::grp::planes_gradients(x, v, ws, launch, w, s);
  if (a.dx && (rc = product(x, a.dtype, ws, launch, w, s)) != PIC_OK) return rc;
  return a.dw ? product(v, a.dtype, ws, launch, w, s) : PIC_OK;
}

template <typename Args, typename F>
int64_t count_bytes(const Args* a, F f) {
  if (!args_ok(a)) return -1;
  pic::lin::Arena ws{nullptr};
  Chain none{nullptr};
  f(*a, ws, false, pic::lin::Waits{}, none);
  return ws.used;
}

template <typename Args, typename F>
int run(const Args* a, F f, void* workspace, size_t bytes, void* stream) {
  const int64_t need = count_bytes(a, f);
  if (need < 0 || bytes < static_cast<size_t>(need)) return PIC_ERR_INVALID_ARG;
  if (need > 0 && (!workspace || !aligned(workspace, 256))) return PIC_ERR_INVALID_ARG;
  const int rc = pic::lin::device_status();
  if (rc != PIC_OK) return rc;
  pic::lin::Waits w;
  if (!pic::lin::call_waits(w)) return PIC_ERR_CUDA;
  pic::lin::Arena ws{static_cast<char*>(workspace)};
  Chain s{static_cast<cudaStream_t>(stream)};
  const int r = f(*a, ws, true, w, s);
  if (r == PIC_ERR_CUDA) cudaGetLastError();
  return r;
}

}  // namespace

extern "C" {

int64_t pic_grouped_linear_workspace_bytes(const pic_grouped_linear_args* a) { return count_bytes(a, forward); }

int pic_grouped_linear(const pic_grouped_linear_args* a, void* workspace, size_t workspace_bytes, void* stream) {
  return run(a, forward, workspace, workspace_bytes, stream);
}

int64_t pic_grouped_linear_backward_workspace_bytes(const pic_grouped_linear_grad_args* a) { return count_bytes(a, backward); }

int pic_grouped_linear_backward(const pic_grouped_linear_grad_args* a, void* workspace, size_t workspace_bytes, void* stream) {
  return run(a, backward, workspace, workspace_bytes, stream);
}

int pic_grouped_linear_check(void* stream) {
  // (after a timeout the offsets' word is left for the next check: one code tells of one)
  for (const int word : {0, 1}) {
    const int flag = pic::lin::take_status(word, static_cast<cudaStream_t>(stream));
    if (flag < 0) return PIC_ERR_CUDA;
    if (flag) return word == 0 ? PIC_ERR_TIMEOUT : PIC_ERR_INVALID_ARG;
  }
  return PIC_OK;
}

}  // extern "C"
