// C ABI of the output layer's training operators: argument checks, then launches.
#include <algorithm>
#include <cmath>
#include <new>
#include <string>
#include <vector>

#include "adamw.hpp"
#include "internal.hpp"
#include "linear.hpp"

using namespace tbias;

namespace {

constexpr int64_t kMostRows = (int64_t)1 << 24, kMostValues = (int64_t)1 << 36;
constexpr int32_t kMostWidth = 1 << 16;

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

int hip_fail(hipError_t e, const char* what) {
  return fail(TB_EHIP, std::string(what) + ": " + hipGetErrorString(e));
}

struct Buf {
  const void* p;
  int64_t bytes;
  const char* name;
};

// The first n_out buffers are written: they may share memory with no other.
template <int N>
int check_apart(const Buf (&b)[N], int n_out) {
  for (int i = 0; i < n_out; ++i)
    for (int j = i + 1; j < N; ++j)
      if (b[i].p && b[j].p && b[i].bytes > 0 && b[j].bytes > 0 &&
          overlap({b[i].p, b[i].bytes}, {b[j].p, b[j].bytes}))
        return fail(TB_EINVAL, std::string(b[i].name) + " overlaps " + b[j].name);
  return TB_OK;
}

int check_sizes(int32_t dtype, int64_t n_rows, int32_t width, int32_t v_plus_blank,
                int64_t w_stride) {
  if (dtype != TB_F32 && dtype != TB_BF16) return fail(TB_EINVAL, "unknown dtype");
  if (n_rows < 0 || n_rows > kMostRows) return fail(TB_EINVAL, "n_rows outside [0, 2^24]");
  if (width < 1 || width > kMostWidth) return fail(TB_EINVAL, "width outside [1, 2^16]");
  if (v_plus_blank < 2 || v_plus_blank > TB_MAX_ROW)
    return fail(TB_EINVAL, "v_plus_blank " + std::to_string(v_plus_blank) + " outside [2, " +
                               std::to_string(TB_MAX_ROW) + "]");
  if (w_stride < width || w_stride > ((int64_t)1 << 30))
    return fail(TB_EINVAL, "w_stride outside [width, 2^30]");
  return TB_OK;
}

int check_matrix(const void* p, int32_t dtype, int64_t stride, int32_t width, const char* name) {
  if (!aligned(p, dtype == TB_F32 ? 4 : 2)) return fail(TB_EINVAL, std::string(name) + " misaligned");
  if (stride < width || stride > ((int64_t)1 << 30))
    return fail(TB_EINVAL, std::string(name) + "_stride outside [width, 2^30]");
  return TB_OK;
}

int check_four(const void* p, const char* name, bool needed) {
  if (!p && needed) return fail(TB_EINVAL, std::string(name) + " is NULL");
  if (p && !aligned(p, 4)) return fail(TB_EINVAL, std::string(name) + " not 4-byte aligned");
  return TB_OK;
}

int linear_call(const linear::Call& c, void* workspace, int64_t workspace_bytes, void* hip_stream,
                const char* what) {
  int r;
  if ((r = check_sizes(c.dtype, c.n, c.D, c.C, c.w_stride))) return r;
  const bool any = c.n > 0;  // without rows only dw and db are touched
  if (any && !c.x) return fail(TB_EINVAL, "x is NULL");
  if (any && (r = check_matrix(c.x, c.dtype, c.x_stride, c.D, "x"))) return r;
  if (any && !c.w) return fail(TB_EINVAL, "w is NULL");
  if (any && (r = check_matrix(c.w, c.dtype, c.w_stride, c.D, "w"))) return r;
  const int64_t size = c.dtype == TB_F32 ? 4 : 2;
  if (c.bias && !aligned(c.bias, size)) return fail(TB_EINVAL, "bias misaligned");
  if ((r = check_four(c.target, "target", any))) return r;
  if ((r = check_four(c.weight, "weight", false))) return r;
  if ((r = check_four(c.d_loss, "d_loss", false))) return r;
  if ((r = check_four(c.d_lse, "d_lse", false))) return r;
  if ((r = check_four(c.lse, "lse", false))) return r;
  if ((r = check_four(c.out_loss, "out_loss", false))) return r;
  if ((r = check_four(c.lse_low, "lse_low", false))) return r;
  if ((r = check_four(c.out_lse, "out_lse", false))) return r;
  if ((r = check_four(c.out_low, "out_low", false))) return r;
  if (c.dx && any && (r = check_matrix(c.dx, c.dtype, c.dx_stride, c.D, "dx"))) return r;
  if (c.dw && (r = check_matrix(c.dw, c.dtype, c.dw_stride, c.D, "dw"))) return r;
  if (c.db && !aligned(c.db, size)) return fail(TB_EINVAL, "db misaligned");
  if (!any && !c.dw && !c.db) return TB_OK;
  const linear::Layout plan = linear::plan(c);
  const int64_t need = plan.total;
  if (!workspace || workspace_bytes < need)
    return fail(TB_ENOMEM, "workspace holds " + std::to_string(workspace ? workspace_bytes : 0) +
                               " bytes, the call needs " + std::to_string(need));
  if (!aligned(workspace, 256)) return fail(TB_EINVAL, "workspace not 256-byte aligned");
  auto rows = [&](int64_t n, int64_t stride) {
    return n > 0 ? ((n - 1) * stride + c.D) * size : 0;
  };
  const Buf bufs[] = {{c.out_loss, c.n * 4, "out_loss"},
                      {c.out_lse, c.n * 4, "out_lse"},
                      {c.out_low, c.n * 4, "out_low"},
                      {c.dx, rows(c.n, c.dx_stride), "dx"},
                      {c.dw, rows(c.C, c.dw_stride), "dw"},
                      {c.db, c.C * size, "db"},
                      {workspace, need, "workspace"},
                      {c.x, rows(c.n, c.x_stride), "x"},
                      {c.w, rows(c.C, c.w_stride), "w"},
                      {c.bias, c.C * size, "bias"},
                      {c.target, c.n * 4, "target"},
                      {c.weight, c.n * 4, "weight"},
                      {c.lse, c.n * 4, "lse"},
                      {c.lse_low, c.n * 4, "lse_low"},
                      {c.d_loss, c.d_step ? c.n * 4 : 4, "d_loss"},
                      {c.d_lse, c.n * 4, "d_lse"}};
  if ((r = check_apart(bufs, 7))) return r;
  const hipError_t e = linear::run(c, plan, workspace, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return hip_fail(e, what);
  return TB_OK;
}

}  // namespace

extern "C" int64_t tb_linear_xent_workspace_bytes(int32_t dtype, int64_t n_rows, int32_t width,
                                                  int32_t v_plus_blank, const void* w,
                                                  int64_t w_stride, int32_t grads,
                                                  int32_t with_lse) {
  if (check_sizes(dtype, n_rows, width, v_plus_blank, w_stride)) return -1;
  if (grads < 0 || grads > 7 || with_lse < 0 || with_lse > 1) {
    fail(TB_EINVAL, "grads outside [0, 7] or with_lse not 0 or 1");
    return -1;
  }
  linear::Call c = {};
  c.w = w;
  c.dtype = dtype;
  c.n = n_rows;
  c.D = width;
  c.C = v_plus_blank;
  c.w_stride = w_stride;
  // (not dereferenced: which results are asked for, and whether lse is there)
  static float some;
  c.lse = with_lse ? &some : nullptr;
  c.dx = grads & 1 ? &some : nullptr;
  c.dw = grads & 2 ? &some : nullptr;
  c.db = grads & 4 ? &some : nullptr;
  return linear::most_workspace(c);
}

extern "C" int tb_linear_xent(const void* x, const void* w, const void* bias, int32_t dtype,
                              int64_t n_rows, int32_t width, int32_t v_plus_blank,
                              int64_t x_stride, int64_t w_stride, const int32_t* target,
                              const float* weight, float* out_loss, float* out_lse,
                              float* out_low, void* dx, int64_t dx_stride, void* dw,
                              int64_t dw_stride, void* db,
                              void* workspace, int64_t workspace_bytes, void* hip_stream) {
  if (n_rows > 0 && !out_loss && !out_lse && !out_low && !dx && !dw && !db)
    return fail(TB_EINVAL, "every output is NULL");
  const linear::Call c = {x,      w,      bias,    dtype,   n_rows,   width,   v_plus_blank,
                          x_stride, w_stride, target, weight, nullptr, nullptr, 0, nullptr, nullptr,
                          out_loss, out_lse, out_low, dx, dw, db, dx_stride, dw_stride};
  return linear_call(c, workspace, workspace_bytes, hip_stream, "linear_xent launch");
}

extern "C" int tb_linear_xent_grad(const void* x, const void* w, const void* bias, int32_t dtype,
                                   int64_t n_rows, int32_t width, int32_t v_plus_blank,
                                   int64_t x_stride, int64_t w_stride, const int32_t* target,
                                   const float* weight, const float* lse, const float* lse_low,
                                   const float* d_loss, int32_t d_loss_step,
                                   const float* d_lse, void* dx, int64_t dx_stride, void* dw,
                                   int64_t dw_stride, void* db, void* workspace,
                                   int64_t workspace_bytes, void* hip_stream) {
  if (n_rows > 0 && !dx && !dw && !db) return fail(TB_EINVAL, "dx, dw and db are all NULL");
  if (!lse && n_rows > 0) return fail(TB_EINVAL, "lse is NULL");
  if (d_loss_step != 0 && d_loss_step != 1) return fail(TB_EINVAL, "d_loss_step must be 0 or 1");
  static const float none = 0.f;  // (without rows nothing reads it)
  const linear::Call c = {x,      w,      bias,    dtype,   n_rows,   width,   v_plus_blank,
                          x_stride, w_stride, target, weight, d_loss, d_lse, d_loss_step,
                          lse ? lse : &none, lse_low,
                          nullptr, nullptr, nullptr, dx, dw, db, dx_stride, dw_stride};
  return linear_call(c, workspace, workspace_bytes, hip_stream, "linear_xent_grad launch");
}

// ---- AdamW

namespace {

struct Span8 {
  uintptr_t begin, end;
  int32_t tensor;
  bool written;
};

// No written buffer may share memory with another: neighbours in the order of their
// addresses tell.
int check_spans(std::vector<Span8>& s) {
  std::sort(s.begin(), s.end(), [](const Span8& a, const Span8& b) {
    return a.begin != b.begin ? a.begin < b.begin : a.end < b.end;
  });
  // furthest ends so far, of written buffers and of all
  uintptr_t written = 0, any = 0;
  for (const Span8& x : s) {
    if (x.begin < written || (x.written && x.begin < any))
      return fail(TB_EINVAL, "a buffer of tensor " + std::to_string(x.tensor) +
                                 " shares memory with another that is written");
    any = std::max(any, x.end);
    if (x.written) written = std::max(written, x.end);
  }
  return TB_OK;
}

int check_tensor(const tb_adamw_tensor& t, int32_t i) {
  if (t.n < 0 || t.n > kMostValues)
    return fail(TB_EINVAL, "tensor " + std::to_string(i) + ": n outside [0, 2^36]");
  return TB_OK;
}

int bad_buffer(int32_t i, const char* name) {
  return fail(TB_EINVAL,
              "tensor " + std::to_string(i) + ": " + name + " is NULL or not aligned to its type");
}

}  // namespace

extern "C" int tb_adamw_step(const tb_adamw_tensor* tensors, int32_t n_tensors, int32_t dtype,
                             int32_t state_bits, double lr, double beta1, double beta2, double eps,
                             double weight_decay, int64_t step, const float* lr_dev,
                             const int64_t* step_dev, const float* grad_scale, uint32_t seed,
                             void* hip_stream) try {
  int r;
  if (n_tensors < 0 || (n_tensors > 0 && !tensors)) return fail(TB_EINVAL, "bad tensors");
  if (dtype != TB_F32 && dtype != TB_BF16) return fail(TB_EINVAL, "unknown dtype");
  if (state_bits != 32 && state_bits != 8) return fail(TB_EINVAL, "state_bits must be 32 or 8");
  if (!(lr >= 0) || !std::isfinite(lr) || !(weight_decay >= 0) || !std::isfinite(weight_decay) ||
      !(eps >= 0) || !std::isfinite(eps))
    return fail(TB_EINVAL, "lr, weight_decay and eps must be finite and not negative");
  if (!(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1))
    return fail(TB_EINVAL, "beta1 and beta2 must be in [0, 1)");
  if (step < 1) return fail(TB_EINVAL, "step must be at least 1");
  if ((r = check_four(lr_dev, "lr_dev", false))) return r;
  if (step_dev && !aligned(step_dev, 8)) return fail(TB_EINVAL, "step_dev not 8-byte aligned");
  if ((r = check_four(grad_scale, "grad_scale", false))) return r;
  const int64_t size = dtype == TB_F32 ? 4 : 2, state = state_bits == 32 ? 4 : 1;
  std::vector<Span8> spans;
  spans.reserve((size_t)n_tensors * 7 + 3);
  bool some = false, master = false;
  for (int32_t i = 0; i < n_tensors; ++i) {
    const tb_adamw_tensor& t = tensors[i];
    if ((r = check_tensor(t, i))) return r;
    if (t.n == 0) continue;
    if (!t.param || !aligned(t.param, size)) return bad_buffer(i, "param");
    if (!t.grad || !aligned(t.grad, size)) return bad_buffer(i, "grad");
    if (!t.m || !aligned(t.m, state)) return bad_buffer(i, "m");
    if (!t.v || !aligned(t.v, state)) return bad_buffer(i, "v");
    if (state == 1 && (!t.m_unit || !aligned(t.m_unit, 4))) return bad_buffer(i, "m_unit");
    if (state == 1 && (!t.v_unit || !aligned(t.v_unit, 4))) return bad_buffer(i, "v_unit");
    if (t.master && (dtype != TB_BF16 || !aligned(t.master, 4)))
      return fail(TB_EINVAL, "tensor " + std::to_string(i) +
                                 ": master copies are float32 and of bfloat16 parameters");
    if (some && master != (t.master != nullptr))
      return fail(TB_EINVAL, "master copies of some tensors only");
    some = true;
    master = t.master != nullptr;
    auto add = [&](const void* p, int64_t bytes, bool written) {
      const uintptr_t b = reinterpret_cast<uintptr_t>(p);
      spans.push_back({b, b + (uintptr_t)bytes, i, written});
    };
    add(t.param, t.n * size, true);
    add(t.grad, t.n * size, false);
    add(t.m, t.n * state, true);
    add(t.v, t.n * state, true);
    if (state == 1) {
      add(t.m_unit, (t.n + 255) / 256 * 4, true);
      add(t.v_unit, (t.n + 255) / 256 * 4, true);
    }
    if (t.master) add(t.master, t.n * 4, true);
  }
  if (!some) return TB_OK;
  auto scalar = [&](const void* p, uintptr_t bytes) {
    const uintptr_t b = reinterpret_cast<uintptr_t>(p);
    if (p) spans.push_back({b, b + bytes, -1, false});
  };
  scalar(lr_dev, 4);
  scalar(step_dev, 8);
  scalar(grad_scale, 4);
  if ((r = check_spans(spans))) return r;
  const adamw::Step s = {dtype,  state_bits, master,   lr,         beta1, beta2, eps, weight_decay,
                         step, lr_dev, step_dev, grad_scale, seed};
  const hipError_t e = adamw::step(tensors, n_tensors, s, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return hip_fail(e, "adamw_step launch");
  return TB_OK;
} catch (const std::bad_alloc&) {
  return fail(TB_ENOMEM, "out of host memory");
}

extern "C" int tb_adamw_moments(const tb_adamw_tensor* tensors, int32_t n_tensors,
                                float* const* out_m, float* const* out_v, void* hip_stream) try {
  int r;
  if (n_tensors < 0 || (n_tensors > 0 && (!tensors || !out_m || !out_v)))
    return fail(TB_EINVAL, "bad tensors, out_m or out_v");
  std::vector<Span8> spans;
  spans.reserve((size_t)n_tensors * 6);
  for (int32_t i = 0; i < n_tensors; ++i) {
    const tb_adamw_tensor& t = tensors[i];
    if ((r = check_tensor(t, i))) return r;
    if (t.n == 0) continue;
    if (!t.m) return bad_buffer(i, "m");
    if (!t.v) return bad_buffer(i, "v");
    if (!t.m_unit || !aligned(t.m_unit, 4)) return bad_buffer(i, "m_unit");
    if (!t.v_unit || !aligned(t.v_unit, 4)) return bad_buffer(i, "v_unit");
    if (!out_m[i] || !aligned(out_m[i], 4)) return bad_buffer(i, "out_m");
    if (!out_v[i] || !aligned(out_v[i], 4)) return bad_buffer(i, "out_v");
    auto add = [&](const void* p, int64_t bytes, bool written) {
      const uintptr_t b = reinterpret_cast<uintptr_t>(p);
      spans.push_back({b, b + (uintptr_t)bytes, i, written});
    };
    add(t.m, t.n, false);
    add(t.v, t.n, false);
    add(t.m_unit, (t.n + 255) / 256 * 4, false);
    add(t.v_unit, (t.n + 255) / 256 * 4, false);
    add(out_m[i], t.n * 4, true);
    add(out_v[i], t.n * 4, true);
  }
  if ((r = check_spans(spans))) return r;
  const hipError_t e =
      adamw::moments(tensors, n_tensors, out_m, out_v, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return hip_fail(e, "adamw_moments launch");
  return TB_OK;
} catch (const std::bad_alloc&) {
  return fail(TB_ENOMEM, "out of host memory");
}
