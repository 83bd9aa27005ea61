// C ABI shim: synchronous argument checks, then asynchronous launches.
#include <atomic>
#include <cstring>
#include <string>

#include "internal.hpp"
#include "launch.hpp"
#include "rows.hpp"

using namespace tbias;

namespace {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int check_arena(const tb_arena* a) {
  if (!a) return fail(TB_EINVAL, "arena is NULL");
  if (!a->base) return fail(TB_EINVAL, "arena base is NULL");
  if (!aligned(a->base, 256)) return fail(TB_EINVAL, "arena base not 256-byte aligned");
  const tb_arena_layout& L = a->layout;
  if (L.n_models < 1 || L.v_plus_blank < 2 || L.n_states < L.n_models || L.total_bytes <= 0)
    return fail(TB_EINVAL, "arena layout is not initialised");
  if (L.v_plus_blank > kMaxV1)
    return fail(TB_EINVAL, "v_plus_blank " + std::to_string(L.v_plus_blank) +
                               " exceeds the supported maximum " + std::to_string(kMaxV1));
  return TB_OK;
}

int hip_fail(hipError_t e, const char* what) {
  return fail(TB_EHIP, std::string(what) + ": " + hipGetErrorString(e));
}

int check_i32(const void* p, const char* name) {
  if (!p) return fail(TB_EINVAL, std::string(name) + " is NULL");
  if (!aligned(p, 4)) return fail(TB_EINVAL, std::string(name) + " not 4-byte aligned");
  return TB_OK;
}

int check_logits(const void* logits, int32_t dtype, int64_t row_stride, int32_t V1) {
  if (dtype != TB_F32 && dtype != TB_BF16) return fail(TB_EINVAL, "unknown dtype");
  if (!logits) return fail(TB_EINVAL, "logits is NULL");
  if (!aligned(logits, dtype == TB_F32 ? 4 : 2)) return fail(TB_EINVAL, "logits misaligned");
  if (row_stride < V1)
    return fail(TB_EINVAL, "row_stride " + std::to_string(row_stride) + " < V+1 = " +
                               std::to_string(V1));
  return TB_OK;
}

std::atomic<int32_t> g_greedy_kernel{kGreedyAuto};
std::atomic<int32_t> g_beam_kernel{kBeamAuto};
std::atomic<uint32_t> g_spin_limit{0u};

}  // namespace

namespace tbias {
int32_t debug_greedy_kernel() { return g_greedy_kernel.load(std::memory_order_relaxed); }
int32_t debug_beam_kernel() { return g_beam_kernel.load(std::memory_order_relaxed); }
uint32_t debug_spin_limit() { return g_spin_limit.load(std::memory_order_relaxed); }
}  // namespace tbias

extern "C" int tb_debug_select_kernels(int32_t greedy, int32_t beam) {
  if (greedy < kGreedyAuto || greedy > kGreedyRef) return fail(TB_EINVAL, "unknown greedy kernel");
  if (beam < kBeamAuto || beam > kBeamNoPipe) return fail(TB_EINVAL, "unknown beam kernel");
  g_greedy_kernel.store(greedy, std::memory_order_relaxed);
  g_beam_kernel.store(beam, std::memory_order_relaxed);
  return TB_OK;
}

extern "C" int tb_debug_set_spin_limit(uint32_t polls) {
  g_spin_limit.store(polls, std::memory_order_relaxed);
  return TB_OK;
}

extern "C" int tb_debug_launch_empty(int32_t grid, int32_t block, int32_t lds_bytes,
                                     void* hip_stream) {
  if (grid < 1 || block < 1 || block > 1024 || lds_bytes < 0 || lds_bytes > 160 * 1024)
    return fail(TB_EINVAL, "launch shape out of range");
  hipError_t e = launch_empty(grid, block, lds_bytes, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return hip_fail(e, "empty kernel launch");
  return TB_OK;
}

extern "C" int tb_graphs_upload(const tb_graphs* g, void* dev_base, int64_t bytes,
                                void* hip_stream, tb_arena* out) {
  if (!g || !dev_base || !out) return fail(TB_EINVAL, "NULL argument");
  if (!aligned(dev_base, 256)) return fail(TB_EINVAL, "dev_base not 256-byte aligned");
  if (bytes < g->layout.total_bytes) return fail(TB_ENOMEM, "device buffer too small");
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  hipError_t e = hipMemcpyAsync(dev_base, g->image.data(), (size_t)g->layout.total_bytes,
                                hipMemcpyHostToDevice, st);
  if (e != hipSuccess) return hip_fail(e, "hipMemcpyAsync");
  e = hipStreamSynchronize(st);
  if (e != hipSuccess) return hip_fail(e, "hipStreamSynchronize");
  out->base = dev_base;
  out->layout = g->layout;
  return TB_OK;
}

extern "C" int tb_init_states(const tb_arena* a, int32_t B, int32_t K, const int32_t* model_ids,
                              int32_t* states, float* scores, void* hip_stream) {
  int r;
  if ((r = check_arena(a))) return r;
  if (B < 1) return fail(TB_EINVAL, "B must be >= 1");
  if (K < 1 || K > TB_MAX_BEAM) return fail(TB_EINVAL, "K outside [1, TB_MAX_BEAM]");
  if ((r = check_i32(model_ids, "model_ids"))) return r;
  if ((r = check_i32(states, "states"))) return r;
  if (scores && !aligned(scores, 4)) return fail(TB_EINVAL, "scores not 4-byte aligned");
  hipError_t e = launch_init_states(make_view(*a), B, K, model_ids, states, scores,
                                    static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return hip_fail(e, "init_states launch");
  return TB_OK;
}

extern "C" int tb_init_beam_stream(const tb_arena* a, int32_t B, int32_t K,
                                   const int32_t* model_ids, int32_t* states, float* scores,
                                   tb_hyp* hyps, int32_t* tree_len, void* hip_stream) {
  int r;
  if ((r = check_arena(a))) return r;
  if (B < 1) return fail(TB_EINVAL, "B must be >= 1");
  if (K < 1 || K > TB_MAX_BEAM) return fail(TB_EINVAL, "K outside [1, TB_MAX_BEAM]");
  if ((r = check_i32(model_ids, "model_ids"))) return r;
  if ((r = check_i32(states, "states"))) return r;
  if ((r = check_i32(scores, "scores"))) return r;
  if ((r = check_i32(tree_len, "tree_len"))) return r;
  if (!hyps || !aligned(hyps, 8)) return fail(TB_EINVAL, "hyps NULL or not 8-byte aligned");
  hipError_t e = launch_init_beam_stream(make_view(*a), B, K, model_ids, states, scores, hyps,
                                         tree_len, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return hip_fail(e, "init_beam_stream launch");
  return TB_OK;
}

extern "C" int tb_reset_stream(const tb_arena* a, int32_t B, int32_t b, int32_t new_model_id,
                               int32_t K, int32_t* model_ids, int32_t* states, float* scores,
                               void* hip_stream) {
  int r;
  if ((r = check_arena(a))) return r;
  if (B < 1) return fail(TB_EINVAL, "B must be >= 1");
  if (b < 0 || b >= B) return fail(TB_EINVAL, "stream index outside [0, B)");
  if (K < 1 || K > TB_MAX_BEAM) return fail(TB_EINVAL, "K outside [1, TB_MAX_BEAM]");
  if (new_model_id < -1 || new_model_id >= a->layout.n_models)
    return fail(TB_ERANGE, "model id " + std::to_string(new_model_id) + " outside [-1, " +
                               std::to_string(a->layout.n_models) + ")");
  if ((r = check_i32(model_ids, "model_ids"))) return r;
  if ((r = check_i32(states, "states"))) return r;
  if (scores && !aligned(scores, 4)) return fail(TB_EINVAL, "scores not 4-byte aligned");
  hipError_t e = launch_reset_stream(b, new_model_id, K, model_ids, states, scores,
                                     static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return hip_fail(e, "reset_stream launch");
  return TB_OK;
}

extern "C" int tb_boost_step_greedy(const tb_arena* a, const void* logits, int32_t dtype,
                                    int32_t T, int32_t B, int64_t row_stride,
                                    const int32_t* model_ids, int32_t* states, int32_t* out_tok,
                                    int32_t* out_state, float* out_score, void* hip_stream) {
  int r;
  if ((r = check_arena(a))) return r;
  if (T < 0) return fail(TB_EINVAL, "T must be >= 0");
  if (B < 1) return fail(TB_EINVAL, "B must be >= 1");
  if (T == 0) return TB_OK;  // no-op: buffers are not touched (and may be NULL)
  if ((r = check_logits(logits, dtype, row_stride, a->layout.v_plus_blank))) return r;
  if ((r = check_i32(model_ids, "model_ids"))) return r;
  if ((r = check_i32(states, "states"))) return r;
  if ((r = check_i32(out_tok, "out_tok"))) return r;
  if ((r = check_i32(out_state, "out_state"))) return r;
  if ((r = check_i32(out_score, "out_score"))) return r;
  hipError_t e = launch_greedy(make_view(*a), logits, dtype, T, B, row_stride, model_ids, states,
                               out_tok, out_state, out_score,
                               static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return hip_fail(e, "greedy launch");
  return TB_OK;
}

extern "C" int tb_boost_step_beam(const tb_arena* a, const void* logits, int32_t dtype, int32_t T,
                                  int32_t B, int32_t K, int64_t row_stride,
                                  const int32_t* model_ids, int32_t* states, float* scores,
                                  int32_t* out_tok, int32_t* out_parent, int32_t* out_state,
                                  float* out_step, float* out_cum, void* hip_stream) {
  int r;
  if ((r = check_arena(a))) return r;
  if (T < 0) return fail(TB_EINVAL, "T must be >= 0");
  if (B < 1) return fail(TB_EINVAL, "B must be >= 1");
  if (K < 1 || K > TB_MAX_BEAM) return fail(TB_EINVAL, "K outside [1, TB_MAX_BEAM]");
  if (K > a->layout.v_plus_blank) return fail(TB_EINVAL, "K exceeds V+1");
  if (T == 0) return TB_OK;  // no-op: buffers are not touched (and may be NULL)
  if ((r = check_logits(logits, dtype, row_stride, a->layout.v_plus_blank))) return r;
  if ((r = check_i32(model_ids, "model_ids"))) return r;
  if ((r = check_i32(states, "states"))) return r;
  if ((r = check_i32(scores, "scores"))) return r;
  if ((r = check_i32(out_tok, "out_tok"))) return r;
  if ((r = check_i32(out_parent, "out_parent"))) return r;
  if ((r = check_i32(out_state, "out_state"))) return r;
  if ((r = check_i32(out_step, "out_step"))) return r;
  if ((r = check_i32(out_cum, "out_cum"))) return r;
  hipError_t e = launch_beam(make_view(*a), logits, dtype, T, B, K, row_stride, model_ids, states,
                             scores, out_tok, out_parent, out_state, out_step, out_cum,
                             static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return hip_fail(e, "beam launch");
  return TB_OK;
}

extern "C" int tb_boost_step_beam_stream(const tb_arena* a, const void* logits, int32_t dtype,
                                         int32_t T, int32_t B, int32_t K, int64_t row_stride,
                                         const int32_t* model_ids, int32_t* states, float* scores,
                                         tb_hyp* hyps, int32_t* tree, int32_t tree_cap,
                                         int32_t* tree_len, int32_t recombine, int32_t* out_tok,
                                         int32_t* out_parent, int32_t* out_state, float* out_step,
                                         float* out_cum, void* hip_stream) {
  int r;
  if ((r = check_arena(a))) return r;
  if (T < 0) return fail(TB_EINVAL, "T must be >= 0");
  if (B < 1) return fail(TB_EINVAL, "B must be >= 1");
  if (K < 1 || K > TB_MAX_BEAM) return fail(TB_EINVAL, "K outside [1, TB_MAX_BEAM]");
  if (K > a->layout.v_plus_blank) return fail(TB_EINVAL, "K exceeds V+1");
  if (tree_cap < 0) return fail(TB_EINVAL, "tree_cap must be >= 0");
  if (T == 0) return TB_OK;  // no-op: buffers are not touched (and may be NULL)
  if ((r = check_logits(logits, dtype, row_stride, a->layout.v_plus_blank))) return r;
  if ((r = check_i32(model_ids, "model_ids"))) return r;
  if ((r = check_i32(states, "states"))) return r;
  if ((r = check_i32(scores, "scores"))) return r;
  if ((r = check_i32(tree_len, "tree_len"))) return r;
  if (!hyps || !aligned(hyps, 8)) return fail(TB_EINVAL, "hyps NULL or not 8-byte aligned");
  if (tree_cap > 0 && (r = check_i32(tree, "tree"))) return r;
  if ((r = check_i32(out_tok, "out_tok"))) return r;
  if ((r = check_i32(out_parent, "out_parent"))) return r;
  if ((r = check_i32(out_state, "out_state"))) return r;
  if ((r = check_i32(out_step, "out_step"))) return r;
  if ((r = check_i32(out_cum, "out_cum"))) return r;
  hipError_t e = launch_beam_stream(make_view(*a), logits, dtype, T, B, K, row_stride, model_ids,
                                    states, scores, hyps, tree, tree_cap, tree_len, recombine,
                                    out_tok, out_parent, out_state, out_step, out_cum,
                                    static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return hip_fail(e, "streaming beam launch");
  return TB_OK;
}

// ---- row operators

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 40;  // sizes in bytes stay far from overflowing

// A buffer of a row operator.
struct RowBuf {
  const void* p;
  int64_t bytes;
  const char* name;
};

int check_rows(const void* logits, int32_t dtype, int64_t n_rows, int32_t v_plus_blank,
               int64_t row_stride, float temperature) {
  int r;
  if (v_plus_blank < 2 || v_plus_blank > TB_MAX_ROW)
    return fail(TB_EINVAL, "v_plus_blank " + std::to_string(v_plus_blank) + " outside [2, " +
                               std::to_string(TB_MAX_ROW) + "]");
  if ((r = check_logits(logits, dtype, row_stride, v_plus_blank))) return r;
  if (row_stride > INT64_MAX / 8 / n_rows) return fail(TB_EINVAL, "row_stride too large");
  if (!(temperature >= 1e-4f && temperature <= 1e4f))
    return fail(TB_EINVAL, "temperature outside [1e-4, 1e4]");
  return TB_OK;
}

int check_count(int64_t n_rows) {
  if (n_rows < 0 || n_rows > kMaxRows) return fail(TB_EINVAL, "n_rows outside [0, 2^40]");
  return TB_OK;
}

int check_list(int32_t n, const char* name) {
  if (n < 0 || n > TB_MAX_LIST)
    return fail(TB_EINVAL, std::string(name) + " outside [0, TB_MAX_LIST]");
  return TB_OK;
}

int check_opt(const void* p, const char* name) {
  if (p && !aligned(p, 4)) return fail(TB_EINVAL, std::string(name) + " not 4-byte aligned");
  return TB_OK;
}

int check_grad(const void* grad, int32_t dtype, int64_t n_rows, int64_t grad_stride, int32_t V1) {
  if (!aligned(grad, dtype == TB_F32 ? 4 : 2)) return fail(TB_EINVAL, "grad misaligned");
  if (grad_stride < V1)
    return fail(TB_EINVAL, "grad_stride " + std::to_string(grad_stride) + " < V+1 = " +
                               std::to_string(V1));
  if (grad_stride > INT64_MAX / 8 / n_rows) return fail(TB_EINVAL, "grad_stride too large");
  return TB_OK;
}

int64_t row_bytes(int64_t n_rows, int64_t stride, int32_t V1, int32_t dtype) {
  return ((n_rows - 1) * stride + V1) * (dtype == TB_F32 ? 4 : 2);
}

// The first n_out buffers are written: they may share memory with no other.
template <int N>
int check_apart(const RowBuf (&b)[N], int n_out) {
  for (int i = 0; i < n_out; ++i)
    for (int j = i + 1; j < N; ++j)
      if (b[i].p && b[j].p && b[i].bytes > 0 && b[j].bytes > 0 &&
          overlap({b[i].p, b[i].bytes}, {b[j].p, b[j].bytes}))
        return fail(TB_EINVAL, std::string(b[i].name) + " overlaps " + b[j].name);
  return TB_OK;
}

// The rows and their plan; workspace for rows in segments.
int make_rows(const void* logits, int32_t dtype, int64_t n_rows, int32_t V1, int64_t row_stride,
              float temperature, bool grad, int32_t n_alt, void* workspace,
              int64_t workspace_bytes, rows::Rows* a, rows::Plan* p) {
  *p = rows::plan(dtype, n_rows, V1, grad);
  const int64_t need = rows::workspace_bytes(*p, n_rows, n_alt);
  if (need > 0) {
    if (!workspace || workspace_bytes < need)
      return fail(TB_ENOMEM, "workspace holds " + std::to_string(workspace ? workspace_bytes : 0) +
                                 " bytes, the call needs " + std::to_string(need));
    if (!aligned(workspace, 16)) return fail(TB_EINVAL, "workspace not 16-byte aligned");
  }
  const double c = 1.4426950408889634 / (double)temperature;
  *a = {logits, row_stride, 0, n_rows, V1, p->n_seg, p->seg, (float)c,
        (float)(1.0 / (double)temperature), static_cast<float4*>(workspace)};
  return TB_OK;
}

}  // namespace

extern "C" int64_t tb_rows_workspace_bytes(int32_t dtype, int64_t n_rows, int32_t v_plus_blank,
                                           int32_t n_alt) {
  if ((dtype != TB_F32 && dtype != TB_BF16) || n_rows < 0 || n_rows > kMaxRows ||
      v_plus_blank < 2 ||
      v_plus_blank > TB_MAX_ROW || n_alt < 0 || n_alt > TB_MAX_LIST) {
    fail(TB_EINVAL, "bad dtype, n_rows, v_plus_blank or n_alt");
    return -1;
  }
  return rows::most_workspace(dtype, n_rows, v_plus_blank, n_alt);
}

extern "C" int tb_debug_rows_plan(int32_t dtype, int64_t n_rows, int32_t v_plus_blank,
                                  int32_t grad, int32_t out[3]) {
  if ((dtype != TB_F32 && dtype != TB_BF16) || n_rows < 1 || n_rows > kMaxRows ||
      v_plus_blank < 2 || v_plus_blank > TB_MAX_ROW || (grad != 0 && grad != 1) || !out)
    return fail(TB_EINVAL, "bad dtype, n_rows, v_plus_blank, grad or out");
  const rows::Plan p = rows::plan(dtype, n_rows, v_plus_blank, grad != 0);
  out[0] = rows::kShape[p.shape].nwr;
  out[1] = rows::kShape[p.shape].np;
  out[2] = p.n_seg;
  return TB_OK;
}

extern "C" int tb_token_logprobs(const void* logits, int32_t dtype, int64_t n_rows,
                                 int32_t v_plus_blank, int64_t row_stride, float temperature,
                                 const int32_t* tokens, int32_t n_tok, float* out_logprob,
                                 float* out_lse, float* out_entropy, int32_t n_alt,
                                 int32_t* out_alt, float* out_alt_logprob, void* workspace,
                                 int64_t workspace_bytes, void* hip_stream) {
  int r;
  if ((r = check_count(n_rows))) return r;
  if ((r = check_list(n_tok, "n_tok"))) return r;
  if ((r = check_list(n_alt, "n_alt"))) return r;
  if (n_rows == 0) return TB_OK;  // no-op: buffers are not touched (and may be NULL)
  if ((r = check_rows(logits, dtype, n_rows, v_plus_blank, row_stride, temperature))) return r;
  if (n_tok > 0 && (r = check_i32(tokens, "tokens"))) return r;
  if (n_tok > 0 && (r = check_i32(out_logprob, "out_logprob"))) return r;
  if ((r = check_opt(out_lse, "out_lse"))) return r;
  if ((r = check_opt(out_entropy, "out_entropy"))) return r;
  if (n_alt > 0 && (r = check_i32(out_alt, "out_alt"))) return r;
  if (n_alt > 0 && (r = check_i32(out_alt_logprob, "out_alt_logprob"))) return r;
  rows::Rows a;
  rows::Plan p;
  if ((r = make_rows(logits, dtype, n_rows, v_plus_blank, row_stride, temperature, false, n_alt,
                     workspace, workspace_bytes, &a, &p)))
    return r;
  const int64_t part = rows::workspace_bytes(p, n_rows, 0);
  const RowBuf bufs[] = {{n_tok ? out_logprob : nullptr, n_rows * n_tok * 4, "out_logprob"},
                         {out_lse, n_rows * 4, "out_lse"},
                         {out_entropy, n_rows * 4, "out_entropy"},
                         {n_alt ? out_alt : nullptr, n_rows * n_alt * 4, "out_alt"},
                         {n_alt ? out_alt_logprob : nullptr, n_rows * n_alt * 4, "out_alt_logprob"},
                         {workspace, rows::workspace_bytes(p, n_rows, n_alt), "workspace"},
                         {logits, row_bytes(n_rows, row_stride, v_plus_blank, dtype), "logits"},
                         {n_tok ? tokens : nullptr, n_rows * n_tok * 4, "tokens"}};
  if ((r = check_apart(bufs, 6))) return r;
  const rows::ScoreIO io = {tokens, n_tok, out_logprob, out_lse, out_entropy, n_alt, out_alt,
                            out_alt_logprob,
                            reinterpret_cast<int2*>(static_cast<unsigned char*>(workspace) + part)};
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  hipError_t e = dtype == TB_F32 ? rows::score_f32(a, io, p, st) : rows::score_bf16(a, io, p, st);
  if (e != hipSuccess) return hip_fail(e, "token_logprobs launch");
  return TB_OK;
}

extern "C" int tb_token_logprobs_grad(const void* logits, int32_t dtype, int64_t n_rows,
                                      int32_t v_plus_blank, int64_t row_stride, float temperature,
                                      const int32_t* tokens, int32_t n_tok,
                                      const float* d_logprob, const float* d_lse,
                                      const float* d_entropy, void* grad, int64_t grad_stride,
                                      void* workspace, int64_t workspace_bytes,
                                      void* hip_stream) {
  int r;
  if ((r = check_count(n_rows))) return r;
  if ((r = check_list(n_tok, "n_tok"))) return r;
  if (n_rows == 0) return TB_OK;  // no-op: buffers are not touched (and may be NULL)
  if ((r = check_rows(logits, dtype, n_rows, v_plus_blank, row_stride, temperature))) return r;
  if (n_tok > 0 && (r = check_i32(tokens, "tokens"))) return r;
  if (n_tok > 0 && (r = check_i32(d_logprob, "d_logprob"))) return r;
  if ((r = check_opt(d_lse, "d_lse"))) return r;
  if ((r = check_opt(d_entropy, "d_entropy"))) return r;
  if (!grad) return fail(TB_EINVAL, "grad is NULL");
  if ((r = check_grad(grad, dtype, n_rows, grad_stride, v_plus_blank))) return r;
  rows::Rows a;
  rows::Plan p;
  if ((r = make_rows(logits, dtype, n_rows, v_plus_blank, row_stride, temperature, true, 0,
                     workspace, workspace_bytes, &a, &p)))
    return r;
  const bool in_place = grad == logits && grad_stride == row_stride;
  const RowBuf bufs[] = {
      {grad, row_bytes(n_rows, grad_stride, v_plus_blank, dtype), "grad"},
      {workspace, rows::workspace_bytes(p, n_rows, 0), "workspace"},
      {in_place ? nullptr : logits, row_bytes(n_rows, row_stride, v_plus_blank, dtype), "logits"},
      {n_tok ? tokens : nullptr, n_rows * n_tok * 4, "tokens"},
      {n_tok ? d_logprob : nullptr, n_rows * n_tok * 4, "d_logprob"},
      {d_lse, n_rows * 4, "d_lse"},
      {d_entropy, n_rows * 4, "d_entropy"}};
  if ((r = check_apart(bufs, 2))) return r;
  const rows::GradIO io = {tokens, n_tok, d_logprob, d_lse, d_entropy, grad, grad_stride};
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  hipError_t e = dtype == TB_F32 ? rows::grad_f32(a, io, p, st) : rows::grad_bf16(a, io, p, st);
  if (e != hipSuccess) return hip_fail(e, "token_logprobs_grad launch");
  return TB_OK;
}

extern "C" int tb_distill(const void* logits, int32_t dtype, int64_t n_rows, int32_t v_plus_blank,
                          int64_t row_stride, float temperature, const int32_t* teacher_tok,
                          const float* teacher_score, int32_t n_teacher, int32_t tail,
                          const float* weight, float* out_loss, void* grad, int64_t grad_stride,
                          void* workspace, int64_t workspace_bytes, void* hip_stream) {
  int r;
  if ((r = check_count(n_rows))) return r;
  if (n_teacher < 1 || n_teacher > TB_MAX_LIST)
    return fail(TB_EINVAL, "n_teacher outside [1, TB_MAX_LIST]");
  if (tail != 0 && tail != 1) return fail(TB_EINVAL, "tail must be 0 or 1");
  if (n_rows == 0) return TB_OK;  // no-op: buffers are not touched (and may be NULL)
  if ((r = check_rows(logits, dtype, n_rows, v_plus_blank, row_stride, temperature))) return r;
  if ((r = check_i32(teacher_tok, "teacher_tok"))) return r;
  if ((r = check_i32(teacher_score, "teacher_score"))) return r;
  if ((r = check_opt(weight, "weight"))) return r;
  if ((r = check_opt(out_loss, "out_loss"))) return r;
  if (!out_loss && !grad) return fail(TB_EINVAL, "out_loss and grad are both NULL");
  if (grad && (r = check_grad(grad, dtype, n_rows, grad_stride, v_plus_blank))) return r;
  rows::Rows a;
  rows::Plan p;
  if ((r = make_rows(logits, dtype, n_rows, v_plus_blank, row_stride, temperature, grad != nullptr,
                     0, workspace, workspace_bytes, &a, &p)))
    return r;
  const bool in_place = grad == logits && grad_stride == row_stride;
  const RowBuf bufs[] = {
      {grad, grad ? row_bytes(n_rows, grad_stride, v_plus_blank, dtype) : 0, "grad"},
      {out_loss, n_rows * 4, "out_loss"},
      {workspace, rows::workspace_bytes(p, n_rows, 0), "workspace"},
      {in_place ? nullptr : logits, row_bytes(n_rows, row_stride, v_plus_blank, dtype), "logits"},
      {teacher_tok, n_rows * n_teacher * 4, "teacher_tok"},
      {teacher_score, n_rows * n_teacher * 4, "teacher_score"},
      {weight, n_rows * 4, "weight"}};
  if ((r = check_apart(bufs, 3))) return r;
  const rows::DistillIO io = {teacher_tok, teacher_score, n_teacher, tail, weight, out_loss,
                              grad, grad_stride};
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  hipError_t e =
      dtype == TB_F32 ? rows::distill_f32(a, io, p, st) : rows::distill_bf16(a, io, p, st);
  if (e != hipSuccess) return hip_fail(e, "distill launch");
  return TB_OK;
}
