// Cross entropy of a linear layer without its logits (linear.hpp): gathering of the
// rows, what joins the tiles' results, and the launches of a call.
#include "linear_gemm.hpp"

namespace tbias {
namespace linear {

namespace {

// ---- the rows that take part

struct Gather {
  int64_t n;
  int32_t C;
  const int32_t* target;
  const float *weight, *d_loss, *d_lse, *lse;
  int32_t grads, rows_up;  // rows_up: gathered rows there is room for
  Meta* meta;
  int32_t *idx, *inv, *tgt;
  float *a, *b, *lse_c;
  float *out_loss, *out_lse;
};

constexpr int kRowsEach = 8;  // rows of a thread at a time

// One workgroup: order and arguments of the rows that take part. 16 rows cost about as
// much as one, so 16,384 rows take two rounds.
__global__ void __launch_bounds__(1024) gather_kernel(const Gather g) {
  __shared__ int32_t sums[16];
  __shared__ float tops[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int32_t before = 0;
  float top = 0.f;
  for (int64_t r0 = 0; r0 < g.n; r0 += 1024 * kRowsEach) {
    const int64_t first = r0 + (int64_t)threadIdx.x * kRowsEach;
    int32_t t[kRowsEach];
    float a[kRowsEach], b[kRowsEach], l[kRowsEach];
    int32_t mine = 0;
#pragma unroll
    for (int e = 0; e < kRowsEach; ++e) {
      const int64_t r = first + e;
      const bool in = r < g.n;
      t[e] = in ? g.target[r] : -1;
      const float w = in && g.weight ? g.weight[r] : 1.f;
      b[e] = w;
      a[e] = w;
      l[e] = 0.f;
      bool keep = t[e] != -1 && w != 0.f;
      if (g.grads) {
        if (in && g.d_loss) b[e] = w * g.d_loss[r];
        a[e] = b[e] + (in && g.d_lse ? g.d_lse[r] : 0.f);
        if (in && g.lse) l[e] = g.lse[r];
        // a row without a gradient is left out, unless its loss is asked for
        if (g.lse) keep = keep && (a[e] != 0.f || b[e] != 0.f);
      }
      if (keep && (uint32_t)t[e] >= (uint32_t)g.C) {
        t[e] = -2;
        a[e] = b[e] = __builtin_nanf("");
      }
      if (!keep) t[e] = -1;
      mine += t[e] != -1;
    }
    int32_t upto = mine;  // of this wave's lanes up to this one
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int32_t v = __shfl_up(upto, d);
      if (lane >= d) upto += v;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int32_t at = before + upto - mine, all = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      if (w < wave) at += sums[w];
      all += sums[w];
    }
    before += all;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kRowsEach; ++e) {
      const int64_t r = first + e;
      if (r >= g.n) break;
      if (t[e] == -1) {
        g.inv[r] = -1;
        if (g.out_loss) g.out_loss[r] = 0.f;
        if (g.out_lse) g.out_lse[r] = 0.f;
        continue;
      }
      // an empty row (no token above -inf) has no gradient
      if (l[e] == -__builtin_huge_valf()) a[e] = b[e] = l[e] = 0.f;
      g.inv[r] = at;
      g.idx[at] = (int32_t)r;
      g.tgt[at] = t[e];
      g.a[at] = a[e];
      g.b[at] = b[e];
      g.lse_c[at] = l[e];
      if (fabsf(a[e]) < __builtin_huge_valf()) top = fmaxf(top, fabsf(a[e]));
      if (fabsf(b[e]) < __builtin_huge_valf()) top = fmaxf(top, fabsf(b[e]));
      ++at;
    }
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 0; w < 16; ++w) top = fmaxf(top, tops[w]);
    // (no further, so that rows of far smaller weights keep their place in float32)
    top = fminf(fmaxf(top, 0x1p-24f), 0x1p24f);
    *g.meta = {before, top, 1.f / top};
  }
}

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

// Rows of a matrix as planes, padded with zeros to dp values: the gathered rows idx
// and zeros up to a multiple of kTile, or (idx NULL) all n of them.
template <class T>
__global__ void __launch_bounds__(256)
    planes_kernel(const T* x, int64_t stride, int32_t D, int32_t dp, const int32_t* idx,
                  const Meta* meta, int64_t n, uint16_t* out, int64_t plane) {
  constexpr int PLANES = sizeof(T) == 4 ? 3 : 1;
  const int64_t each = dp / 4;
  const int64_t have = idx ? meta->n : n, rows = idx ? up(have, kTile) : n;
  const bool whole = (stride * sizeof(T)) % 16 == 0 && (uintptr_t)x % 16 == 0;
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < rows * each;
       at += (int64_t)gridDim.x * 256) {
    const int64_t row = at / each;
    const int d = (int)(at - row * each) * 4;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (row < have) {
      const T* from = x + (idx ? (int64_t)idx[row] : row) * stride + d;
      if (whole && d + 4 <= D) {
        if constexpr (sizeof(T) == 4) {
          const float4 q = *reinterpret_cast<const float4*>(from);
          v[0] = q.x;
          v[1] = q.y;
          v[2] = q.z;
          v[3] = q.w;
        } else {
          const uint2 q = *reinterpret_cast<const uint2*>(from);
          v[0] = low16(q.x);
          v[1] = high16(q.x);
          v[2] = low16(q.y);
          v[3] = high16(q.y);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (d + e < D) v[e] = widen(from[e]);
      }
    }
    uint2 p[PLANES];
    planes4<PLANES>(v, p);
#pragma unroll
    for (int s = 0; s < PLANES; ++s)
      *reinterpret_cast<uint2*>(out + s * plane + row * dp + d) = p[s];
  }
}

// ---- what joins the tiles

// One wave a gathered row: log-sum-exp and loss.
struct Finish {
  const Meta* meta;
  const float2* part;
  int32_t n_part;
  const float* hit;
  const int32_t *idx, *tgt;
  const float* weight;
  float *lse_c, *a, *b;
  float *out_loss, *out_lse;
};

__global__ void __launch_bounds__(256) finish_kernel(const Finish f) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= f.meta->n) return;
  const float2* part = f.part + row * f.n_part;
  float m = -__builtin_huge_valf();
  for (int i = lane; i < f.n_part; i += 64) m = fmaxf(m, part[i].x);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  const float base = m == -__builtin_huge_valf() ? 0.f : m;
  float sum = 0.f;
  for (int i = lane; i < f.n_part; i += 64) {
    const float2 v = part[i];
    // (a part without a value has maximum -inf and sum 0; a NaN in either stays)
    sum += v.y * __builtin_amdgcn_exp2f((v.x - base) * kLog2e);
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
  if (lane != 0) return;
  const float lse = base + logf(sum);
  const int64_t r = f.idx[row];
  if (f.out_lse) f.out_lse[r] = lse;
  if (f.out_loss) {
    const float hit = f.tgt[row] < 0 ? __builtin_nanf("") : f.hit[row];
    const float nll = lse == -__builtin_huge_valf() && hit == lse ? __builtin_huge_valf() : lse - hit;
    f.out_loss[r] = f.weight ? f.weight[r] * nll : nll;
  }
  if (lse == -__builtin_huge_valf()) {
    f.lse_c[row] = 0.f;
    f.a[row] = f.b[row] = 0.f;
  } else {
    f.lse_c[row] = lse;
  }
}

template <class T>
__device__ __forceinline__ void store_row4(T* o, const float* v, int left) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < left) store_out(o + e, v[e]);
}

// out[r] = scale * the sum of the splits' rows inv[r] (or r); 0 for the rows left out.
template <class T>
__global__ void __launch_bounds__(256)
    join_kernel(const float* acc, int64_t split, int32_t splits, int32_t lda, const int32_t* inv,
                const Meta* meta, T* out, int64_t ldo, int64_t n, int32_t D) {
  const int64_t each = (D + 3) / 4;
  const float scale = meta->scale;
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < n * each;
       at += (int64_t)gridDim.x * 256) {
    const int64_t row = at / each;
    const int d = (int)(at - row * each) * 4;
    const int64_t from = inv ? inv[row] : row;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (from >= 0) {
      const float* p = acc + from * lda + d;
      for (int s = 0; s < splits; ++s) v += *reinterpret_cast<const f32x4*>(p + s * split);
    }
    const float w[4] = {v[0] * scale, v[1] * scale, v[2] * scale, v[3] * scale};
    store_row4(out + row * ldo + d, w, D - d);
  }
}

// db[c] = scale * the sum of the row groups' columns.
template <class T>
__global__ void __launch_bounds__(256)
    columns_kernel(const float* col, int32_t ldg, const Meta* meta, T* db, int32_t n) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= n) return;
  const int groups = (int)up(meta->n, kTile) / 64;
  float sum = 0.f;
  for (int q = 0; q < groups; ++q) sum += col[(int64_t)q * ldg + c];
  store_out(db + c, sum * meta->scale);
}

// ---- workspace

constexpr int64_t kGradBytes = 256ll << 20;  // of the gradients of a piece's logits

struct Layout {
  int64_t np, dp, planes;      // gathered rows and values a row, rounded up
  bool copy_w;
  int32_t n_part;
  int32_t piece, pieces;       // tokens of a piece of the vocabulary
  int32_t split_x, split_w;
  int64_t meta, idx, inv, tgt, a, b, lse, hit, part, x, w, G, acc_x, acc_w, col, total;
};

int splits(int64_t tiles, int64_t steps) {
  // enough workgroups for every CU, each with a few steps
  int64_t s = tiles < 1 || tiles >= 160 ? 1 : (256 + tiles - 1) / tiles;
  s = s > steps / 4 ? steps / 4 : s;
  return (int)(s < 1 ? 1 : s > 64 ? 64 : s);
}

Layout plan(const Call& c) {
  Layout L = {};
  const bool f32 = c.dtype == TB_F32;
  L.planes = f32 ? 3 : 1;
  L.np = up(c.n, kTile);
  L.dp = up(c.D, kStep);
  L.copy_w = f32 || c.D % kStep != 0 || c.w_stride % 8 != 0 || (uintptr_t)c.w % 16 != 0;
  L.n_part = 2 * (int32_t)(up(c.C, kTile) / kTile);
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t here = at;
    at += up(bytes, 256);
    return here;
  };
  L.meta = take(sizeof(Meta));
  L.idx = take(c.n * 4);
  L.inv = take(c.n * 4);
  L.tgt = take(L.np * 4);
  L.a = take(L.np * 4);
  L.b = take(L.np * 4);
  L.lse = take(L.np * 4);
  L.hit = take(L.np * 4);
  if (!c.lse) L.part = take(L.np * L.n_part * 8);
  L.x = take(L.planes * L.np * L.dp * 2);
  if (L.copy_w) L.w = take(L.planes * c.C * L.dp * 2);
  if (c.dx || c.dw || c.db) {
    // pieces of the vocabulary of about kGradBytes of gradients, of equal sizes
    const int64_t all = L.planes * L.np * 2 * c.C;
    int64_t pieces = (all + kGradBytes / 2) / kGradBytes;
    pieces = pieces < 1 ? 1 : pieces;
    L.piece = (int32_t)up((c.C + pieces - 1) / pieces, kTile);
    L.pieces = (c.C + L.piece - 1) / L.piece;
    L.G = take(L.planes * L.np * L.piece * 2);
    const int64_t td = (L.dp + kTile - 1) / kTile;
    if (c.dx) {
      L.split_x = splits(td * (L.np / kTile), L.piece / kStep);
      L.acc_x = take(L.split_x * L.np * L.dp * 4);
    }
    if (c.dw) {
      L.split_w = splits(td * (L.piece / kTile), L.np / kStep);
      if (L.split_w > 1) L.acc_w = take(L.split_w * (int64_t)L.piece * L.dp * 4);
    }
    if (c.db) L.col = take(L.np / 64 * L.piece * 4);
  }
  L.total = at;
  return L;
}

unsigned blocks(int64_t work) {
  const int64_t b = (work + 255) / 256;
  return (unsigned)(b < 1 ? 1 : b > 8192 ? 8192 : b);
}

template <class T>
hipError_t run_t(const Call& c, char* ws, hipStream_t st) {
  const bool f32 = sizeof(T) == 4;
  const Layout L = plan(c);
  const bool grads = c.dx || c.dw || c.db;
  Meta* meta = reinterpret_cast<Meta*>(ws + L.meta);
  auto i32 = [&](int64_t at) { return reinterpret_cast<int32_t*>(ws + at); };
  auto flt = [&](int64_t at) { return reinterpret_cast<float*>(ws + at); };
  auto u16 = [&](int64_t at) { return reinterpret_cast<uint16_t*>(ws + at); };
  int32_t *idx = i32(L.idx), *inv = i32(L.inv), *tgt = i32(L.tgt);
  float *a = flt(L.a), *b = flt(L.b), *lse = flt(L.lse);
  const Gather ga = {c.n, c.C, c.target, c.weight, c.d_loss, c.d_lse, c.lse, grads, (int32_t)L.np,
                     meta, idx, inv, tgt, a, b, lse, c.out_loss, c.out_lse};
  gather_kernel<<<dim3(1), dim3(1024), 0, st>>>(ga);
  planes_kernel<T><<<dim3(blocks(L.np * (L.dp / 4))), dim3(256), 0, st>>>(
      static_cast<const T*>(c.x), c.x_stride, c.D, (int32_t)L.dp, idx, meta, c.n, u16(L.x),
      L.np * L.dp);
  if (L.copy_w && c.n > 0)
    planes_kernel<T><<<dim3(blocks(c.C * (L.dp / 4))), dim3(256), 0, st>>>(
        static_cast<const T*>(c.w), c.w_stride, c.D, (int32_t)L.dp, nullptr, nullptr, c.C, u16(L.w),
        c.C * L.dp);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;

  const Operand X = {u16(L.x), L.np * L.dp, L.dp, (int32_t)L.np, (int32_t)L.np};
  const Operand W = {L.copy_w ? u16(L.w) : static_cast<const uint16_t*>(c.w), c.C * L.dp,
                     L.copy_w ? L.dp : c.w_stride, c.C, c.C};
  Gemm g = {};
  g.meta = meta;
  g.bias = c.bias;
  g.C = c.C;
  g.row = {tgt, a, b, lse};
  g.k = (int32_t)L.dp;
  g.splits = 1;
  g.Q = X;
  g.tq = (int32_t)(L.np / kTile);
  g.D = c.D;
  if (!c.lse && c.n > 0) {
    g.P = W;
    g.tp = (c.C + kTile - 1) / kTile;
    g.part = reinterpret_cast<float2*>(ws + L.part);
    g.n_part = L.n_part;
    g.hit = flt(L.hit);
    e = f32 ? stats_f32(g, st) : stats_bf16(g, st);
    if (e != hipSuccess) return e;
    const Finish f = {meta, g.part, L.n_part, g.hit, idx, tgt, c.weight, lse, a, b, c.out_loss,
                      c.out_lse};
    finish_kernel<<<dim3((unsigned)((c.n + 3) / 4)), dim3(256), 0, st>>>(f);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!grads) return hipSuccess;

  const int32_t td = (int32_t)((L.dp + kTile - 1) / kTile);
  for (int32_t piece = 0; piece < L.pieces; ++piece) {
    const int32_t c0 = piece * L.piece, n = c.C - c0 < L.piece ? c.C - c0 : L.piece;
    const int32_t cols = (int32_t)up(n, kTile);
    Gemm z = g;
    z.P = W;
    z.P.p += c0 * W.ld;
    z.P.n = n;
    z.tp = cols / kTile;
    z.c0 = c0;
    z.G = u16(L.G);
    z.g_plane = L.np * L.piece;
    z.ldg = L.piece;
    z.col = c.db ? flt(L.col) : nullptr;
    e = f32 ? logit_grad_f32(z, st) : logit_grad_bf16(z, st);
    if (e != hipSuccess) return e;
    const Operand G = {z.G, z.g_plane, L.piece, (int32_t)L.np, n};
    if (c.db) {
      columns_kernel<T><<<dim3((n + 255) / 256), dim3(256), 0, st>>>(
          flt(L.col), L.piece, meta, static_cast<T*>(c.db) + c0, n);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    if (c.dx) {
      // sum over the piece's tokens; a transposed operand's columns are the layer's width
      Gemm x = g;
      x.P = {W.p + c0 * W.ld, W.plane, W.ld, (int32_t)L.dp, n};
      x.Q = G;
      x.tp = td;
      x.splits = L.split_x;
      x.k = (int32_t)up(n, kStep);
      x.acc = flt(L.acc_x);
      x.acc_split = L.np * L.dp;
      x.lda = (int32_t)L.dp;
      x.add = piece > 0;
      e = f32 ? dx_f32(x, st) : dx_bf16(x, st);
      if (e != hipSuccess) return e;
    }
    if (c.dw) {
      Gemm w = g;
      w.P = {X.p, X.plane, X.ld, (int32_t)L.dp, (int32_t)L.np};
      w.Q = {G.p, G.plane, G.ld, L.piece, (int32_t)L.np};
      w.tp = td;
      w.tq = cols / kTile;
      w.n_q = n;
      w.splits = L.split_w;
      w.k = (int32_t)L.np;
      T* out = static_cast<T*>(c.dw) + c0 * c.dw_stride;
      if (L.split_w > 1) {
        w.acc = flt(L.acc_w);
        w.acc_split = (int64_t)L.piece * L.dp;
        w.lda = (int32_t)L.dp;
      } else {
        w.out = out;
        w.ldo = c.dw_stride;
      }
      e = f32 ? dw_f32(w, st) : dw_bf16(w, st);
      if (e != hipSuccess) return e;
      if (L.split_w > 1) {
        join_kernel<T><<<dim3(blocks((int64_t)n * ((c.D + 3) / 4))), dim3(256), 0, st>>>(
            w.acc, w.acc_split, L.split_w, w.lda, nullptr, meta, out, c.dw_stride, n, c.D);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
      }
    }
  }
  if (c.dx)
    join_kernel<T><<<dim3(blocks(c.n * ((c.D + 3) / 4))), dim3(256), 0, st>>>(
        flt(L.acc_x), L.np * L.dp, L.split_x, (int32_t)L.dp, inv, meta, static_cast<T*>(c.dx),
        c.dx_stride, c.n, c.D);
  return hipGetLastError();
}

}  // namespace

int64_t workspace_bytes(const Call& c) { return plan(c).total; }

hipError_t run(const Call& c, void* workspace, hipStream_t st) {
  char* ws = static_cast<char*>(workspace);
  return c.dtype == TB_F32 ? run_t<float>(c, ws, st) : run_t<uint16_t>(c, ws, st);
}

}  // namespace linear
}  // namespace tbias
