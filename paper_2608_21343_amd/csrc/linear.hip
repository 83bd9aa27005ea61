// Cross entropy of a linear layer without its logits (linear.hpp): gathering of the
// rows, what joins the tiles' results, and the launches of a call.
#include <algorithm>

#include "linear_gemm.hpp"

namespace tbias {
namespace linear {

namespace {

// ---- the rows that take part

struct Gather {
  int64_t n;
  int32_t C;
  const int32_t* target;
  const float *weight, *d_loss, *d_lse, *lse, *lse_low;
  int32_t d_step;
  bool grads;
  Meta* meta;
  int32_t* counts;  // per group: rows that take part ...
  float* tops;      // ... and their largest finite |a|, |b|; NULL for a single group
  int32_t *idx, *inv, *tgt;
  float *a, *b, *lse_c, *r, *m;
  float *out_loss, *out_lse, *out_low;
  // the features, and their planes
  int64_t stride;
  int32_t D, dp;
  uint16_t* out;
  void* dx;  // rows that are left out get 0 here; or NULL
  int64_t dx_stride;
  int32_t blocks;  // workgroups that gather
  bool paired;     // every row's features twice, kPair rows apart
};

// Rows of a count, in 256s, and rows that a workgroup gathers. Up to 2048 rows are one
// group, which every workgroup counts, so that no launch counts before it, and take many
// workgroups, for their latency (2048 rows of 1024 float32: 21 us with 16 rows each, 13
// with 4). More rows are counted in groups of 256, since a workgroup counts its own group
// once more; workgroups of 16 rows, since in float32 each raises one word of the whole
// (16,000 rows of 512: 21 us, with groups of 2048 rows 25, with 4 rows each 34).
constexpr int kOnly = 8, kRowsOnly = 4, kMany = 1, kRowsMany = 16;
__host__ __device__ inline int64_t group_rows(int64_t n) {
  return 256 * (n <= 256 * kOnly ? kOnly : kMany);
}

struct Row {
  int32_t target;  // -1: left out, -2: out of range
  float a, b;
};

__device__ __forceinline__ Row row_of(const Gather& g, int64_t r) {
  Row o = {-1, 0.f, 0.f};
  if (r >= g.n) return o;
  o.target = g.target[r];
  const float w = g.weight ? g.weight[r] : 1.f;
  o.a = o.b = w;
  bool keep = o.target != -1 && w != 0.f;
  if (g.grads) {
    if (g.d_loss) o.b = w * g.d_loss[r * g.d_step];
    o.a = o.b + (g.d_lse ? g.d_lse[r] : 0.f);
    // a row without a gradient is left out, unless its loss is asked for
    if (g.lse) keep = keep && (o.a != 0.f || o.b != 0.f);
  }
  if (!keep) {
    o.target = -1;
  } else if ((uint32_t)o.target >= (uint32_t)g.C) {
    o.target = -2;
    o.a = o.b = __builtin_nanf("");
  }
  return o;
}

__device__ __forceinline__ float finite_top(const Row& o) {
  const float a = fabsf(o.a), b = fabsf(o.b), inf = __builtin_huge_valf();
  return o.target == -1 ? 0.f : fmaxf(a < inf ? a : 0.f, b < inf ? b : 0.f);
}

// Sums of two counts and the maximum of a float over a workgroup of 256.
__device__ __forceinline__ void join256(int32_t* x, int32_t* y, float* top) {
  __shared__ int32_t xs[4], ys[4];
  __shared__ float ts[4];
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    *x += __shfl_xor(*x, d);
    *y += __shfl_xor(*y, d);
    *top = fmaxf(*top, __shfl_xor(*top, d));
  }
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    xs[wave] = *x;
    ys[wave] = *y;
    ts[wave] = *top;
  }
  __syncthreads();
  *x = xs[0] + xs[1] + xs[2] + xs[3];
  *y = ys[0] + ys[1] + ys[2] + ys[3];
  *top = fmaxf(fmaxf(ts[0], ts[1]), fmaxf(ts[2], ts[3]));
}

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

// Four values of a row from d on, 0 behind its end. `wide`: aligned to 16 bytes.
__device__ __forceinline__ void load4(const float* x, int d, int D, bool wide, float* v) {
  if (wide && d + 4 <= D) {
    const float4 q = *reinterpret_cast<const float4*>(x + d);
    v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = d + e < D ? x[d + e] : 0.f;
  }
}
__device__ __forceinline__ void load4(const uint16_t* x, int d, int D, bool wide, float* v) {
  if (wide && d + 4 <= D) {
    const uint2 q = *reinterpret_cast<const uint2*>(x + d);
    v[0] = low16(q.x), v[1] = high16(q.x), v[2] = low16(q.y), v[3] = high16(q.y);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = d + e < D ? widen(x[d + e]) : 0.f;
  }
}

// Of the weights' copy as planes.
struct Weights {
  int64_t stride;
  int32_t D, dp, C;
  const float* bias;  // float32 only
  float* tops;        // [kTops] the largest finite value of some tokens each; float32 only
  uint16_t* out;
};
constexpr int kTops = 1024;

// A token that the bias takes out of every sum.
__device__ __forceinline__ bool masked(const float* bias, int64_t c) {
  return bias && bias[c] < -0x1p100f;
}

// One of kTops workgroups: the largest finite value of its rows' tokens.
__device__ __forceinline__ void top_of(const Weights& g, const float* w, int at) {
  const int lane = threadIdx.x & 63;
  const bool wide = g.stride % 4 == 0 && (uintptr_t)w % 16 == 0;
  int32_t none = 0;
  float top = 0.f;
  for (int64_t c = (int64_t)at * 4 + (threadIdx.x >> 6); c < g.C; c += 4 * kTops) {
    if (masked(g.bias, c)) continue;
#pragma unroll 4
    for (int d = 4 * lane; d < g.D; d += 256) {
      float v[4];
      load4(w + c * g.stride, d, g.D, wide, v);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (fabsf(v[e]) < __builtin_huge_valf()) top = fmaxf(top, fabsf(v[e]));
    }
  }
  join256(&none, &none, &top);
  if (threadIdx.x == 0) g.tops[at] = top;
}

// Rows that take part; behind the groups of rows (float32) the weights' largest values.
__global__ void __launch_bounds__(256)
    count_kernel(const Gather g, const Weights of, const float* w) {
  const int groups = gridDim.x - (w ? kTops : 0);
  if ((int)blockIdx.x >= groups) {
    top_of(of, w, blockIdx.x - groups);
    return;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) g.meta->T = 0;
  int32_t count = 0, none = 0;
  float top = 0.f;
  const int64_t first = blockIdx.x * group_rows(g.n);
  for (int64_t r = first + threadIdx.x; r < first + group_rows(g.n); r += 256) {
    const Row o = row_of(g, r);
    count += o.target != -1;
    top = fmaxf(top, finite_top(o));
  }
  join256(&count, &none, &top);
  if (threadIdx.x == 0 && g.counts) {
    g.counts[blockIdx.x] = count;
    g.tops[blockIdx.x] = top;
  }
}

// Raises *to to the largest of a workgroup's values (not negative, of the waves' first
// lanes), whatever the order; one atomic a workgroup, and none where it changes nothing.
__device__ __forceinline__ void raise(uint32_t* to, float v) {
  __shared__ float tops[4];
  if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = v;
  __syncthreads();
  if (threadIdx.x == 0) {
    const uint32_t top = __float_as_uint(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])));
    if (top > __hip_atomic_load(to, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) atomicMax(to, top);
  }
}

// One wave: a row as planes of dp values, and (float32) the unit it is divided by.
// `most`: its largest value. Up to 2048 values stay in registers; longer rows are read
// twice, the second time from the caches.
template <class T>
__device__ __forceinline__ float row_planes(const T* x, int D, int dp, bool wide, uint16_t* out,
                                            float* most) {
  constexpr int kKept = 8;
  const int lane = threadIdx.x & 63;
  float kept[kKept][4];
  float unit = 1.f, inverse = 1.f, top = 0.f;
  const bool keep = D <= kKept * 256;
  auto size = [&](const float* v) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (fabsf(v[e]) < __builtin_huge_valf()) top = fmaxf(top, fabsf(v[e]));
  };
  auto store = [&](int d, const float* v) {
    const float w[4] = {v[0] * inverse, v[1] * inverse, v[2] * inverse, v[3] * inverse};
    uint2 p[Elem<T>::PLANES];
    Elem<T>::planes4(w, p);
#pragma unroll
    for (int s = 0; s < Elem<T>::PLANES; ++s)
      *reinterpret_cast<uint2*>(out + place<Elem<T>::PLANES>(d) + s * kTurn) = p[s];
  };
  if (keep) {
#pragma unroll
    for (int k = 0; k < kKept; ++k)
      if (256 * k < dp) load4(x, 256 * k + 4 * lane, D, wide, kept[k]);
  }
  if (Elem<T>::kScaled) {
    if (keep) {
#pragma unroll
      for (int k = 0; k < kKept; ++k)
        if (256 * k < dp) size(kept[k]);
    } else {
      for (int d = 4 * lane; d < D; d += 256) {
        float v[4];
        load4(x, d, D, wide, v);
        size(v);
      }
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    unit = unit_of(top);
    inverse = 1.f / unit;
  }
  *most = top;
  if (keep) {
#pragma unroll
    for (int k = 0; k < kKept; ++k)
      if (256 * k + 4 * lane < dp) store(256 * k + 4 * lane, kept[k]);
  } else {
    for (int d = 4 * lane; d < dp; d += 256) {
      float v[4];
      load4(x, d, D, wide, v);
      store(d, v);
    }
  }
  return unit;
}

template <class T>
__device__ __forceinline__ bool rows_wide(const T* x, int64_t stride) {
  return stride * sizeof(T) % 16 == 0 && (uintptr_t)x % 16 == 0;
}

// One of `blocks` workgroups: the weights' planes, one wave a row.
template <class T>
__device__ __forceinline__ void planes_of(const Weights& g, const T* w, Meta* meta, int block,
                                          int blocks) {
  const int lane = threadIdx.x & 63;
  const bool wide = rows_wide(w, g.stride);
  float inverse = 1.f;
  if (Elem<T>::kScaled) {
    int32_t none = 0;
    float top = 0.f;
    for (int i = threadIdx.x; i < kTops; i += 256) top = fmaxf(top, g.tops[i]);
    join256(&none, &none, &top);
    const float unit = unit_of(top);
    if (block == 0 && threadIdx.x == 0) meta->S = unit;
    inverse = 1.f / unit;
  }
  for (int64_t c = (int64_t)block * 4 + (threadIdx.x >> 6); c < g.C;
       c += (int64_t)blocks * 4) {
    const bool hidden = Elem<T>::kScaled && masked(g.bias, c);
#pragma unroll 4
    for (int d = 4 * lane; d < g.dp; d += 256) {
      float v[4];
      load4(w + c * g.stride, d, g.D, wide, v);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        // (a masked token may be larger than the others: its logits stay numbers)
        const bool bound = hidden && fabsf(v[e]) < __builtin_huge_valf();
        v[e] *= inverse;
        if (bound) v[e] = __builtin_amdgcn_fmed3f(v[e], -0x1p15f, 0x1p15f);
      }
      uint2 p[Elem<T>::PLANES];
      Elem<T>::planes4(v, p);
#pragma unroll
      for (int s = 0; s < Elem<T>::PLANES; ++s)
        *reinterpret_cast<uint2*>(g.out + c * Elem<T>::PLANES * g.dp +
                                  place<Elem<T>::PLANES>(d) + s * kTurn) = p[s];
    }
  }
}

// ROWS rows: their place among those that take part, their arguments and planes.
// The rows before them are counted again up to the group's start, and groups by
// their counts, so that no launch has to wait for a sum over all of them. The workgroups
// behind those of the rows make the weights' planes, where they are copied, meanwhile.
template <class T, int EACH, int ROWS>
__global__ void __launch_bounds__(256) gather_kernel(const Gather g, const T* x, const Weights of,
                                                      const T* w) {
  if ((int)blockIdx.x >= g.blocks) {
    planes_of(of, w, g.meta, blockIdx.x - g.blocks, gridDim.x - g.blocks);
    return;
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row0 = (int64_t)blockIdx.x * ROWS;
  constexpr int64_t kGroup = 256 * EACH;
  const int64_t group = row0 / kGroup, groups = (g.n + kGroup - 1) / kGroup;
  int32_t before = 0, all = 0;
  float top = 0.f;
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    const int64_t r = group * kGroup + e * 256 + threadIdx.x;
    const Row o = row_of(g, r);
    before += o.target != -1 && r < row0;
    all += o.target != -1;
    top = fmaxf(top, finite_top(o));
  }
  if (groups > 1) {
    all = 0;
    for (int64_t i = threadIdx.x; i < groups; i += 256) {
      const int32_t count = g.counts[i];
      all += count;
      if (i < group) before += count;
      top = fmaxf(top, g.tops[i]);
    }
  }
  join256(&before, &all, &top);

  __shared__ int32_t places[ROWS];
  lds_poison(places, sizeof(places));
  if (wave == 0) {
    const int64_t r = row0 + lane;
    Row o = {-1, 0.f, 0.f};
    if (lane < ROWS) o = row_of(g, r);
    const uint64_t keep = __ballot(o.target != -1);
    const int32_t at = before + __popcll(keep & ((1ull << lane) - 1));
    if (lane < ROWS) places[lane] = o.target != -1 ? at : -1;
    if (lane < ROWS && r < g.n) {
      if (o.target == -1) {
        g.inv[r] = -1;
        if (g.out_loss) g.out_loss[r] = 0.f;
        if (g.out_lse) g.out_lse[r] = 0.f;
        if (g.out_low) g.out_low[r] = 0.f;
      } else {
        float lse = g.lse ? g.lse[r] : 0.f;
        // an empty row (no token above -inf) has no gradient
        if (lse == -__builtin_huge_valf()) o.a = o.b = lse = 0.f;
        // (exp(z - lse) has then the whole log-sum-exp in it: where p is near 1, p - 1 is
        // as exact as p)
        if (g.lse_low) o.a *= expf(-g.lse_low[r]);
        if (Elem<T>::kScaled) {
          float m = fmaxf(fabsf(o.a), fabsf(o.b));
          if (!(m > 0.f)) m = 1.f;  // (0 or NaN)
          o.a /= m;
          o.b /= m;
          g.m[at] = m;
        }
        g.inv[r] = at;
        g.idx[at] = (int32_t)r;
        g.tgt[at] = o.target;
        g.a[at] = o.a;
        g.b[at] = o.b;
        g.lse_c[at] = lse;
      }
    }
  }
  if ((int)blockIdx.x == g.blocks - 1 && threadIdx.x == 0) {
    // (no further, so that rows of far smaller weights keep their place in float32)
    top = fminf(fmaxf(top, 0x1p-24f), 0x1p24f);
    g.meta->n = all;
    g.meta->scale = top;
    g.meta->inverse = 1.f / top;
  }
  __syncthreads();
  const bool wide = rows_wide(x, g.stride);
  float weighty = 0.f;
  for (int i = wave; i < ROWS; i += 4) {
    const int32_t at = places[i];
    if (at < 0) {
      if (g.dx && row0 + i < g.n)
        for (int d = lane; d < g.D; d += 64)
          static_cast<T*>(g.dx)[(row0 + i) * g.dx_stride + d] = T(0);
      continue;
    }
    float most;
    const float unit = row_planes<T>(x + (row0 + i) * g.stride, g.D, g.dp, wide,
                                     g.out + (int64_t)at * Elem<T>::PLANES * g.dp, &most);
    if (!Elem<T>::kScaled && g.paired)
      row_planes<T>(x + (row0 + i) * g.stride, g.D, g.dp, wide,
                    g.out + (int64_t)(at + kPair) * g.dp, &most);
    if (Elem<T>::kScaled && lane == 0) {
      g.r[at] = unit;
      const float with = most * g.m[at];  // (written by this workgroup)
      if (with < __builtin_huge_valf()) weighty = fmaxf(weighty, with);
    }
  }
  if (Elem<T>::kScaled && g.grads) raise(&g.meta->T, weighty);
  if ((int)blockIdx.x == g.blocks - 1) {
    // the zeros behind the last row
    const int64_t row = Elem<T>::PLANES * g.dp, end = (g.paired ? kPair : up(all, kStep)) * row;
    for (int64_t i = all * row + 4 * threadIdx.x; i < end; i += 1024) {
      *reinterpret_cast<uint2*>(g.out + i) = make_uint2(0, 0);
      if (g.paired) *reinterpret_cast<uint2*>(g.out + kPair * row + i) = make_uint2(0, 0);
    }
  }
}

// float32: the planes of x_i m_i / T of the gathered rows, by some workgroups behind those of
// the rows' statistics or by a launch of its own.
struct Weighted {
  const float* x;
  int64_t stride;
  int32_t D, dp;
  const int32_t* idx;
  const float* m;
  uint16_t* out;
  int32_t blocks;
};
__device__ __forceinline__ void weighted_of(const Weighted& g, const Meta& meta, int block) {
  const int lane = threadIdx.x & 63;
  const bool wide = rows_wide(g.x, g.stride);
  const int64_t have = meta.n, rows = up(have, kStep);
  const float inverse = 1.f / unit_of(__uint_as_float(meta.T));
  for (int64_t i = (int64_t)block * 4 + (threadIdx.x >> 6); i < rows; i += (int64_t)g.blocks * 4) {
    const float* from = i < have ? g.x + (int64_t)g.idx[i] * g.stride : nullptr;
    const float scale = i < have ? g.m[i] : 0.f;
    for (int d = 4 * lane; d < g.dp; d += 256) {
      float v[4] = {0.f, 0.f, 0.f, 0.f};
      if (from && d < g.D) {
        load4(from, d, g.D, wide, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = v[e] * scale * inverse;
      }
      uint2 p[2];
      Elem<float>::planes4(v, p);
      uint16_t* to = g.out + i * 2 * g.dp + place<2>(d);
      *reinterpret_cast<uint2*>(to) = p[0];
      *reinterpret_cast<uint2*>(to + kTurn) = p[1];
    }
  }
}
__global__ void __launch_bounds__(256) weighted_kernel(const Weighted g, const Meta* meta) {
  weighted_of(g, *meta, blockIdx.x);
}

// ---- what joins the tiles

// Log-sum-exp and loss, of gathered rows, whose parts lie by their place or (by_row) by
// their row; or (idx NULL) of all rows, and 0 for those left out.
struct Finish {
  const Meta* meta;
  const float2* part;
  int32_t n_part;
  const float* hit;
  const int32_t *idx, *target;  // target of every row of x
  bool by_row;
  int32_t n, C;
  const float* weight;
  float *lse_c, *a, *b;
  float *out_loss, *out_lse, *out_low;
};

// Maximum (or sum) over L lanes: part of a wave, or the four waves of a workgroup.
template <int L, bool MAX>
__device__ __forceinline__ float over(float v, float* lds) {
#pragma unroll
  for (int d = L < 64 ? L / 2 : 32; d > 0; d >>= 1)
    v = MAX ? fmaxf(v, __shfl_xor(v, d)) : v + __shfl_xor(v, d);
  if (L <= 64) return v;
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return MAX ? fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3]))
             : (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// L lanes a row: 16 for up to 128 parts (32,768 rows of 66: 7 us instead of 13 with a
// wave each), or the workgroup for few rows with many parts.
template <int L>
__global__ void __launch_bounds__(256) finish_kernel(const Finish f, const Weighted g) {
  if ((int)blockIdx.x < g.blocks) {
    weighted_of(g, *f.meta, blockIdx.x);
    return;
  }
  static_assert(L == 16 || L == 64 || L == 256, "lanes of a row");
  __shared__ float lds[2][4];
  lds_poison(lds, sizeof(lds));
  const int lane = threadIdx.x % L;
  const int64_t at = ((int64_t)(blockIdx.x - g.blocks) * 256 + threadIdx.x) / L;
  if (at >= (f.idx ? f.meta->n : f.n)) return;
  const int64_t row = f.idx ? f.idx[at] : at, from = f.by_row ? row : at;
  const int32_t t = f.target[row];
  const float weight = f.weight ? f.weight[row] : 1.f;
  if (!f.idx && (t == -1 || weight == 0.f)) {
    if (lane == 0 && f.out_loss) f.out_loss[row] = 0.f;
    if (lane == 0 && f.out_lse) f.out_lse[row] = 0.f;
    if (lane == 0 && f.out_low) f.out_low[row] = 0.f;
    return;
  }
  const float2* part = f.part + from * f.n_part;
  float m = -__builtin_huge_valf();
  for (int i = lane; i < f.n_part; i += L) m = fmaxf(m, part[i].x);
  m = over<L, true>(m, lds[0]);
  const float base = m == -__builtin_huge_valf() ? 0.f : m;
  float sum = 0.f;
  for (int i = lane; i < f.n_part; i += L) {
    const float2 v = part[i];
    // (a part without a value has maximum -inf and sum 0; a NaN in either stays)
    sum += v.y * __builtin_amdgcn_exp2f((v.x - base) * kLog2e);
  }
  sum = over<L, false>(sum, lds[1]);
  if (lane != 0) return;
  const float rest = logf(sum), lse = base + rest;
  if (f.out_lse) f.out_lse[row] = lse;
  if (f.out_low) {
    // what the rounding of that sum left, exactly
    const float rounded = lse - base, low = (base - (lse - rounded)) + (rest - rounded);
    f.out_low[row] = fabsf(lse) < __builtin_huge_valf() ? low : 0.f;
  }
  if (f.out_loss) {
    // (the maximum first: a small loss keeps its digits; an empty row's is +inf)
    float nll = lse == -__builtin_huge_valf() ? -lse : (base - f.hit[from]) + rest;
    if ((uint32_t)t >= (uint32_t)f.C) nll = __builtin_nanf("");
    f.out_loss[row] = f.weight ? weight * nll : nll;
  }
  if (!f.idx) return;
  if (lse == -__builtin_huge_valf()) {
    f.lse_c[at] = 0.f;
    f.a[at] = f.b[at] = 0.f;
  } else {
    // a exp(z - lse), with nothing of lse rounded
    f.lse_c[at] = base;
    f.a[at] /= sum;
  }
}

// The gradients of logits that are kept: ROWS gathered rows by 256 tokens a workgroup, a
// quarter of them a wave. The rows behind the last one, up to a multiple of kStep, get
// zeros, and so do the tokens.
struct Kept {
  const Meta* meta;
  const float* z;
  int32_t ldz;
  const int32_t* idx;  // rows of z, or NULL: gathered ones
  RowArgs row;
  int32_t C, cols;
  bool paired;  // what the rounding of a row left goes kPair rows further on
  uint16_t* G;
  float* col;
};

template <class T, int ROWS>
__global__ void __launch_bounds__(256) kept_kernel(const Kept k) {
  typedef Elem<T> El;
  const Meta meta = *k.meta;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row0 = (int64_t)blockIdx.y * ROWS + ROWS / 4 * wave;
  const int c0 = blockIdx.x * 256 + 4 * lane;
  if ((int64_t)blockIdx.y * ROWS >= up(meta.n, kStep)) return;
  const float norm = El::kScaled ? 1.f : meta.inverse;
  float cs[4] = {0.f, 0.f, 0.f, 0.f};
  if (c0 < k.cols) {
#pragma unroll 4
    for (int i = 0; i < ROWS / 4; ++i) {
      const int64_t at = row0 + i;
      float v[4] = {0.f, 0.f, 0.f, 0.f};
      if (at < meta.n) {
        const float* z = k.z + (k.idx ? (int64_t)k.idx[at] : at) * k.ldz + c0;
        const float lse = k.row.lse[at], a = k.row.a[at] * norm, b = k.row.b[at] * norm;
        const int t = k.row.target[at] - c0;
        const f32x4 l = *reinterpret_cast<const f32x4*>(z);
        const float m = El::kScaled ? k.row.m[at] : 1.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (c0 + e >= k.C) continue;
          v[e] = a * __builtin_amdgcn_exp2f((l[e] - lse) * kLog2e) - (t == e ? b : 0.f);
          cs[e] += v[e] * m;
          if (El::kScaled) v[e] *= 0x1p14f;
        }
      }
      uint2 p[El::PLANES];
      El::planes4(v, p);
      if (!El::kScaled && k.paired) {
        if (at >= kPair) continue;
        float left[4] = {v[0] - low16(p[0].x), v[1] - high16(p[0].x), v[2] - low16(p[0].y),
                         v[3] - high16(p[0].y)};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (!(fabsf(left[e]) < __builtin_huge_valf())) left[e] = 0.f;
        uint2 q[El::PLANES];
        El::planes4(left, q);
        *reinterpret_cast<uint2*>(k.G + (at + kPair) * k.ldz + c0) = q[0];
      }
#pragma unroll
      for (int s = 0; s < El::PLANES; ++s)
        *reinterpret_cast<uint2*>(k.G + at * El::PLANES * k.ldz + place<El::PLANES>(c0) +
                                  s * kTurn) = p[s];
    }
  }
  if (!k.col) return;
  __shared__ float4 sums[4][64];
  lds_poison(sums, sizeof(sums));
  sums[wave][lane] = make_float4(cs[0], cs[1], cs[2], cs[3]);
  __syncthreads();
  if (wave == 0 && c0 < k.cols) {
    const float4 a = sums[0][lane], b = sums[1][lane], c = sums[2][lane], d = sums[3][lane];
    *reinterpret_cast<float4*>(k.col + (int64_t)blockIdx.y * k.ldz + c0) =
        make_float4((a.x + b.x) + (c.x + d.x), (a.y + b.y) + (c.y + d.y),
                    (a.z + b.z) + (c.z + d.z), (a.w + b.w) + (c.w + d.w));
  }
}

// out[r] = the sum of the splits' rows inv[r] (dx; 0 for the rows left out) or r (dw).
template <class T>
__global__ void __launch_bounds__(256)
    join_kernel(const Gemm g, const int32_t* inv, T* out, int64_t ldo, int64_t n) {
  const int64_t each = (g.D + 3) / 4;
  const Meta meta = *g.meta;
  const bool wide = ldo % 4 == 0 && (uintptr_t)out % (4 * sizeof(T)) == 0;
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < n * each;
       at += (int64_t)gridDim.x * 256) {
    const int64_t row = at / each;
    const int d = (int)(at - row * each) * 4;
    const int64_t from = inv ? inv[row] : row;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    Scale scale = {0.f, 0};
    if (from >= 0) {
      const float* p = g.acc + from * g.lda + d;
      for (int s = 0; s < g.splits; ++s) {
        v += *reinterpret_cast<const f32x4*>(p + s * g.acc_split);
        if (g.paired) v += *reinterpret_cast<const f32x4*>(p + s * g.acc_split + kPair * g.lda);
      }
      scale = inv ? dx_scale<T>(g, meta, from) : dw_scale<T>(meta);
    }
    float w[4] = {0.f, 0.f, 0.f, 0.f};
    if (from >= 0)
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = scaled<T>(v[e], scale);
    store4(out + row * ldo + d, w, wide, g.D - d);
  }
}

// db[c] = the sum of the columns over the blocks of `rows` rows (rows_rest from token `main`
// on): 64 tokens a workgroup, a sixteenth of the blocks each wave.
template <class T>
__global__ void __launch_bounds__(1024)
    columns_kernel(const float* col, int32_t ldg, const Meta* meta, int32_t rows, int32_t main,
                   int32_t rows_rest, T* db, int32_t n) {
  __shared__ float sums[16][64];
  lds_poison(sums, sizeof(sums));
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = blockIdx.x * 64 + lane;
  if (c >= main) rows = rows_rest;
  const int tiles = (meta->n + rows - 1) / rows;
  float sum = 0.f;
  if (c < n)
    for (int q = wave; q < tiles; q += 16) sum += col[(int64_t)q * ldg + c];
  sums[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && c < n) {
#pragma unroll
    for (int w = 1; w < 16; ++w) sum += sums[w][lane];
    store_out(db + c, Elem<T>::kScaled ? sum : sum * meta->scale);
  }
}

// ---- workspace

// Of the gradients of a piece's logits (4096 x 2048 bfloat16 against 131,073 tokens in pieces of
// 256 MB 7.4 ms, of 128 8.4, of 64 10.2), and of logits that are kept.
constexpr int64_t kGradBytes = 256ll << 20;
constexpr int64_t kMostStride = 1 << 22;      // of weights that are read where they are
// Rows that linear_few.hip takes, whatever a call returns: its logits differ in their last
// bits from those of the tiles, so a call that gives lse and the one that takes it, and a call's
// statistics and gradients, go by one rule (their logits are always kept: 64 rows against 2^20
// tokens are 256 MB). It reads the weights once for 16 bfloat16 rows and is bound by that (16
// rows of 1024 against 131,073 tokens 54 us, tiles 86; 32 rows 62 and 85; 64 rows 89 and 84),
// float32 ones without a copy of the weights (64 rows against 131,073 tokens 218 us, tiles
// with the copy 475). With gradients the copy is made in any case: steps and backward passes
// of 17 to 64 float32 rows take up to a quarter longer than with tiles' logits (32,769
// tokens: 32 rows 254 us and 236, 64 rows 306 and 243), bfloat16 ones up to a tenth.
int32_t few_rows(bool f32) { return f32 ? 64 : 32; }

// How a product is cut: tiles of 256 x 256, or smaller ones where those would leave CUs
// idle, and parts of the summed axis where that still leaves them idle. The costs are in
// stages of a tile of 256 (1.3 us in bfloat16, measured at full load); a smaller tile's
// takes longer for its size, since its operands are read from LDS more often, and every
// tile costs some besides (first loads, epilogue), parts a way through memory. Steps, chosen so
// and in tiles of 256 alone: 1511 bfloat16 rows of 336 against 612 tokens 52 and 86 us, 1000
// float32 rows of 512 against 4097 124 and 158, 16,000 against 1025 292 and 326; chosen so
// and without parts: the last 292 and 400, 300 bfloat16 rows of 1024 against 50,001 230 and 490.
// `full`: no tile of which less than half of P is there, since what a tile writes has its place
// in memory (the gradients of 1,048,576 float32 rows against 50 tokens 256 MB, and 1 GB in
// tiles of 256).
Cut cut(int64_t p, int64_t q, int64_t steps, int64_t stages, bool parts, bool full = false) {
  Cut best = {256, 1, 0};
  const struct {
    int32_t tile;
    double step, fixed;
  } sizes[] = {{256, 1.0, 4.0}, {128, 0.36, 2.5}, {64, 0.15, 1.5}};
  // parts are written and read once more, 7 MB in the time of a stage
  const double way = 8.0 * (double)p * (double)q / 7e6;
  for (const auto& s : sizes) {
    if (full && s.tile >= 2 * up(p, kStep)) continue;
    const int64_t tiles = ((p + s.tile - 1) / s.tile) * ((q + s.tile - 1) / s.tile);
    for (int n = 1; n <= (parts ? 64 : 1) && n <= (steps + 3) / 4; ++n) {
      const double rounds = (double)((tiles * n + 255) / 256);
      const double cost = rounds * ((double)((steps + n - 1) / n) * stages * s.step + s.fixed) +
                          (n > 1 ? 4.0 + n * way : 0.0);
      if (best.cost == 0 || cost < best.cost * 0.97) best = {s.tile, n, cost};
    }
  }
  return best;
}

// The tokens of a product: those in whole tiles of 256, and where it pays the few behind
// them on their own. A vocabulary and its blank are often one more than a multiple of 256,
// and a row of tiles for that one token may be a round of the whole card (a step of 2048 x
// 1024 float32 against 32,769 tokens 1483 us, and 1666 without; of 2000 x 512 bfloat16
// against 8193 165 and 182).
constexpr int64_t kRest = 64;  // tokens that may be on their own
Strips strips(int64_t tokens, int64_t others, int64_t steps, int64_t stages, bool parts,
              bool full = false) {
  Strips s = {(int32_t)tokens, {cut(tokens, others, steps, stages, parts, full), {64, 1, 0}}};
  const int64_t rest = tokens % 256, main = tokens - rest;
  if (rest == 0 || rest > kRest || main == 0) return s;
  const Cut a = cut(main, others, steps, stages, parts, full);
  const Cut b = cut(rest, others, steps, stages, parts, full);
  // (a launch of its own: 4 us)
  if (a.cost + b.cost + 3.0 < s.cut[0].cost) s = {(int32_t)main, {a, b}};
  return s;
}

}  // namespace

Layout plan(const Call& c) {
  Layout L = {};
  const bool f32 = c.dtype == TB_F32;
  L.planes = f32 ? 2 : 1;
  const bool grads = c.dx || c.dw || c.db;
  L.np = up(c.n, kTile);
  L.dp = up(c.D, kStep);
  // (the loads of a stage reach the 256 rows of a tile by 32-bit distances in bytes)
  L.copy_w = f32 || c.D % kStep != 0 || c.w_stride % 8 != 0 || (uintptr_t)c.w % 16 != 0 ||
             c.w_stride > kMostStride;
  // few rows are read where they are (16-byte aligned, of whole pieces of 16 bytes)
  const int64_t size = f32 ? 4 : 2;
  const bool read = c.D * size % 16 == 0 && c.w_stride * size % 16 == 0 &&
                    (uintptr_t)c.w % 16 == 0 && c.x_stride * size % 16 == 0 &&
                    (uintptr_t)c.x % 16 == 0;
  L.few = read && c.n <= few_rows(f32);
  // (the loss of few rows needs no copies)
  L.gather = grads || !L.few;
  L.copy_w = L.copy_w && L.gather;
  // products of planes that a step takes
  const int64_t stages = f32 ? 3 : 1;
  L.stats = strips(c.C, c.n, L.dp / kStep, stages, false, grads);
  L.n_part = few_parts(c.C);
  if (!L.few) {
    const int32_t main = L.stats.main, rest = c.C - main;
    const int32_t a = L.stats.cut[0].tile, b = L.stats.cut[1].tile;
    L.n_part = 2 * ((main + a - 1) / a + (rest + b - 1) / b);
  }
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t here = at;
    at += up(bytes, 256);
    return here;
  };
  L.meta = take(sizeof(Meta));
  const int64_t groups = (c.n + group_rows(c.n) - 1) / group_rows(c.n);
  L.counts = take((groups + 1) * 4);  // (without rows one is written all the same)
  L.tops = take((groups + 1) * 4);
  L.idx = take(c.n * 4);
  L.inv = take(c.n * 4);
  L.tgt = take(L.np * 4);
  L.a = take(L.np * 4);
  L.b = take(L.np * 4);
  L.lse = take(L.np * 4);
  if (f32) L.r = take(L.np * 4);
  if (f32) L.m = take(L.np * 4);
  if (f32) L.most = take(kTops * 4);
  L.hit = take(L.np * 4);
  if (!c.lse || L.few || c.n <= kPair) L.part = take(c.n * L.n_part * 8);
  if (L.gather) L.px = take(L.planes * L.np * L.dp * 2);
  if (f32 && c.dw) L.pxm = take(L.planes * L.np * L.dp * 2);
  if (L.copy_w) L.pw = take(L.planes * c.C * L.dp * 2);
  if (grads) {
    // Logits that the statistics write and the gradients read again (float32, up to 256 MB)
    // cost less than another product: a step of 16,000 x 512 float32 against 1025 tokens 292
    // us instead of 313, of 300 x 1024 bfloat16 against 50,001 230 instead of 258.
    const bool pair = !f32 && c.n > 0 && c.n <= kPair;  // (without rows there is nothing to keep)
    L.kept = (!c.lse || L.few || pair) && c.n * up(c.C, kTile) * 4 <= kGradBytes;
    // Pieces of the vocabulary of about kGradBytes of gradients, of equal sizes. Those of kept
    // logits are made by 64 rows, others by tiles.
    L.rows_g = L.kept ? up(c.n, kStep) : L.np;
    const int64_t all = L.planes * L.rows_g * 2 * up(c.C, kStep);
    int64_t pieces = (all + kGradBytes / 2) / kGradBytes;
    // (a few tokens more than whole tiles go with the last piece, and none is without a tile)
    pieces = std::max<int64_t>(std::min(pieces, (c.C - kRest + kTile - 1) / kTile), 1);
    L.piece = (int32_t)up(pieces == 1 ? c.C : (c.C - kRest + pieces - 1) / pieces, kTile);
    L.pieces = pieces == 1 ? 1 : (int32_t)((c.C - kRest + L.piece - 1) / L.piece);
    const int32_t last = c.C - (L.pieces - 1) * L.piece;
    const int32_t most = std::max(last, std::min(c.C, L.piece));
    L.kept = L.kept && L.pieces == 1;
    if (!L.kept) L.rows_g = L.np;
    L.paired = L.kept && pair;
    L.grad = strips(last, c.n, L.dp / kStep, stages, false, true);
    L.grad_all = cut(L.piece, c.n, L.dp / kStep, stages, false);
    // (a row ends where the last tile that writes it does)
    auto reach = [](const Strips& s, int32_t tokens) {
      return (int32_t)(s.main < tokens ? s.main + up(tokens - s.main, s.cut[1].tile)
                                       : up(tokens, s.cut[0].tile));
    };
    L.ldg = L.kept ? (int32_t)up(c.C, kStep) : reach(L.grad, last);
    if (L.kept && !L.few) L.ldg = reach(L.stats, c.C);
    if (L.pieces > 1) L.ldg = std::max(L.ldg, L.piece);
    L.G = take(L.planes * L.rows_g * L.ldg * 2);
    // (by 16 rows where 64 would leave CUs idle: a step of 1511 bfloat16 rows of 336 against 612
    // tokens 51 us by 64, 47 by 16; of 16,000 float32 rows of 512 against 1025 288 and 300)
    L.kept_rows = up(c.n, 64) / 64 * ((c.C + 255) / 256) < 1024 ? 16 : 64;
    if (L.kept) L.z = take(c.n * L.ldg * 4);
    if (c.dx) {
      L.x = cut(L.dp, c.n, up(most, kStep) / kStep, stages, true);
      L.direct = L.x.parts == 1 && !L.paired;
      L.rows_x = L.paired ? 2 * kPair : c.n;
      if (!L.direct || L.pieces > 1) L.acc_x = take(L.x.parts * L.rows_x * L.dp * 4);
    }
    if (c.dw) {
      // (the last piece's cut: all others have whole tiles)
      L.w = strips(last, L.dp, L.np / kStep, stages, true);
      L.w_all = cut(L.piece, L.dp, L.np / kStep, stages, true);
      // (strip by strip: the one token behind whole tiles may be summed in many parts)
      auto sums = [&](int64_t tokens, const Cut& cut) {
        return cut.parts > 1 ? cut.parts * tokens * L.dp * 4 : 0;
      };
      L.acc_w = take(std::max({sums(L.w.main, L.w.cut[0]), sums(last - L.w.main, L.w.cut[1]),
                               L.pieces > 1 ? sums(L.piece, L.w_all) : 0}));
    }
    if (c.db) L.col = take(L.rows_g / (L.kept ? L.kept_rows : 64) * L.ldg * 4);
  }
  L.total = at;
  return L;
}

namespace {

unsigned blocks(int64_t work) {
  const int64_t b = (work + 255) / 256;
  return (unsigned)(b < 1 ? 1 : b > 8192 ? 8192 : b);
}

template <class T>
hipError_t run_t(const Call& c, const Layout& L, char* ws, hipStream_t st) {
  constexpr bool f32 = sizeof(T) == 4;
  const bool grads = c.dx || c.dw || c.db;
  Meta* meta = reinterpret_cast<Meta*>(ws + L.meta);
  auto i32 = [&](int64_t at) { return reinterpret_cast<int32_t*>(ws + at); };
  auto flt = [&](int64_t at) { return reinterpret_cast<float*>(ws + at); };
  auto u16 = [&](int64_t at) { return reinterpret_cast<uint16_t*>(ws + at); };
  int32_t *idx = i32(L.idx), *inv = i32(L.inv), *tgt = i32(L.tgt);
  float *a = flt(L.a), *b = flt(L.b), *lse = flt(L.lse);
  float *r = f32 ? flt(L.r) : nullptr, *m = f32 ? flt(L.m) : nullptr;
  const int64_t groups = (c.n + group_rows(c.n) - 1) / group_rows(c.n);
  const int rows = groups > 1 ? kRowsMany : kRowsOnly;
  const Gather ga = {c.n,    c.C,  c.target, c.weight,   c.d_loss,
                     c.d_lse, c.lse, c.lse_low, c.d_step,
                     grads,  meta, i32(L.counts), flt(L.tops), idx, inv, tgt,
                     a,      b,    lse, r, m, c.out_loss, c.out_lse, c.out_low,
                     c.x_stride, c.D, (int32_t)L.dp, u16(L.px),
                     L.direct ? c.dx : nullptr, c.dx_stride,
                     (int32_t)std::max<int64_t>((c.n + rows - 1) / rows, 1), L.paired};
  const Weights weights = {c.w_stride, c.D, (int32_t)L.dp, c.C,
                           f32 ? static_cast<const float*>(c.bias) : nullptr,
                           f32 ? flt(L.most) : nullptr, u16(L.pw)};
  // (float32: it also clears what the others take maxima into)
  if (L.gather && (groups != 1 || f32)) {
    const bool tops = f32 && c.n > 0;
    const int64_t all = std::max<int64_t>(groups, 1) + (tops ? kTops : 0);
    count_kernel<<<dim3((unsigned)all), dim3(256), 0, st>>>(
        ga, weights, tops ? static_cast<const float*>(c.w) : nullptr);
  }
  if (L.gather) {
    const auto gather = groups > 1 ? &gather_kernel<T, kMany, kRowsMany>
                                   : &gather_kernel<T, kOnly, kRowsOnly>;
    const int more = !L.copy_w || c.n == 0 ? 0 : c.C < 8192 ? (c.C + 3) / 4 : 2048;
    gather<<<dim3((unsigned)(ga.blocks + more)), dim3(256), 0, st>>>(
        ga, static_cast<const T*>(c.x), weights, static_cast<const T*>(c.w));
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;

  constexpr int PL = Elem<T>::PLANES;
  const Operand X = {u16(L.px), PL * L.dp, (int32_t)L.np, (int32_t)L.np};
  const Operand W = {L.copy_w ? u16(L.pw) : static_cast<const uint16_t*>(c.w),
                     L.copy_w ? PL * L.dp : c.w_stride, c.C, c.C};
  Gemm g = {};
  g.meta = meta;
  g.bias = c.bias;
  g.C = c.C;
  g.row = {tgt, a, b, lse, r, m};
  g.k = (int32_t)L.dp;
  g.splits = 1;
  g.Q = X;
  g.D = c.D;
  g.idx = idx;
  auto tiles = [](int64_t n, const Cut& cut) { return (int32_t)((n + cut.tile - 1) / cut.tile); };
  // The launches over the tokens of a product, strip by strip: at(g, first token of the
  // strip, its tokens, its cut) completes and launches one.
  auto over = [&](const Strips& s, int32_t tokens, auto at) {
    hipError_t r = at(0, std::min(s.main, tokens), s.cut[0]);
    return r != hipSuccess || s.main >= tokens ? r : at(s.main, tokens - s.main, s.cut[1]);
  };
  Weighted weighted = {};
  if constexpr (f32) {
    if (c.dw && c.n > 0)
      weighted = {static_cast<const float*>(c.x), c.x_stride, c.D, (int32_t)L.dp, idx, m,
                  u16(L.pxm), (int32_t)(c.n < 8192 ? (c.n + 3) / 4 : 2048)};
  }
  // (with lse at hand: the logits alone)
  if ((!c.lse || L.kept) && c.n > 0) {
    float2* part = reinterpret_cast<float2*>(ws + L.part);
    float *hit = flt(L.hit), *z = L.kept ? flt(L.z) : nullptr;
    if (L.few) {
      const Few f = {c.x,      c.w,      c.bias,   c.x_stride, c.w_stride, (int32_t)c.n, c.D, c.C,
                     c.target, L.n_part, few_each(c.C), part, hit, z, L.ldg};
      e = few(f, c.dtype, st);
    } else {
      e = over(L.stats, c.C, [&](int32_t first, int32_t n, const Cut& cut) {
        Gemm s = g;
        s.P = {W.p + first * W.ld, W.ld, n, n};
        s.tile = cut.tile;
        s.tp = tiles(n, cut);
        s.tq = tiles(c.n, cut);
        s.c0 = first;
        s.part = part + (first ? 2 * tiles(first, L.stats.cut[0]) : 0);
        s.n_part = L.n_part;
        s.hit = hit;
        s.z = z ? z + first : nullptr;
        s.ldg = L.ldg;
        return f32 ? stats_f32(s, st) : stats_bf16(s, st);
      });
    }
    if (e != hipSuccess) return e;
  }
  if (!c.lse && c.n > 0) {
    const Finish f = {meta, reinterpret_cast<float2*>(ws + L.part), L.n_part, flt(L.hit),
                      L.gather ? idx : nullptr, c.target, L.few, (int32_t)c.n, c.C, c.weight,
                      lse, a, b, c.out_loss, c.out_lse, c.out_low};
    const int lanes = L.n_part <= 128 ? 16 : c.n <= 1024 && L.n_part >= 256 ? 256 : 64;
    const auto finish =
        lanes == 16 ? &finish_kernel<16> : lanes == 64 ? &finish_kernel<64> : &finish_kernel<256>;
    finish<<<dim3((unsigned)(weighted.blocks + (c.n * lanes + 255) / 256)), dim3(256), 0, st>>>(
        f, weighted);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!grads) return hipSuccess;

  if (c.lse && weighted.blocks) {
    weighted_kernel<<<dim3(weighted.blocks), dim3(256), 0, st>>>(weighted, meta);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  Operand XM = X;  // of dw
  if (f32) XM.p = u16(L.pxm);
  for (int32_t piece = 0; piece < L.pieces; ++piece) {
    const bool last = piece + 1 == L.pieces;
    const int32_t c0 = piece * L.piece, n = last ? c.C - c0 : L.piece;
    const Strips grad = last ? L.grad : Strips{n, {L.grad_all, L.grad_all}};
    const Operand G = {u16(L.G), PL * L.ldg, (int32_t)L.rows_g, n};
    float* col = c.db ? flt(L.col) : nullptr;
    if (L.kept && c.n > 0) {
      const Kept k = {meta, flt(L.z), L.ldg, L.few ? idx : nullptr, g.row, c.C,
                      (int32_t)up(c.C, kStep), L.paired, u16(L.G), col};
      const auto make = L.kept_rows == 16 ? &kept_kernel<T, 16> : &kept_kernel<T, 64>;
      make<<<dim3((c.C + 255) / 256, (unsigned)(up(c.n, 64) / L.kept_rows)), dim3(256), 0, st>>>(k);
      e = hipGetLastError();
    } else {
      e = over(grad, n, [&](int32_t first, int32_t n, const Cut& cut) {
        Gemm z = g;
        z.P = {W.p + (c0 + first) * W.ld, W.ld, n, n};
        z.tile = cut.tile;
        z.tp = tiles(n, cut);
        z.tq = tiles(c.n, cut);
        z.c0 = c0 + first;
        z.G = u16(L.G) + PL * first;
        z.ldg = L.ldg;
        z.col = col ? col + first : nullptr;
        return f32 ? logit_grad_f32(z, st) : logit_grad_bf16(z, st);
      });
    }
    if (e != hipSuccess) return e;
    if (c.db) {
      columns_kernel<T><<<dim3((n + 63) / 64), dim3(1024), 0, st>>>(
          col, L.ldg, meta, L.kept ? L.kept_rows : grad.cut[0].tile, grad.main,
          L.kept ? L.kept_rows : grad.cut[1].tile, static_cast<T*>(c.db) + c0, n);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    if (c.dx) {
      // sum over the piece's tokens; a transposed operand's columns are the layer's width
      Gemm x = g;
      x.P = {W.p + c0 * W.ld, W.ld, (int32_t)L.dp, n};
      x.Q = G;
      x.tile = L.x.tile;
      x.tp = tiles(L.dp, L.x);
      x.tq = tiles(c.n, L.x);
      x.splits = L.x.parts;
      x.k = (int32_t)up(n, kStep / PL);  // (a stage has a token at least)
      x.acc = flt(L.acc_x);
      if (L.direct && last) {
        x.out = c.dx;
        x.ldo = c.dx_stride;
      }
      x.acc_split = L.rows_x * L.dp;
      x.lda = (int32_t)L.dp;
      x.add = piece > 0;
      x.paired = L.paired;
      e = f32 ? dx_f32(x, st) : dx_bf16(x, st);
      if (e != hipSuccess) return e;
    }
    if (c.dw) {
      const Strips all = last ? L.w : Strips{n, {L.w_all, L.w_all}};
      e = over(all, n, [&](int32_t first, int32_t n, const Cut& cut) {
        Gemm w = g;
        w.P = {XM.p, XM.ld, (int32_t)L.dp, (int32_t)L.np};
        w.c0 = c0 + first;
        w.Q = {G.p + PL * first, G.ld, L.ldg - first, (int32_t)L.np};
        w.tile = cut.tile;
        w.tp = tiles(L.dp, cut);
        w.tq = tiles(n, cut);
        w.n_q = n;
        w.splits = cut.parts;
        w.k = (int32_t)L.np;
        T* out = static_cast<T*>(c.dw) + (c0 + first) * c.dw_stride;
        if (cut.parts == 1) {
          w.out = out;
          w.ldo = c.dw_stride;
          return f32 ? dw_f32(w, st) : dw_bf16(w, st);
        }
        w.acc = flt(L.acc_w);
        w.acc_split = (int64_t)n * L.dp;
        w.lda = (int32_t)L.dp;
        const hipError_t r = f32 ? dw_f32(w, st) : dw_bf16(w, st);
        if (r != hipSuccess) return r;
        join_kernel<T><<<dim3(blocks((int64_t)n * ((c.D + 3) / 4))), dim3(256), 0, st>>>(
            w, nullptr, out, c.dw_stride, n);
        return hipGetLastError();
      });
      if (e != hipSuccess) return e;
    }
  }
  if (c.dx && c.n > 0 && !L.direct) {
    Gemm x = g;
    x.splits = L.x.parts;
    x.acc = flt(L.acc_x);
    x.acc_split = L.rows_x * L.dp;
    x.lda = (int32_t)L.dp;
    x.paired = L.paired;
    join_kernel<T><<<dim3(blocks(c.n * ((c.D + 3) / 4))), dim3(256), 0, st>>>(
        x, inv, static_cast<T*>(c.dx), c.dx_stride, c.n);
  }
  return hipGetLastError();
}

}  // namespace

int64_t most_workspace(Call c) {
  // wherever x lies, which few rows' kernel goes by
  c.x_stride = c.w_stride;
  c.x = nullptr;
  const int64_t aligned = plan(c).total;
  if (c.n > few_rows(true)) return aligned;
  c.x = reinterpret_cast<const void*>(1);
  return std::max(aligned, plan(c).total);
}

hipError_t run(const Call& c, const Layout& L, void* workspace, hipStream_t st) {
  char* ws = static_cast<char*>(workspace);
  return c.dtype == TB_F32 ? run_t<float>(c, L, ws, st) : run_t<uint16_t>(c, L, ws, st);
}

}  // namespace linear
}  // namespace tbias
