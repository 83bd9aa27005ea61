// The products of the linear cross entropy: tiles of 256 x 256 by eight waves of
// 128 x 64, sums of 16 x 16 x 32 matrix instructions in registers, operands staged
// through LDS by asynchronous 16-byte loads, two stages of 64 values of the summed
// axis.
//
// An operand whose rows run along the summed axis lies in LDS as [row, 64] with its
// 16-byte pieces exchanged by row, so that the 16 rows of a fragment's read cover
// all banks once. One whose rows run across it lies as [64, column] with its 32-byte
// pieces exchanged, and is read through the transposing LDS read.
#pragma once

#include "linear.hpp"

namespace tbias {
namespace linear {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((address_space(3))) char lds_char;

constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kLoads = kTile * kStep * 2 / (16 * kThreads);  // of a lane, for a stage of an operand
constexpr int kOperandBytes = kTile * kStep * 2;
constexpr int kStageBytes = 2 * kOperandBytes;

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
__device__ __forceinline__ float low16(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float high16(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }

// An operand of one type: its planes, the products of them that are summed (the
// largest last), and the matrix instruction.
template <class T>
struct Elem;
template <>
struct Elem<uint16_t> {
  static constexpr int PLANES = 1, PAIRS = 1;
  static constexpr bool kScaled = false;
  __device__ static inline int p(int) { return 0; }
  __device__ static inline int q(int) { return 0; }
  __device__ static inline void planes4(const float* v, uint2* out) {
    out[0] = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
  }
  __device__ static inline f32x4 mfma(s16x8 a, s16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Elem<float> {
  static constexpr int PLANES = 2, PAIRS = 3;  // (1, 0) (0, 1) (0, 0)
  static constexpr bool kScaled = true;
  __device__ static inline int p(int s) { return s == 0 ? 1 : 0; }
  __device__ static inline int q(int s) { return s == 1 ? 1 : 0; }
  __device__ static inline void planes4(const float* v, uint2* out) {
    const f16x2 a = {(_Float16)v[0], (_Float16)v[1]}, b = {(_Float16)v[2], (_Float16)v[3]};
    const f16x2 c = {(_Float16)(v[0] - (float)a[0]), (_Float16)(v[1] - (float)a[1])};
    const f16x2 d = {(_Float16)(v[2] - (float)b[0]), (_Float16)(v[3] - (float)b[1])};
    out[0] = make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
    out[1] = make_uint2(__builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d));
  }
  __device__ static inline f32x4 mfma(s16x8 a, s16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};

// Where a lane's 16-byte loads of a stage come from, in bytes from the operand's
// tile (i0, k0).
template <bool TR>
__device__ __forceinline__ void lane_offsets(const Operand& o, int32_t i0, int32_t k_left,
                                             uint32_t (&off)[kLoads]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int it = 0; it < kLoads; ++it) {
    const int at = (it * kWaves + wave) * 64 + lane;
    if (!TR) {
      const int row = at >> 3, piece = (at & 7) ^ ((row >> 1) & 7);
      const int r = min(row, o.n - 1 - i0);
      off[it] = (uint32_t)r * (uint32_t)(o.ld * 2) + piece * 16;
    } else {
      const int k = at / (kTile / 8), piece = at % (kTile / 8);
      const int f = (k & 3) | ((k >> 1) & 4);
      const int col = (((piece >> 1) ^ f) * 2 + (piece & 1)) * 8;
      off[it] = (uint32_t)min(k, k_left - 1) * (uint32_t)(o.ld * 2) + min(col, o.n - 8 - i0) * 2;
    }
  }
}

// One 16-byte load of every lane, straight into LDS: lane l's piece goes to `to` + 16 l.
// In assembly, because the compiler would wait for every load in flight before each
// transposing read (it cannot tell the two stages apart): 693 TFLOP/s of dw instead of
// %DW%. It has no result register; land() waits for it.
__device__ __forceinline__ void load_lds(uint32_t to, const char* base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(to), "v"(off), "s"(base)
               : "memory");
}

// Waits until at most N of this wave's loads into LDS are in flight.
template <int N>
__device__ __forceinline__ void land() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "i"(N) : "memory");
}

// The order of a block with READS LDS reads and 32 products: a read every product or two.
template <int READS>
__device__ __forceinline__ void interleave() {
  constexpr int kEach = READS > 16 ? 1 : 2;
#pragma unroll
  for (int r = 0; r < READS; ++r) {
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // LDS read
    __builtin_amdgcn_sched_group_barrier(0x008, kEach, 0);  // product
  }
  __builtin_amdgcn_sched_group_barrier(0x008, 32 - READS * kEach, 0);
}

__device__ __forceinline__ void load_stage(uint32_t to, const char* base,
                                           const uint32_t (&off)[kLoads]) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int it = 0; it < kLoads; ++it) load_lds(to + (it * kWaves + wave) * 1024, base, off[it]);
}

// Fragment of 16 rows from i (a multiple of 16) and 32 summed values from 32 * ks:
// lane l holds row l % 16, values 8 (l / 16) ...
template <bool TR>
__device__ __forceinline__ s16x8 fragment(const lds_char* tile, int i, int ks) {
  const int lane = threadIdx.x & 63;
  if (!TR) {
    const int r = lane & 15, piece = ((lane >> 4) + 4 * ks) ^ (r >> 1);
    return *reinterpret_cast<const __attribute__((address_space(3))) s16x8*>(
        tile + (i + r) * (kStep * 2) + piece * 16);
  }
  const int k = 8 * (lane >> 4) + ((lane & 15) >> 2);
  const int f = (k & 3) | ((k >> 1) & 4);
  const lds_char* at = tile + (k + 32 * ks) * (kTile * 2) + (((i >> 4) ^ f) * 32) + (lane & 3) * 8;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)at);
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)(at + 4 * kTile * 2));
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

__device__ __forceinline__ float load_bias(const float* b, int64_t i) { return b[i]; }
__device__ __forceinline__ float load_bias(const uint16_t* b, int64_t i) {
  return __uint_as_float((uint32_t)b[i] << 16);
}
__device__ __forceinline__ void store_out(float* o, float v) { *o = v; }
__device__ __forceinline__ void store_out(uint16_t* o, float v) { *o = (uint16_t)pack2(v, 0.f); }
// Up to four values; `wide`: the place is aligned to four.
__device__ __forceinline__ void store4(float* o, const float* v, bool wide, int left) {
  if (wide && left >= 4) {
    *reinterpret_cast<float4*>(o) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) o[e] = v[e];
  }
}
__device__ __forceinline__ void store4(uint16_t* o, const float* v, bool wide, int left) {
  if (wide && left >= 4) {
    *reinterpret_cast<uint2*>(o) = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) store_out(o + e, v[e]);
  }
}

// The power of two that brings values of up to `top` to at most 2^15 when they are
// divided by it (1 for none, and for what is not finite).
__device__ __forceinline__ float unit_of(float top) {
  const int e = (int)(__float_as_uint(top) >> 23 & 255);
  return e == 0 || e == 255 ? 1.f : __uint_as_float((uint32_t)max(e - 14, 17) << 23);
}

// S; a token without weights has s_c = 0, which counts as S for its gradient.
__device__ __forceinline__ float top_unit(const Meta& meta) {
  return meta.S ? __uint_as_float(meta.S) : 1.f;
}

// What row q of a piece of dw is multiplied with.
template <class T>
__device__ __forceinline__ float dw_scale(const Gemm& g, const Meta& meta, int q) {
  if (!Elem<T>::kScaled) return meta.scale;
  const float top = top_unit(meta), s = g.s[g.c0 + q];
  return (s > 0.f ? top / s : 1.f) * 0x1p-14f * unit_of(__uint_as_float(meta.T));
}

template <int KIND, class T>
__global__ void __launch_bounds__(kThreads, 2) gemm_kernel(const Gemm g) {
  typedef Elem<T> El;
  constexpr bool TP = KIND == kDx || KIND == kDw, TQ = KIND == kDw;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  lds_char* lds = (lds_char*)smem;
  const uint32_t lds_at = (uint32_t)(uintptr_t)lds;
  lds_poison(smem, 2 * kStageBytes);

  const Meta meta = *g.meta;
  // Workgroups go round the eight dies: each gets a run of neighbouring tiles, four
  // of P by all of Q at a time, so that what a die's tiles read meets in its L2.
  const int total = g.tp * g.tq * g.splits, each = (total + 7) / 8;
  int id = (blockIdx.x & 7) * each + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= each || id >= total) return;
  const int split = id / (g.tp * g.tq);
  id -= split * (g.tp * g.tq);
  const int group = id / (4 * g.tq), in = id - group * 4 * g.tq;
  const int wide = min(4, g.tp - group * 4);
  const int tq = in / wide, tp = group * 4 + in % wide;
  const int p0 = tp * kTile, q0 = tq * kTile;
  int k_all = g.k;
  if (KIND == kDw) k_all = min(k_all, (meta.n + kStep - 1) / kStep * kStep);
  else if (q0 >= meta.n) return;
  const int steps_all = k_all / kStep, each_split = (steps_all + g.splits - 1) / g.splits;
  const int first = min(split * each_split, steps_all);
  const int steps = min(each_split, steps_all - first);

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wp = (wave >> 2) * 128, wq = (wave & 3) * 64;
  // lane l holds q = l % 16 and p = 4 (l / 16) ... of each 16 x 16
  const int lq = lane & 15, lp = 4 * (lane >> 4);
  const int c_wave = g.c0 + p0 + wp + lp;  // first token of the lane, of 4 in every 16
  constexpr bool kLogits = KIND == kStats || KIND == kLogitGrad;
  const T* bias = static_cast<const T*>(g.bias);
  f32x4 acc[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (kLogits && !El::kScaled) {
    // sums begin at the bias, and at -inf behind the last token
    if (bias) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          acc[i][0][e] = load_bias(bias, min(c_wave + 16 * i + e, g.C - 1));
    }
    if (g.c0 + p0 + kTile > g.C) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c_wave + 16 * i + e >= g.C) acc[i][0][e] = -__builtin_huge_valf();
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 1; j < 4; ++j) acc[i][j] = acc[i][0];
  }

  uint32_t off_p[kLoads], off_q[kLoads];
  lane_offsets<TP>(g.P, p0, kStep, off_p);
  lane_offsets<TQ>(g.Q, q0, kStep, off_q);
  const char* base_p = (const char*)(g.P.p + (TP ? p0 : p0 * g.P.ld));
  const char* base_q = (const char*)(g.Q.p + (TQ ? q0 : q0 * g.Q.ld));
  const int64_t step_p = TP ? g.P.ld * (kStep * 2) : kStep * 2;
  const int64_t step_q = TQ ? g.Q.ld * (kStep * 2) : kStep * 2;
  auto issue = [&](int s, int buf) {
    const int k = first + s / El::PAIRS, pair = s % El::PAIRS;
    const char* bp = base_p + k * step_p + El::p(pair) * g.P.plane * 2;
    const char* bq = base_q + k * step_q + El::q(pair) * g.Q.plane * 2;
    if (TP && KIND == kDx) {
      // the last tokens: rows of w behind them are not read
      const int left = g.P.kn - k * kStep;
      if (left < kStep) lane_offsets<TP>(g.P, p0, left, off_p);
    }
    load_stage(lds_at + buf * kStageBytes, bp, off_p);
    load_stage(lds_at + buf * kStageBytes + kOperandBytes, bq, off_q);
  };
  // Fragments of one half of a stage are read while the products of the other half run.
  // A stage's second half is in registers before the barrier in its middle, so behind
  // that its place takes the stage after next, whose loads then have a whole stage's
  // time; and no wave waits for LDS right after a barrier.
  s16x8 pa[2][8], qb[2][4];
  auto read = [&](int buf, int half) {
    const lds_char* P = lds + buf * kStageBytes;
    const lds_char* Q = P + kOperandBytes;
#pragma unroll
    for (int j = 0; j < 4; ++j) qb[half][j] = fragment<TQ>(Q, wq + 16 * j, half);
#pragma unroll
    for (int i = 0; i < 8; ++i) pa[half][i] = fragment<TP>(P, wp + 16 * i, half);
  };
  auto multiply = [&](int half) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = El::mfma(pa[half][i], qb[half][j], acc[i][j]);
    interleave<(TP ? 16 : 8) + (TQ ? 8 : 4)>();
  };
  const int n_stage = steps * El::PAIRS;
  if (n_stage > 0) {
    issue(0, 0);
    if (n_stage > 1) {
      issue(1, 1);
      land<2 * kLoads>();
    } else {
      land<0>();
    }
    __syncthreads();
    read(0, 0);
    for (int s = 0; s < n_stage; ++s) {
      read(s & 1, 1);
      multiply(0);
      land<0>();  // the next stage
      __syncthreads();
      if (s + 2 < n_stage) issue(s + 2, s & 1);
      read((s + 1) & 1, 0);  // (behind the last stage nothing uses it)
      multiply(1);
    }
  }

  if (kLogits && El::kScaled) {
    float r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = g.row.r[min(q0 + wq + 16 * j + lq, meta.n - 1)];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = c_wave + 16 * i + e, at = min(c, g.C - 1);
        const float s = g.s[at];
        float add = bias ? load_bias(bias, at) : 0.f;
        if (c >= g.C) add = -__builtin_huge_valf();
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j][e] = acc[i][j][e] * s * r[j] + add;
      }
  }
  if (KIND == kStats) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = q0 + wq + 16 * j + lq;
      // the row's target among the lane's tokens
      const int t = (row < meta.n ? g.row.target[row] : -1) - c_wave;
      const bool mine = t >= 0 && t < 128 && (t & 12) == 0;
      if (__ballot(mine)) {
        float hit = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (t == 16 * i + e) hit = acc[i][j][e];
        if (mine) g.hit[row] = hit;
      }
      float m = -__builtin_huge_valf();
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) m = fmaxf(m, acc[i][j][e]);
      m = fmaxf(m, __shfl_xor(m, 16));
      m = fmaxf(m, __shfl_xor(m, 32));
      // (a NaN among the logits is no maximum, but it is in the sum)
      const float base = m == -__builtin_huge_valf() ? 0.f : m;
      // one rounding for all terms: it moves the log-sum-exp by half a step of m
      const float shift = -base * kLog2e;
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          sum[e] += __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][j][e], kLog2e, shift));
      float all = (sum[0] + sum[1]) + (sum[2] + sum[3]);
      all += __shfl_xor(all, 16);
      all += __shfl_xor(all, 32);
      if (row < meta.n && lane < 16)
        g.part[(int64_t)row * g.n_part + 2 * tp + (wave >> 2)] = make_float2(m, all);
    }
  }
  if (KIND == kLogitGrad) {
    float cs[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) cs[i][e] = 0.f;
    float to_f16[8][4];
    if (El::kScaled) {
      const float top = 0x1p14f / top_unit(meta);
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float s = g.s[min(c_wave + 16 * i + e, g.C - 1)];
          to_f16[i][e] = s > 0.f ? s * top : 0x1p14f;
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = q0 + wq + 16 * j + lq;
      const bool in = row < meta.n;
      const float norm = El::kScaled ? 1.f : meta.inverse;
      const float lse = in ? g.row.lse[row] : 0.f, shift = -lse * kLog2e;
      const float a = in ? g.row.a[row] * norm : 0.f;
      const float m = El::kScaled && in ? g.row.m[row] : 0.f;
      const int t = (in ? g.row.target[row] : -1) - c_wave;
      const bool mine = t >= 0 && t < 128 && (t & 12) == 0;
      // G over the logits
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          // float32: the difference first, whose rounding is small where p is not
          const float z = acc[i][j][e];
          const float p = __builtin_amdgcn_exp2f(El::kScaled ? (z - lse) * kLog2e
                                                             : __builtin_fmaf(z, kLog2e, shift));
          acc[i][j][e] = in ? a * p : 0.f;
        }
      if (__ballot(mine)) {
        const float b = in ? g.row.b[row] * norm : 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (t == 16 * i + e) acc[i][j][e] -= b;
      }
      if (g.col) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) cs[i][e] += El::kScaled ? acc[i][j][e] * m : acc[i][j][e];
      }
      uint16_t* to = g.G + (int64_t)row * g.ldg + p0 + wp + lp;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = El::kScaled ? acc[i][j][e] * to_f16[i][e] : acc[i][j][e];
        uint2 out[El::PLANES];
        El::planes4(v, out);
#pragma unroll
        for (int s = 0; s < El::PLANES; ++s)
          *reinterpret_cast<uint2*>(to + s * g.g_plane + 16 * i) = out[s];
      }
    }
    if (g.col) {
      // the tile's columns: over 16 lanes, then over the four waves through LDS
      float* sums = reinterpret_cast<float*>(smem);  // [4, kTile]
      __syncthreads();  // (the last stage is read)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v = cs[i][e];
          v += __shfl_xor(v, 1);
          v += __shfl_xor(v, 2);
          v += __shfl_xor(v, 4);
          v += __shfl_xor(v, 8);
          cs[i][e] = v;
        }
        if (lq == 0)
          *reinterpret_cast<float4*>(sums + (wave & 3) * kTile + wp + lp + 16 * i) =
              make_float4(cs[i][0], cs[i][1], cs[i][2], cs[i][3]);
      }
      __syncthreads();
      const int c = threadIdx.x;
      if (c < kTile)
        g.col[(int64_t)tq * g.ldg + p0 + c] =
            (sums[c] + sums[kTile + c]) + (sums[2 * kTile + c] + sums[3 * kTile + c]);
    }
  }
  if (KIND == kDx || KIND == kDw) {
    const bool wide = g.ldo % 4 == 0 && (uintptr_t)g.out % (4 * sizeof(T)) == 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int q = q0 + wq + 16 * j + lq;
      if (q >= (KIND == kDx ? meta.n : g.n_q)) continue;
      float scale = 1.f;
      if (KIND == kDw && g.out) scale = dw_scale<T>(g, meta, q);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int d = p0 + wp + 16 * i + lp;
        if (KIND == kDw && g.out) {
          const float v[4] = {acc[i][j][0] * scale, acc[i][j][1] * scale, acc[i][j][2] * scale,
                              acc[i][j][3] * scale};
          store4(static_cast<T*>(g.out) + q * g.ldo + d, v, wide, g.D - d);
        } else if (d < g.lda) {
          f32x4* o = reinterpret_cast<f32x4*>(g.acc + split * g.acc_split + (int64_t)q * g.lda + d);
          *o = g.add ? *o + acc[i][j] : acc[i][j];
        }
      }
    }
  }
}

template <int KIND, class T>
hipError_t launch(const Gemm& g, hipStream_t st) {
  const int64_t total = (int64_t)g.tp * g.tq * g.splits;
  if (total <= 0) return hipSuccess;
  const int64_t grid = up(total, 8);
  if (grid > most_groups(kThreads)) return hipErrorInvalidValue;
  (void)hipFuncSetAttribute(reinterpret_cast<const void*>(&gemm_kernel<KIND, T>),
                            hipFuncAttributeMaxDynamicSharedMemorySize, 2 * kStageBytes);
  gemm_kernel<KIND, T><<<dim3((unsigned)grid), dim3(kThreads), 2 * kStageBytes, st>>>(g);
  return hipGetLastError();
}

}  // namespace linear
}  // namespace tbias
