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
typedef __attribute__((ext_vector_type(4))) short s16x4;
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

// The planes of four values.
template <int PLANES>
__device__ __forceinline__ void planes4(const float* v, uint2* out) {
  float r[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
  for (int s = 0; s < PLANES; ++s) {
    out[s] = make_uint2(pack2(r[0], r[1]), pack2(r[2], r[3]));
    if (s + 1 < PLANES) {
      r[0] -= low16(out[s].x);
      r[1] -= high16(out[s].x);
      r[2] -= low16(out[s].y);
      r[3] -= high16(out[s].y);
    }
  }
}

// The pairs of planes that are multiplied, the largest products last.
template <int PLANES>
struct Pairs;
template <>
struct Pairs<1> {
  static constexpr int N = 1;
  __device__ static inline int p(int) { return 0; }
  __device__ static inline int q(int) { return 0; }
};
template <>
struct Pairs<3> {
  static constexpr int N = 6;  // (2,0) (0,2) (1,1) (1,0) (0,1) (0,0)
  __device__ static inline int p(int s) { return (0x52 >> (2 * s)) & 3; }
  __device__ static inline int q(int s) { return (0x118 >> (2 * s)) & 3; }
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

__device__ __forceinline__ void load_stage(lds_char* to, const char* base,
                                           const uint32_t (&off)[kLoads]) {
  const int wave = threadIdx.x >> 6;
#pragma unroll
  for (int it = 0; it < kLoads; ++it)
    __builtin_amdgcn_global_load_lds(
        (const __attribute__((address_space(1))) void*)(base + off[it]),
        (__attribute__((address_space(3))) void*)(to + (it * kWaves + wave) * 1024), 16, 0, 0);
}

// Fragment of 16 rows from i (a multiple of 16) and 32 summed values from 32 * ks:
// lane l holds row l % 16, values 8 (l / 16) ...
template <bool TR>
__device__ __forceinline__ bf16x8 fragment(const lds_char* tile, int i, int ks) {
  const int lane = threadIdx.x & 63;
  if (!TR) {
    const int r = lane & 15, piece = ((lane >> 4) + 4 * ks) ^ (r >> 1);
    return *reinterpret_cast<const __attribute__((address_space(3))) bf16x8*>(
        tile + (i + r) * (kStep * 2) + piece * 16);
  }
  const int k = 8 * (lane >> 4) + ((lane & 15) >> 2);
  const int f = (k & 3) | ((k >> 1) & 4);
  const lds_char* at = tile + (k + 32 * ks) * (kTile * 2) + (((i >> 4) ^ f) * 32) + (lane & 3) * 8;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)at);
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)(at + 4 * kTile * 2));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

__device__ __forceinline__ float load_bias(const float* b, int64_t i) { return b[i]; }
__device__ __forceinline__ float load_bias(const uint16_t* b, int64_t i) {
  return __uint_as_float((uint32_t)b[i] << 16);
}
__device__ __forceinline__ void store_out(float* o, float v) { *o = v; }
__device__ __forceinline__ void store_out(uint16_t* o, float v) { *o = (uint16_t)pack2(v, 0.f); }

template <int KIND, class T>
__global__ void __launch_bounds__(kThreads, 2) gemm_kernel(const Gemm g) {
  constexpr int PLANES = sizeof(T) == 4 ? 3 : 1;
  typedef Pairs<PLANES> Pr;
  constexpr bool TP = KIND == kDx || KIND == kDw, TQ = KIND == kDw;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  lds_char* lds = (lds_char*)smem;
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
  f32x4 acc[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  uint32_t off_p[kLoads], off_q[kLoads];
  lane_offsets<TP>(g.P, p0, kStep, off_p);
  lane_offsets<TQ>(g.Q, q0, kStep, off_q);
  const char* base_p = (const char*)(g.P.p + (TP ? p0 : p0 * g.P.ld));
  const char* base_q = (const char*)(g.Q.p + (TQ ? q0 : q0 * g.Q.ld));
  const int64_t step_p = TP ? g.P.ld * (kStep * 2) : kStep * 2;
  const int64_t step_q = TQ ? g.Q.ld * (kStep * 2) : kStep * 2;
  auto issue = [&](int s, int buf) {
    const int k = first + s / Pr::N, pair = s % Pr::N;
    const char* bp = base_p + k * step_p + Pr::p(pair) * g.P.plane * 2;
    const char* bq = base_q + k * step_q + Pr::q(pair) * g.Q.plane * 2;
    if (TP && KIND == kDx) {
      // the last tokens: rows of w behind them are not read
      const int left = g.P.kn - k * kStep;
      if (left < kStep) lane_offsets<TP>(g.P, p0, left, off_p);
    }
    load_stage(lds + buf * kStageBytes, bp, off_p);
    load_stage(lds + buf * kStageBytes + kOperandBytes, bq, off_q);
  };
  const int n_stage = steps * Pr::N;
  if (n_stage > 0) issue(0, 0);
  for (int s = 0; s < n_stage; ++s) {
    __syncthreads();  // stage s has landed, and the other buffer is read
    if (s + 1 < n_stage) issue(s + 1, (s + 1) & 1);
    const lds_char* P = lds + (s & 1) * kStageBytes;
    const lds_char* Q = P + kOperandBytes;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      bf16x8 b[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) b[j] = fragment<TQ>(Q, wq + 16 * j, ks);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bf16x8 a = fragment<TP>(P, wp + 16 * i, ks);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b[j], acc[i][j], 0, 0, 0);
      }
    }
  }

  // lane l holds q = l % 16 and p = 4 (l / 16) ... of each 16 x 16
  const int lq = lane & 15, lp = 4 * (lane >> 4);
  if (KIND == kStats || KIND == kLogitGrad) {
    const T* bias = static_cast<const T*>(g.bias);
    const int c_wave = g.c0 + p0 + wp + lp;
    const bool last = g.c0 + p0 + kTile > g.C;
    if (bias) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float add = load_bias(bias, min(c_wave + 16 * i + e, g.C - 1));
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][j][e] += add;
        }
    }
    if (last) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c_wave + 16 * i + e >= g.C) {
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j][e] = -__builtin_huge_valf();
          }
    }
  }
  if (KIND == kStats) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = q0 + wq + 16 * j + lq;
      const int t = row < meta.n ? g.row.target[row] : -1;
      const int c_wave = g.c0 + p0 + wp + lp;
      float m = -__builtin_huge_valf(), hit = 0.f;
      bool mine = false, nan = false;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float z = acc[i][j][e];
          m = fmaxf(m, z);
          nan |= z != z;
          if (c_wave + 16 * i + e == t) {
            hit = z;
            mine = true;
          }
        }
      m = fmaxf(m, __shfl_xor(m, 16));
      m = fmaxf(m, __shfl_xor(m, 32));
      const float base = m == -__builtin_huge_valf() ? 0.f : m;
      float sum = nan ? __builtin_nanf("") : 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          sum += __builtin_amdgcn_exp2f((acc[i][j][e] - base) * kLog2e);
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (row < meta.n) {
        if (lane < 16) g.part[(int64_t)row * g.n_part + 2 * tp + (wave >> 2)] = make_float2(m, sum);
        if (mine) g.hit[row] = hit;
      }
    }
  }
  if (KIND == kLogitGrad) {
    float cs[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) cs[i][e] = 0.f;
    const int c_wave = g.c0 + p0 + wp + lp;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = q0 + wq + 16 * j + lq;
      const bool in = row < meta.n;
      const float lse = in ? g.row.lse[row] : 0.f;
      const float a = in ? g.row.a[row] * meta.inverse : 0.f;
      const float b = in ? g.row.b[row] * meta.inverse : 0.f;
      const int t = in ? g.row.target[row] : -1;
      uint16_t* to = g.G + (int64_t)row * g.ldg + p0 + wp + lp;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f((acc[i][j][e] - lse) * kLog2e);
          const int c = c_wave + 16 * i + e;
          v[e] = in && c < g.C ? a * p - (c == t ? b : 0.f) : 0.f;
          cs[i][e] += v[e];
        }
        uint2 out[PLANES];
        planes4<PLANES>(v, out);
#pragma unroll
        for (int s = 0; s < PLANES; ++s)
          *reinterpret_cast<uint2*>(to + s * g.g_plane + 16 * i) = out[s];
      }
    }
    if (g.col) {
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
          *reinterpret_cast<float4*>(g.col + (int64_t)(4 * tq + (wave & 3)) * g.ldg + p0 + wp + lp +
                                     16 * i) =
              make_float4(cs[i][0], cs[i][1], cs[i][2], cs[i][3]);
      }
    }
  }
  if (KIND == kDx || KIND == kDw) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int q = q0 + wq + 16 * j + lq;
      if (q >= (KIND == kDx ? meta.n : g.n_q)) continue;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int d = p0 + wp + 16 * i + lp;
        if (KIND == kDw && g.out) {
          T* o = static_cast<T*>(g.out) + q * g.ldo + d;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (d + e < g.D) store_out(o + e, acc[i][j][e] * meta.scale);
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
