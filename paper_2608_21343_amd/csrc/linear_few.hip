// Logits of few rows: their statistics, and where they are kept the logits themselves.
//
// With up to 64 rows (32 in bfloat16) a layer's weights are read once and hardly used
// again, so the time is that of reading them. A wave takes up to 16, 32 or 64 rows and its
// share of the tokens, 64 at a time, straight from memory into the operands of the matrix
// instructions: no LDS, no barriers, and every wave keeps several steps of loads in
// flight. Waves begin at different places of their rows: in step they would ask for the
// same part of every row, which the same memory channels hold (8 rows of 1024 bfloat16
// against 131,073 tokens 57 us, 45 so; 268 MB at 6.0 TB/s, 4.9 with nothing of them in a
// cache). Tokens are dealt out in units of 16: tiles of 256 took three rounds of the card's
// CUs for little more than two rounds' worth. Layers of few tokens have a wave for each 16 of
// them, with up to eight steps of loads in flight.
//
// float32 operands are taken apart into three bfloat16 planes in registers (x, the
// rounding of what x leaves, and once more): six products of them, to 2^-26 of the
// whole, which the matrix cores do in the time of the loads; and no scale has to be known
// before the weights are read.
#include "linear_gemm.hpp"

namespace tbias {
namespace linear {

namespace {

constexpr int kFrag = 16;  // tokens of a fragment

// Eight values along the width, as loaded and as planes.
template <class T>
struct Eight;
template <>
struct Eight<uint16_t> {
  static constexpr int PLANES = 1;
  uint4 v;
  __device__ inline void load(const uint16_t* p, bool in) {
    v = in ? *reinterpret_cast<const uint4*>(p) : make_uint4(0, 0, 0, 0);
  }
  __device__ inline void planes(bf16x8* out) const { out[0] = __builtin_bit_cast(bf16x8, v); }
};
template <>
struct Eight<float> {
  static constexpr int PLANES = 3;
  float4 a, b;
  __device__ inline void load(const float* p, bool in) {
    a = in ? reinterpret_cast<const float4*>(p)[0] : make_float4(0.f, 0.f, 0.f, 0.f);
    b = in ? reinterpret_cast<const float4*>(p)[1] : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  __device__ inline void planes(bf16x8* out) const {
    float r[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int s = 0; s < 3; ++s) {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        w[e] = pack2(r[2 * e], r[2 * e + 1]);
        r[2 * e] -= low16(w[e]);
        r[2 * e + 1] -= high16(w[e]);
      }
      out[s] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
    }
  }
};

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

// kP fragments of tokens and NQ of rows at a time.
template <class T, int kP, int NQ>
__global__ void __launch_bounds__(256) few_kernel(const Few f) {
  constexpr int PL = Eight<T>::PLANES;
  constexpr int kSets = kP == 1 ? (PL == 1 ? 8 : 4) : PL == 1 && NQ == 1 ? 4 : 2;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (wave >= f.parts) return;
  const int row0 = blockIdx.y * (NQ * 16);
  const int lq = lane & 15, lk = 8 * (lane >> 4), lp = 4 * (lane >> 4);
  const int64_t units = (f.C + kFrag - 1) / kFrag;
  const int first = wave * f.each, last = (int)min(units, (int64_t)first + f.each);
  const int steps = (f.D + 31) / 32, start = (5 * wave) % steps;
  const T* x[NQ];
  int target[NQ];
  float top[NQ], sum[NQ];
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    const int row = row0 + 16 * q + lq;
    x[q] = static_cast<const T*>(f.x) + min(row, f.n - 1) * f.x_stride + lk;
    target[q] = row < f.n ? f.target[row] : -1;
    top[q] = -__builtin_huge_valf();
    sum[q] = 0.f;
  }
  for (int unit = first; unit < last; unit += kP) {
    const int c0 = unit * kFrag, end = min(f.C, last * kFrag);  // the wave's tokens
    const T* w[kP];
#pragma unroll
    for (int p = 0; p < kP; ++p)
      w[p] = static_cast<const T*>(f.w) + min(c0 + 16 * p + lq, end - 1) * f.w_stride + lk;
    // (the products of lower planes, or every other step's of up to 16 bfloat16 rows, on their
    // own: in one sum all would round at the size of the whole. Losses of sums of 1536 float32
    // values are off by 6e-7 so, by 1.5e-6 in one sum, in the same time; the second sum of more
    // bfloat16 rows took a tenth longer, 67 us of 61, for its registers.)
    f32x4 acc[kP][NQ], low[kP][NQ];
#pragma unroll
    for (int p = 0; p < kP; ++p)
#pragma unroll
      for (int q = 0; q < NQ; ++q) acc[p][q] = low[p][q] = f32x4{0.f, 0.f, 0.f, 0.f};
    Eight<T> a[kSets][kP], b[kSets][NQ];
    auto load = [&](int set, int step) {
      // every wave begins at another place of its rows
      int at = step + start;
      at = at >= steps ? at - steps : at;
      const int k = 32 * at;
      const bool in = step < steps && k + lk < f.D;
#pragma unroll
      for (int p = 0; p < kP; ++p) a[set][p].load(w[p] + (in ? k : 0), in);
#pragma unroll
      for (int q = 0; q < NQ; ++q) b[set][q].load(x[q] + (in ? k : 0), in);
    };
    auto multiply = [&](int set) {
      bf16x8 y[NQ][PL];
#pragma unroll
      for (int q = 0; q < NQ; ++q) b[set][q].planes(y[q]);
#pragma unroll
      for (int p = 0; p < kP; ++p) {
        bf16x8 v[PL];
        a[set][p].planes(v);
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          if constexpr (PL == 3) {
            low[p][q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[2], y[q][0], low[p][q], 0, 0, 0);
            low[p][q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[0], y[q][2], low[p][q], 0, 0, 0);
            low[p][q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[1], y[q][1], low[p][q], 0, 0, 0);
            low[p][q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[1], y[q][0], low[p][q], 0, 0, 0);
            low[p][q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[0], y[q][1], low[p][q], 0, 0, 0);
          }
          f32x4& sum = PL == 1 && NQ == 1 && set % 2 ? low[p][q] : acc[p][q];
          sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[0], y[q][0], sum, 0, 0, 0);
        }
      }
    };
#pragma unroll
    for (int s = 0; s < kSets; ++s) load(s, s);
    for (int k = 0; k < steps; k += kSets)
#pragma unroll
      for (int s = 0; s < kSets; ++s) {
        multiply(s);
        load(s, k + s + kSets);
      }
    const T* bias = static_cast<const T*>(f.bias);
#pragma unroll
    for (int p = 0; p < kP; ++p)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = c0 + 16 * p + lp + e;
        const float add = bias ? to_float(bias[min(c, f.C - 1)]) : 0.f;
#pragma unroll
        for (int q = 0; q < NQ; ++q)
          acc[p][q][e] = c < end ? acc[p][q][e] + low[p][q][e] + add : -__builtin_huge_valf();
      }
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int row = row0 + 16 * q + lq;
      float m = top[q];
#pragma unroll
      for (int p = 0; p < kP; ++p)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          m = fmaxf(m, acc[p][q][e]);
          if (c0 + 16 * p + lp + e == target[q]) f.hit[row] = acc[p][q][e];
        }
      // (a NaN among the logits is no maximum, but it is in the sum)
      const float base = m == -__builtin_huge_valf() ? 0.f : m;
      float s = sum[q] * __builtin_amdgcn_exp2f((top[q] - base) * kLog2e);
#pragma unroll
      for (int p = 0; p < kP; ++p)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          s += __builtin_amdgcn_exp2f((acc[p][q][e] - base) * kLog2e);
      top[q] = m;
      sum[q] = s;
      if (f.z && row < f.n) {
#pragma unroll
        for (int p = 0; p < kP; ++p)
          if (c0 + 16 * p < end)
            *reinterpret_cast<f32x4*>(f.z + (int64_t)row * f.ldz + c0 + 16 * p + lp) = acc[p][q];
      }
    }
  }
  // the four lanes of a row
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
#pragma unroll
    for (int d = 16; d < 64; d <<= 1) {
      const float m2 = __shfl_xor(top[q], d), s2 = __shfl_xor(sum[q], d), m = fmaxf(top[q], m2);
      const float base = m == -__builtin_huge_valf() ? 0.f : m;
      sum[q] = sum[q] * __builtin_amdgcn_exp2f((top[q] - base) * kLog2e) +
               s2 * __builtin_amdgcn_exp2f((m2 - base) * kLog2e);
      top[q] = m;
    }
    const int row = row0 + 16 * q + lq;
    if (lane < 16 && row < f.n)
      f.part[(int64_t)row * f.parts + wave] = make_float2(top[q], sum[q]);
  }
}

template <class T, int kP, int NQ>
void launch_few(const Few& f, hipStream_t st) {
  few_kernel<T, kP, NQ>
      <<<dim3((f.parts + 3) / 4, (f.n + 16 * NQ - 1) / (16 * NQ)), dim3(256), 0, st>>>(f);
}

// More than 32 float32 rows: all of a wave with many tokens, or by 32 of twice as many waves
// (64 rows of 1024 against 131,073 tokens 217 us and 241; of 512 against 4097 27 and 19).
template <class T, int kP>
void few_t(const Few& f, hipStream_t st) {
  if (f.n <= 16) return launch_few<T, kP, 1>(f, st);
  if constexpr (sizeof(T) == 4 && kP == 4) {
    if (f.n > 32) return launch_few<T, kP, 4>(f, st);
  }
  launch_few<T, kP, 2>(f, st);
}

}  // namespace

// A unit a wave where there are no more than 16 waves a CU of them; else a multiple of the
// four that a wave takes at a time, with up to 12 waves a CU.
constexpr int32_t kMost = 12 * 256;
int32_t few_each(int32_t C) {
  const int32_t units = (C + kFrag - 1) / kFrag;
  return units <= 4096 ? 1 : 4 * ((units + 4 * kMost - 1) / (4 * kMost));
}

int32_t few_parts(int32_t C) {
  const int32_t units = (C + kFrag - 1) / kFrag, each = few_each(C);
  return (units + each - 1) / each;
}

hipError_t few(const Few& f, int32_t dtype, hipStream_t st) {
  if (dtype == TB_F32) f.each == 1 ? few_t<float, 1>(f, st) : few_t<float, 4>(f, st);
  else f.each == 1 ? few_t<uint16_t, 1>(f, st) : few_t<uint16_t, 4>(f, st);
  return hipGetLastError();
}

}  // namespace linear
}  // namespace tbias
