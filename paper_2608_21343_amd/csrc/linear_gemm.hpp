// The products of the linear cross entropy: tiles of N x N (256, 128 or 64) by eight waves
// of N / 2 x N / 4, sums of 16 x 16 x 32 matrix instructions in registers, operands staged
// through LDS by asynchronous 16-byte loads, 512 / N stages of 64 values of the summed axis
// (two planes: of 32).
//
// What bounds them is the matrix instructions. In tiles of 256 they are busy two thirds of
// the time of a long sum (rocprofv3: 0.64 to 0.67 of all pipes' cycles, no bank conflicts in
// LDS), at clocks that the card lowers to 1.6 to 1.8 GHz under such work. bfloat16 products
// for 4096 rows of 2048 against 131,073 tokens, traced: statistics 1.69 ms (1300 TFLOP/s; a
// library product of that size 1380), dx 1.82, dw 1.71, gradients of the logits 1.87; float32 ones
// of 2048 x 1024 against 32,769 at 1060 to 1220 TFLOP/s of planes in a traced pass, which is
// a seventh longer than an untraced one. The statistics of a short sum (640 values) spend nearly
// half of their time in the exponentials: 32,768 rows, a tenth left out, against 8193 tokens
// 313 us traced, 990 TFLOP/s (untraced the whole call takes 316).
//
// A CU holds one workgroup: the sums of a tile of 256 take half of a wave's registers, and
// smaller tiles have more stages in the same 128 KB of LDS. In tiles of 128 the LDS reads of
// the fragments take as long as the products.
//
// An operand whose rows run along the summed axis lies in LDS as [row, 64] with its
// 16-byte pieces exchanged by row, so that the 16 rows of a fragment's read cover
// all banks once. One whose rows run across it lies as [64, column] with its 32-byte
// pieces exchanged, and is read through the transposing LDS read.
#pragma once

#include <cstddef>

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
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((address_space(3))) char lds_char;

constexpr int kWaves = 8, kThreads = 64 * kWaves;

// A tile of N x N, by waves of N / 2 x N / 4, and its stages in LDS.
template <int N>
struct Tiling {
  static constexpr int FP = N / 32, FQ = N / 64;             // fragments of 16 of a wave
  static constexpr int kLoads = N / 64;                      // of a lane, for a stage of an operand
  static constexpr int kOperandBytes = N * kStep * 2, kStageBytes = 2 * kOperandBytes;
  static constexpr int kStages = 512 / N;                    // 128 KB of them
  static constexpr int kSets = kStages + 1;                  // of Params
  static constexpr int kParamBytes = 7 * N * 4, kColBytes = 4 * N * 4;
  static constexpr int kLdsBytes = kStages * kStageBytes + kSets * kParamBytes + kColBytes;
};

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
__device__ __forceinline__ float low16(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float high16(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }

// An operand of one type: its planes, and the matrix instruction.
template <class T>
struct Elem;
template <>
struct Elem<uint16_t> {
  static constexpr int PLANES = 1;
  static constexpr bool kScaled = false;
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
  static constexpr int PLANES = 2;
  static constexpr bool kScaled = true;
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

// A lane's first 16-byte load of a stage: the stage's row that it fills and where in a row
// of the operand's memory it comes from, in bytes. The next ones fill rows kNextRows further
// on. Stage rows are the operand's own rows, or (transposed) the summed values: 64, or 32
// of the first plane and the same 32 of the second.
template <int N, bool TR, int PLANES>
struct Lane {
  static constexpr int kNextRows = TR ? kWaves * 512 / N : kWaves * 8;
  static constexpr int kK = TR ? kStep / PLANES : N;  // rows of the operand of a stage
  int row;
  uint32_t bytes;
  // of load `it`, `rows` rows being in memory
  __device__ inline uint32_t at(int it, uint32_t row_bytes, int rows) const {
    return (uint32_t)min((row + it * kNextRows) & (kK - 1), rows - 1) * row_bytes + bytes +
           it * kNextRows / kK * (kTurn * 2);
  }
};

// By how much the 32-byte pieces of row k of a transposed operand's stage are exchanged:
// the eight rows that half a wave reads at once then lie in different banks (rows of 64
// values fill half of the banks, two of them all).
template <int N>
__device__ __forceinline__ int turn_of(int k) {
  return N >= 128 ? (k & 3) | ((k >> 1) & 4) : ((k >> 1) & 1) | ((k >> 2) & 2);
}

template <int N, bool TR, int PLANES>
__device__ __forceinline__ Lane<N, TR, PLANES> lane_of(const Operand& o, int32_t i0) {
  const int at = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 64 + (threadIdx.x & 63);
  if (!TR) {
    const int row = at >> 3;
    return {row, (uint32_t)((at & 7) ^ ((row >> 1) & 7)) * 16};
  }
  const int k = at / (N / 8), piece = at % (N / 8);
  const int col = min((((piece >> 1) ^ turn_of<N>(k)) * 2 + (piece & 1)) * 8, o.n - 8 - i0);
  return {k, (uint32_t)(place<PLANES>(col) + k / (kStep / PLANES) * kTurn) * 2};
}

// An address that is the same in every lane, in scalar registers.
__device__ __forceinline__ const char* uniform(const void* p) {
  const uint64_t a = (uint64_t)(uintptr_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
  return (const char*)(uintptr_t)((uint64_t)hi << 32 | lo);
}

// One 16-byte load of every lane, straight into LDS: lane l's piece goes to `to` + 16 l.
// In assembly, because the compiler would wait for every load in flight before each
// transposing read (it cannot tell the two stages apart): 693 TFLOP/s of dw instead of
// 880. It has no result register; land() waits for it.
__device__ __forceinline__ void load_lds(uint32_t to, const char* base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(to), "v"(off), "s"(base)
               : "memory");
}

// The same of one float, or one bfloat16 in the low half of a word, a lane.
__device__ __forceinline__ void load_lds4(uint32_t to, const char* base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
               :
               : "s"(to), "v"(off), "s"(base)
               : "memory");
}
__device__ __forceinline__ void load_lds2(uint32_t to, const char* base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_ushort %1, %2"
               :
               : "s"(to), "v"(off), "s"(base)
               : "memory");
}

// Waits until at most N of this wave's loads into LDS are in flight.
template <int N>
__device__ __forceinline__ void land() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "i"(N) : "memory");
}

// The order of a block with READS LDS reads and MUL products: a read every product or two.
template <int READS, int MUL>
__device__ __forceinline__ void interleave() {
  constexpr int kEach = 2 * READS <= MUL ? 2 : 1;
#pragma unroll
  for (int r = 0; r < READS; ++r) {
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // LDS read
    __builtin_amdgcn_sched_group_barrier(0x008, kEach, 0);  // product
  }
  if (MUL > READS * kEach) __builtin_amdgcn_sched_group_barrier(0x008, MUL - READS * kEach, 0);
}

// The same of FP x FQ products, column by column, while FP fragments of RP reads and FQ of
// RQ are read, these each in the place of its column's.
template <int FP, int RP, int FQ, int RQ>
__device__ __forceinline__ void interleave_columns() {
  static_assert(FP == 2 * FQ, "two fragments of P a column");
#pragma unroll
  for (int j = 0; j < FQ; ++j) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, FP / 2, 0);  // products
      __builtin_amdgcn_sched_group_barrier(0x100, RP, 0);      // LDS reads
    }
    __builtin_amdgcn_sched_group_barrier(0x100, RQ, 0);
  }
}

// A stage of an operand from `base`, off: of the lane's first load. `rows` of it are in
// memory; the others are read as the last of them.
template <int N, bool TR, int PLANES>
__device__ __forceinline__ void load_stage(uint32_t to, const uint16_t* base, uint32_t off,
                                           const Operand& o, int32_t i0, int32_t rows) {
  typedef Lane<N, TR, PLANES> La;
  constexpr int kLoads = Tiling<N>::kLoads;
  to += __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 1024;
  if (rows >= La::kK) {
    const char* from = uniform(base);
#pragma unroll
    for (int it = 0; it < kLoads; ++it) {
      constexpr int kNext = La::kNextRows;
      load_lds(to + it * kWaves * 1024,
               from + (int64_t)(it * kNext % La::kK) * 2 * o.ld + it * kNext / La::kK * (kTurn * 2),
               off);
    }
  } else {
    const La l = lane_of<N, TR, PLANES>(o, i0);
#pragma unroll
    for (int it = 0; it < kLoads; ++it)
      load_lds(to + it * kWaves * 1024, uniform(base), l.at(it, (uint32_t)(o.ld * 2), rows));
  }
}

// Fragment of 16 rows from i (a multiple of 16) and the ks-th 32 values of a stage (two
// planes: the ks-th plane): lane l holds row l % 16, values 8 (l / 16) ...
template <int N, bool TR>
__device__ __forceinline__ s16x8 fragment(const lds_char* tile, int i, int ks, int lane) {
  if (!TR) {
    const int r = lane & 15, piece = ((lane >> 4) + 4 * ks) ^ (r >> 1);
    return *reinterpret_cast<const __attribute__((address_space(3))) s16x8*>(
        tile + (i + r) * (kStep * 2) + piece * 16);
  }
  const int k = 8 * (lane >> 4) + ((lane & 15) >> 2);
  const lds_char* at =
      tile + (k + 32 * ks) * (N * 2) + (((i >> 4) ^ turn_of<N>(k)) * 32) + (lane & 3) * 8;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)at);
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)(at + 4 * N * 2));
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
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

// Of four blocks of 16 values, of which a lane holds a quarter each (four values: lanes
// l, l + 16, l + 32, l + 48 hold the first to the last), the lane's own block whole: the
// l / 16-th. Stores of 32 bytes a lane fill whole lines; of 8 bytes, as the products
// leave them, they took half as long again as the products of a piece.
__device__ __forceinline__ void gather16(uint2 a, uint2 b, uint2 c, uint2 d, uint4* lo, uint4* hi) {
  auto transpose = [](uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3, uint32_t* t) {
    const u32x2 x = __builtin_amdgcn_permlane32_swap(r0, r2, false, false);
    const u32x2 y = __builtin_amdgcn_permlane32_swap(r1, r3, false, false);
    const u32x2 v = __builtin_amdgcn_permlane16_swap(x[0], y[0], false, false);
    const u32x2 w = __builtin_amdgcn_permlane16_swap(x[1], y[1], false, false);
    t[0] = v[0], t[1] = v[1], t[2] = w[0], t[3] = w[1];
  };
  uint32_t x[4], y[4];
  transpose(a.x, b.x, c.x, d.x, x);
  transpose(a.y, b.y, c.y, d.y, y);
  *lo = make_uint4(x[0], y[0], x[1], y[1]);
  *hi = make_uint4(x[2], y[2], x[3], y[3]);
}

// What sums are multiplied with: by 2^e. Units may be as large or small as their values, so
// a product of two of them could leave float32's range where the result does not.
struct Scale {
  float by;
  int e;
};
__device__ __forceinline__ int exponent_of(float unit) {  // of a power of two
  return (int)(__float_as_uint(unit) >> 23 & 255) - 127;
}
__device__ __forceinline__ float power_of(int e) {
  return __uint_as_float((uint32_t)(e + 127) << 23);
}
template <class T>
__device__ __forceinline__ float scaled(float v, const Scale& s) {
  return Elem<T>::kScaled ? __builtin_amdgcn_ldexpf(v * s.by, s.e) : v * s.by;
}

// Of dw.
template <class T>
__device__ __forceinline__ Scale dw_scale(const Meta& meta) {
  if (!Elem<T>::kScaled) return {meta.scale, 0};
  return {1.f, exponent_of(unit_of(__uint_as_float(meta.T))) - 14};
}

// Of gathered row q of dx.
template <class T>
__device__ __forceinline__ Scale dx_scale(const Gemm& g, const Meta& meta, int64_t q) {
  if (!Elem<T>::kScaled) return {meta.scale, 0};
  const float m = g.row.m[q];
  return {__builtin_amdgcn_frexp_mantf(m),
          __builtin_amdgcn_frexp_expf(m) + exponent_of(meta.S) - 14};
}

// exp(z - base) = 2^(z log2(e) + by) (1 + off): the exponent by one operation, and the
// rounding of `by`, the same for all z, once for their sum. far: the product with log2(e)
// might overflow, so base has to be taken from z before (by and off are 0).
struct Shift {
  float by, off;
  bool far;
};
__device__ __forceinline__ Shift shift_of(float base) {
  const bool far = fabsf(base) > 0x1p100f;
  const float by = far ? 0.f : -base * kLog2e;
  return {by, far ? 0.f : __builtin_fmaf(-base, kLog2e, -by) * kLn2, far};
}

// Per token and row of a tile, kept in LDS for the epilogue.
template <int N>
struct Params {
  uint32_t bias[N];  // float32, or bfloat16 in the low half
  int32_t target[N];
  float lse[N], a[N], b[N], r[N], m[N];
};
constexpr int kGroupP = 4;  // tiles of P that a run takes by all of Q

// A workgroup per CU works through tiles of N x N. The stages of its tiles are one
// sequence: the first ones of the next tile are loaded while the present one's last
// products and its epilogue run.
template <int KIND, class T, int N>
__global__ void __launch_bounds__(kThreads, 2) gemm_kernel(const Gemm g) {
  typedef Elem<T> El;
  constexpr int PL = El::PLANES, kK = kStep / PL;  // summed values of a stage
  constexpr bool TP = KIND == kDx || KIND == kDw, TQ = KIND == kDw;
  constexpr bool kLogits = KIND == kStats || KIND == kLogitGrad;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  lds_char* lds = (lds_char*)smem;
  const uint32_t lds_at = (uint32_t)(uintptr_t)lds;
  typedef Tiling<N> Ti;
  constexpr int FP = Ti::FP, FQ = Ti::FQ, kStages = Ti::kStages, kSets = Ti::kSets;
  static_assert(sizeof(Params<N>) == Ti::kParamBytes, "parameters in LDS");
  Params<N>* params = reinterpret_cast<Params<N>*>(smem + kStages * Ti::kStageBytes);
  lds_poison(smem, Ti::kLdsBytes);

  const Meta meta = *g.meta;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wp = (wave >> 2) * (N / 2), wq = (wave & 3) * (N / 4);

  // Workgroups go round the eight dies: each die has a run of neighbouring tiles, four of P
  // by all of Q at a time, so that what its workgroups read meets in its L2.
  const int tiles_q = KIND == kDw ? g.tq : min(g.tq, (meta.n + N - 1) / N);
  const int tiles = g.tp * tiles_q, total = tiles * g.splits, each = (total + 7) / 8;
  const int stride = gridDim.x >> 3, end = min(((int)(blockIdx.x & 7) + 1) * each, total);
  const int begin = (blockIdx.x & 7) * each + (blockIdx.x >> 3);
  int steps_all = g.k / kK;
  if (KIND == kDw) steps_all = min(steps_all, (meta.n + kK - 1) / kK);
  const int steps_each =
      __builtin_amdgcn_readfirstlane((steps_all + g.splits - 1) / g.splits);
  struct Tile {
    int p, q, split, first, steps;
  };
  auto tile_of = [&](int id) {
    Tile t;
    // (quotients come from vector instructions)
    t.split = __builtin_amdgcn_readfirstlane(id / tiles);
    id -= t.split * tiles;
    const int group = __builtin_amdgcn_readfirstlane(id / (kGroupP * tiles_q));
    const int in = id - group * kGroupP * tiles_q, wide = min(kGroupP, g.tp - group * kGroupP);
    t.q = __builtin_amdgcn_readfirstlane(in / wide);
    t.p = group * kGroupP + in - t.q * wide;
    t.first = min(t.split * steps_each, steps_all);
    t.steps = min(steps_each, steps_all - t.first);
    return t;
  };

  // the sequence of stages that are loaded
  int load_id = begin - stride, load_s = 0, load_n = 0;
  Tile load_tile = {};
  uint32_t off_p = 0, off_q = 0;
  int load_turn = 0;
  // What the epilogue needs, one token or row a lane. A tile's are loaded with its first
  // stage: up to kStages tiles ahead (tiles of one stage), when every wave has left the
  // epilogue before the present tile. So kStages + 1 sets are enough.
  auto load_params = [&](const Tile& t, int turn) {
    const uint32_t to = lds_at + kStages * Ti::kStageBytes + turn * sizeof(Params<N>);
    auto four = [&](const void* from, uint32_t index, uint32_t at) {
      load_lds4(to + at, (const char*)from, 4 * index);
    };
    constexpr int kPer = N / 64;
    if (wave < kPer) {
      const uint32_t c = min(g.c0 + t.p * N + 64 * wave + lane, g.C - 1), at = 256 * wave;
      if (g.bias && sizeof(T) == 4) four(g.bias, c, offsetof(Params<N>, bias) + at);
      if (g.bias && sizeof(T) == 2)
        load_lds2(to + offsetof(Params<N>, bias) + at, (const char*)g.bias, 2 * c);
    } else if (wave >= 4 && wave < 4 + kPer) {
      const uint32_t row = min(t.q * N + 64 * (wave - 4) + lane, meta.n - 1);
      const uint32_t at = 256 * (wave - 4);
      four(g.row.target, row, offsetof(Params<N>, target) + at);
      if (KIND == kLogitGrad) {
        four(g.row.lse, row, offsetof(Params<N>, lse) + at);
        four(g.row.a, row, offsetof(Params<N>, a) + at);
        four(g.row.b, row, offsetof(Params<N>, b) + at);
        if (El::kScaled) four(g.row.m, row, offsetof(Params<N>, m) + at);
      }
      if (El::kScaled) four(g.row.r, row, offsetof(Params<N>, r) + at);
    }
  };
  auto issue = [&](int buf) {
    while (load_s == load_n) {  // (a part may have no steps)
      load_id += stride;
      if (load_id >= end) {
        load_n = load_s + 1;  // (and stays so)
        load_id = end;
        break;
      }
      load_tile = tile_of(load_id);
      load_s = 0;
      load_n = load_tile.steps;
      if (load_n > 0) {
        if (kLogits) load_params(load_tile, load_turn);
        load_turn = load_turn == kSets - 1 ? 0 : load_turn + 1;
        off_p = lane_of<N, TP, PL>(g.P, load_tile.p * N).at(0, (uint32_t)(g.P.ld * 2), N);
        off_q = lane_of<N, TQ, PL>(g.Q, load_tile.q * N).at(0, (uint32_t)(g.Q.ld * 2), N);
      }
    }
    if (load_id >= end) return;
    const int64_t p0 = load_tile.p * N, q0 = load_tile.q * N, k = load_tile.first + load_s;
    const uint16_t* bp = g.P.p + (TP ? k * kK * g.P.ld + p0 * PL : p0 * g.P.ld + k * kStep);
    const uint16_t* bq = g.Q.p + (TQ ? k * kK * g.Q.ld + q0 * PL : q0 * g.Q.ld + k * kStep);
    // (a transposed operand has all of a stage's rows, but for w behind the last token)
    const int rows_p = TP ? (KIND == kDx ? g.P.kn - (int)k * kK : kK) : g.P.n - (int)p0;
    const int rows_q = TQ ? kK : g.Q.n - (int)q0;
    const uint32_t to = lds_at + buf * Ti::kStageBytes;
    load_stage<N, TP, PL>(to, bp, off_p, g.P, (int)p0, rows_p);
    load_stage<N, TQ, PL>(to + Ti::kOperandBytes, bq, off_q, g.Q, (int)q0, rows_q);
    ++load_s;
  };

  // A stage's second half (its second plane) is in registers before the barrier in its
  // middle, so behind that its place takes another stage, whose loads then have all the
  // time that the stages before it take; and no wave waits for LDS right after a barrier.
  f32x4 acc[FP][FQ];
  s16x8 pa[2][FP], qb[2][FQ];
  constexpr int kReadP = (TP ? 2 : 1) * FP, kReadQ = (TQ ? 2 : 1) * FQ;  // LDS reads
  auto read_p = [&](int buf, int half) {
#pragma unroll
    for (int i = 0; i < FP; ++i)
      pa[half][i] = fragment<N, TP>(lds + buf * Ti::kStageBytes, wp + 16 * i, half, lane);
  };
  auto read_q = [&](int buf, int half) {
#pragma unroll
    for (int j = 0; j < FQ; ++j)
      qb[half][j] = fragment<N, TQ>(lds + buf * Ti::kStageBytes + Ti::kOperandBytes, wq + 16 * j,
                                    half, lane);
  };
  auto multiply = [&](int p, int q) {
#pragma unroll
    for (int i = 0; i < FP; ++i)
#pragma unroll
      for (int j = 0; j < FQ; ++j) acc[i][j] = El::mfma(pa[p][i], qb[q][j], acc[i][j]);
  };
  // (by columns, so that each of Q's fragments is free after its FP products)
  auto multiply_by_q = [&](int p, int q) {
#pragma unroll
    for (int j = 0; j < FQ; ++j)
#pragma unroll
      for (int i = 0; i < FP; ++i) acc[i][j] = El::mfma(pa[p][i], qb[q][j], acc[i][j]);
  };

  // Waits for the stage after the present one: those behind it may be in flight, as long
  // as there are any.
  auto land_next = [&]() {
    if (kStages > 2 && load_id < end) land<2 * (kStages - 2) * Ti::kLoads>();
    else land<0>();
  };
#pragma unroll
  for (int s = 0; s < kStages; ++s) issue(s);
  if (kStages > 2 && load_id < end) land<2 * (kStages - 1) * Ti::kLoads>();
  else land<0>();
  __syncthreads();
  int buf = 0, turn = 0;
  for (int id = begin; id < end; id += stride) {
    const Tile tile = tile_of(id);
    const int p0 = tile.p * N, q0 = tile.q * N, n_stage = tile.steps;
    const Params<N>& par = params[turn];
    turn = turn == kSets - 1 ? 0 : turn + 1;
    // (sums of bfloat16 operands begin at the bias)
    constexpr bool kFromBias = kLogits && !El::kScaled;
#pragma unroll
    for (int i = 0; i < FP; ++i) {
      f32x4 from = {0.f, 0.f, 0.f, 0.f};
      if (kFromBias && g.bias) {
        const uint4 b = *reinterpret_cast<const uint4*>(&par.bias[wp + 16 * i + 4 * (lane >> 4)]);
        from = f32x4{low16(b.x), low16(b.y), low16(b.z), low16(b.w)};
      }
#pragma unroll
      for (int j = 0; j < FQ; ++j) acc[i][j] = from;
    }
    read_q(buf, 0);
    read_p(buf, 0);
    for (int s = 0; s < n_stage; ++s) {
      // the first half's products while the second half is read ...
      read_q(buf, 1);
      read_p(buf, 1);
      PL == 1 ? multiply(0, 0) : multiply_by_q(0, 0);
      interleave<kReadP + kReadQ, FP * FQ>();
      land_next();
      __syncthreads();
      issue(buf);
      buf = buf == kStages - 1 ? 0 : buf + 1;
      // ... and the others while the next stage's is (behind the last nothing uses it)
      if constexpr (PL == 1) {
        read_q(buf, 0);
        read_p(buf, 0);
        multiply(1, 1);
        interleave<kReadP + kReadQ, FP * FQ>();
      } else {
        // (the next stage's first half takes the first one's registers, when its products
        // have begun)
        multiply(0, 1);
        __builtin_amdgcn_sched_group_barrier(0x008, FP * FQ, 0);
        read_p(buf, 0);
        multiply_by_q(1, 0);
        read_q(buf, 0);
        interleave_columns<FP, kReadP / FP, FQ, kReadQ / FQ>();
      }
    }

    // (the epilogue's addresses are made here: kept over the loop above they would not
    // leave enough registers for it)
    int of_lane = lane;
    asm volatile("" : "+v"(of_lane));
    // lane l holds q = l % 16 and p = 4 (l / 16) ... of each 16 x 16
    const int lq = of_lane & 15, lp = 4 * (of_lane >> 4);
    const int c_lane = wp + lp;  // first token of the lane in the tile, of 4 in every 16
    if (kLogits) {
      if (El::kScaled) {
        // in two steps, each with about half of S's exponent: with all of it one could
        // overflow on the way to a logit that does not
        const int e_s = exponent_of(meta.S), half = e_s / 2;
        const float first = power_of(half), second = power_of(e_s - half);
        float r[FQ];
#pragma unroll
        for (int j = 0; j < FQ; ++j)
          r[j] = fminf(par.r[wq + 16 * j + lq] * second, 0x1p127f);  // (times 0 it is 0)
#pragma unroll
        for (int i = 0; i < FP; ++i)
#pragma unroll
          for (int j = 0; j < FQ; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] = acc[i][j][e] * first * r[j];
      }
      if (El::kScaled && g.bias) {
#pragma unroll
        for (int i = 0; i < FP; ++i) {
          const f32x4 b = *reinterpret_cast<const f32x4*>(&par.bias[c_lane + 16 * i]);
#pragma unroll
          for (int j = 0; j < FQ; ++j) acc[i][j] += b;
        }
      }
      if (g.c0 + p0 + N > g.C) {
        // nothing behind the last token
#pragma unroll
        for (int i = 0; i < FP; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (g.c0 + p0 + c_lane + 16 * i + e >= g.C) {
#pragma unroll
              for (int j = 0; j < FQ; ++j) acc[i][j][e] = -__builtin_huge_valf();
            }
      }
    }
    if (KIND == kStats) {
      if (g.z) {
#pragma unroll
        for (int j = 0; j < FQ; ++j) {
          const int64_t row = q0 + wq + 16 * j + lq;
          if (row >= meta.n) continue;
#pragma unroll
          for (int i = 0; i < FP; ++i)
            *reinterpret_cast<f32x4*>(g.z + row * g.ldg + p0 + c_lane + 16 * i) = acc[i][j];
        }
      }
#pragma unroll
      for (int j = 0; j < FQ; ++j) {
        const int row = q0 + wq + 16 * j + lq;
        // the row's target among the lane's tokens
        const int t =
            row < meta.n ? par.target[wq + 16 * j + lq] - (g.c0 + p0 + c_lane) : -1;
        const bool here = t >= 0 && t < N / 2 && (t & 12) == 0;
        if (__ballot(here)) {
          float hit = 0.f;
#pragma unroll
          for (int i = 0; i < FP; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (t == 16 * i + e) hit = acc[i][j][e];
          if (here) g.hit[row] = hit;
        }
        float m = -__builtin_huge_valf();
#pragma unroll
        for (int i = 0; i < FP; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) m = fmaxf(m, acc[i][j][e]);
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        // (a NaN among the logits is no maximum, but it is in the sum)
        const float base = m == -__builtin_huge_valf() ? 0.f : m;
        const Shift shift = shift_of(base);
        if (__any(shift.far)) {
#pragma unroll
          for (int i = 0; i < FP; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] -= shift.far ? base : 0.f;
        }
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < FP; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            sum[e] += __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][j][e], kLog2e, shift.by));
        float all = (sum[0] + sum[1]) + (sum[2] + sum[3]);
        all = __builtin_fmaf(all, shift.off, all);
        all += __shfl_xor(all, 16);
        all += __shfl_xor(all, 32);
        if (row < meta.n && of_lane < 16)
          g.part[(int64_t)row * g.n_part + 2 * tile.p + (wave >> 2)] = make_float2(m, all);
      }
    }
    if (KIND == kLogitGrad) {
      const float norm = El::kScaled ? 1.f : meta.inverse;
#pragma unroll
      for (int j = 0; j < FQ; ++j) {
        const int at = wq + 16 * j + lq, row = q0 + at;
        const bool in = row < meta.n;
        const float lse = par.lse[at];
        float a = par.a[at] * norm;
        Shift shift = {};
        if constexpr (!El::kScaled) {  // (float32 has no registers left for it)
          shift = shift_of(lse);
          a = __builtin_fmaf(a, shift.off, a);
          if (__any(shift.far)) {
#pragma unroll
            for (int i = 0; i < FP; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[i][j][e] -= shift.far ? lse : 0.f;
          }
        }
        const int t = in ? par.target[at] - (g.c0 + p0 + c_lane) : -1;
        // G over the logits
#pragma unroll
        for (int i = 0; i < FP; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float z = acc[i][j][e];
            const float p = __builtin_amdgcn_exp2f(El::kScaled ? (z - lse) * kLog2e
                                                               : __builtin_fmaf(z, kLog2e, shift.by));
            acc[i][j][e] = in ? a * p : 0.f;
          }
        if (__ballot(t >= 0 && t < N / 2 && (t & 12) == 0)) {
          const float b = par.b[at] * norm;
#pragma unroll
          for (int i = 0; i < FP; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (t == 16 * i + e) acc[i][j][e] -= b;
        }
      }
      if (g.col) {
        // the tile's columns: over the lane's rows, 16 lanes, and the four waves through LDS
        float* sums = reinterpret_cast<float*>(smem + kStages * Ti::kStageBytes +
                                               kSets * sizeof(Params<N>));
        float m[FQ];
#pragma unroll
        for (int j = 0; j < FQ; ++j) m[j] = El::kScaled ? par.m[wq + 16 * j + lq] : 1.f;
#pragma unroll
        for (int i = 0; i < FP; ++i) {
          float cs[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float v = 0.f;
#pragma unroll
            for (int j = 0; j < FQ; ++j) v += El::kScaled ? acc[i][j][e] * m[j] : acc[i][j][e];
            v += __shfl_xor(v, 1);
            v += __shfl_xor(v, 2);
            v += __shfl_xor(v, 4);
            v += __shfl_xor(v, 8);
            cs[e] = v;
          }
          if (lq == 0)
            *reinterpret_cast<float4*>(sums + (wave & 3) * N + c_lane + 16 * i) =
                make_float4(cs[0], cs[1], cs[2], cs[3]);
        }
        __syncthreads();
        const int c = threadIdx.x;
        if (c < N)
          g.col[(int64_t)tile.q * g.ldg + p0 + c] =
              (sums[c] + sums[N + c]) + (sums[2 * N + c] + sums[3 * N + c]);
        // (the next tile's sums come behind its own barriers)
      }
      // four fragments of tokens at a time (two in tiles of 64, each lane its own four)
      constexpr int kF = FP < 4 ? FP : 4;
#pragma unroll
      for (int part = 0; part < FP / kF; ++part) {
#pragma unroll
        for (int j = 0; j < FQ; ++j) {
          uint2 out[kF][El::PLANES];
#pragma unroll
          for (int i = 0; i < kF; ++i) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float x = acc[kF * part + i][j][e];
              v[e] = El::kScaled ? x * 0x1p14f : x;
            }
            El::planes4(v, out[i]);
          }
          const int64_t row = q0 + wq + 16 * j + lq;
          uint16_t* to = g.G + row * PL * g.ldg + PL * (p0 + wp + 64 * part);
#pragma unroll
          for (int s = 0; s < El::PLANES; ++s) {
            if constexpr (kF == 4) {
              uint4 lo, hi;
              gather16(out[0][s], out[1][s], out[2][s], out[3][s], &lo, &hi);
              uint4* at = reinterpret_cast<uint4*>(to + place<PL>(4 * lp) + s * kTurn);
              at[0] = lo;
              at[1] = hi;
            } else {
#pragma unroll
              for (int i = 0; i < kF; ++i)
                *reinterpret_cast<uint2*>(to + place<PL>(16 * i + lp) + s * kTurn) = out[i][s];
            }
          }
        }
      }
    }
    if (KIND == kDx || KIND == kDw) {
      // rows that can be stored by 16 bytes (bfloat16: and end at one)
      const bool wide = g.ldo % 8 == 0 && (uintptr_t)g.out % 16 == 0 &&
                        (sizeof(T) == 4 || g.D % 8 == 0);
#pragma unroll
      for (int j = 0; j < FQ; ++j) {
        const int q = q0 + wq + 16 * j + lq;
        const bool in = q < (KIND != kDx ? g.n_q : g.paired ? 2 * kPair : meta.n);
        f32x4* sums = reinterpret_cast<f32x4*>(g.acc + tile.split * g.acc_split +
                                               (int64_t)q * g.lda + p0 + c_lane);
        if (g.add && in) {
#pragma unroll
          for (int i = 0; i < FP; ++i)
            if (p0 + c_lane + 16 * i < g.lda) acc[i][j] += sums[4 * i];
        }
        if (!g.out) {
#pragma unroll
          for (int i = 0; i < FP; ++i)
            if (in && p0 + c_lane + 16 * i < g.lda) sums[4 * i] = acc[i][j];
          continue;
        }
        Scale scale = {0.f, 0};
        if (in) scale = KIND == kDx ? dx_scale<T>(g, meta, q) : dw_scale<T>(meta);
        T* o = static_cast<T*>(g.out) + (KIND == kDx && in ? (int64_t)g.idx[q] : q) * g.ldo;
        if constexpr (sizeof(T) == 2 && FP >= 4) {
          if (wide) {
#pragma unroll
            for (int part = 0; part < FP / 4; ++part) {
              uint2 out[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const f32x4 v = acc[4 * part + i][j] * scale.by;
                out[i] = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
              }
              uint4 lo, hi;
              gather16(out[0], out[1], out[2], out[3], &lo, &hi);
              const int d = p0 + wp + 64 * part + 4 * lp;
              if (in && d < g.D) reinterpret_cast<uint4*>(o + d)[0] = lo;
              if (in && d + 8 < g.D) reinterpret_cast<uint4*>(o + d)[1] = hi;
            }
            continue;
          }
        }
        if (in) {
#pragma unroll
          for (int i = 0; i < FP; ++i) {
            const int d = p0 + c_lane + 16 * i;
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = scaled<T>(acc[i][j][e], scale);
            store4(o + d, v, wide, g.D - d);
          }
        }
      }
    }
  }
  land<0>();  // (nothing is left in flight into LDS that another workgroup may get)
}

template <int KIND, class T, int N>
hipError_t launch_n(const Gemm& g, hipStream_t st) {
  constexpr int kLds = Tiling<N>::kLdsBytes;
  const int64_t total = (int64_t)g.tp * g.tq * g.splits;
  if (total <= 0) return hipSuccess;
  if (total > INT32_MAX / 2) return hipErrorInvalidValue;
  const int64_t grid = total < 256 ? up(total, 8) : 256;
  (void)hipFuncSetAttribute(reinterpret_cast<const void*>(&gemm_kernel<KIND, T, N>),
                            hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
  gemm_kernel<KIND, T, N><<<dim3((unsigned)grid), dim3(kThreads), kLds, st>>>(g);
  return hipGetLastError();
}

template <int KIND, class T>
hipError_t launch(const Gemm& g, hipStream_t st) {
  return g.tile == 256   ? launch_n<KIND, T, 256>(g, st)
         : g.tile == 128 ? launch_n<KIND, T, 128>(g, st)
                         : launch_n<KIND, T, 64>(g, st);
}

}  // namespace linear
}  // namespace tbias
