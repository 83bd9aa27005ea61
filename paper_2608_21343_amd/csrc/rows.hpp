// Rows of logits kept in registers: loading, softmax statistics, and the sums
// over a row's segments. Shared by the row operators (log probabilities of
// given tokens, distillation from a teacher's top logits, their gradients).
//
// A row z[0..C) at temperature tau has u = z / tau, m = max z and, in units of
// log2, the exponents t_v = (z_v - m) log2(e) / tau <= 0. The operators need
//
//   S = sum 2^t,  D = sum 2^t t   (entropy = ln S - ln 2 D / S),
//   R = sum of 2^t over the tokens outside a list.
//
// One row takes one, two, four or sixteen waves (plan() below), each lane holding
// NP pieces of 16 bytes, so that every operator reads a row once, also one that
// writes its gradient: 16,384 rows of 8193 bfloat16 103 us (5.2 TB/s read and
// written, as a copy), 65,536 such rows read for log-sum-exp and entropy 172 us
// (6.2 TB/s). Rows longer than the registers of a workgroup are cut into
// segments: a first launch leaves every segment's (m, S, D, R) in the caller's
// workspace, a second one joins them.
#pragma once

#include <climits>

#include "device.hpp"
#include "launch.hpp"

namespace tbias {
namespace rows {

constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLn2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;
constexpr int kThreads = 256;  // of a workgroup whose rows take one wave each
constexpr int kMaxSeg = 64;    // segments of a row: one lane each when they are joined

// Sixteen bytes at the alignment of one element: rows start at any element.
template <class LT>
struct __attribute__((packed, aligned(sizeof(LT)))) Quad {
  uint32_t w[4];
};

template <class LT>
struct Elem;
template <>
struct Elem<float> {
  static constexpr int PV = 4;  // values in 16 bytes
  static constexpr uint32_t kFill = 0xff800000u;  // -inf
  __device__ static inline float get(const uint32_t* w, int e) { return __uint_as_float(w[e]); }
  // a value as it is loaded, and what it is worth
  typedef float Raw;
  static constexpr float kRawNegInf = -__builtin_huge_valf();
  __device__ static inline float widen(float x) { return x; }
  __device__ static inline float narrow(float x) { return x; }
  __device__ static inline void pack(const float* v, uint32_t* w) {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(v[e]);
  }
};
template <>
struct Elem<uint16_t> {
  static constexpr int PV = 8;
  static constexpr uint32_t kFill = 0xff80ff80u;
  // Volatile, so that every pass over a row takes the pairs apart again; held
  // widened from pass to pass they take twice the registers (scratch memory in
  // the longest rows).
  __device__ static inline float get(const uint32_t* w, int e) {
    float x;
    if (e & 1)
      asm volatile("v_and_b32 %0, %2, %1" : "=v"(x) : "v"(w[e / 2]), "s"(0xffff0000u));
    else
      asm volatile("v_lshlrev_b32 %0, 16, %1" : "=v"(x) : "v"(w[e / 2]));
    return x;
  }
  typedef uint32_t Raw;
  static constexpr uint32_t kRawNegInf = 0xff80u;
  // Volatile, too: moved to where the value is loaded, it waits for all loads.
  __device__ static inline float widen(uint32_t x) {
    float y;
    asm volatile("v_lshlrev_b32 %0, 16, %1" : "=v"(y) : "v"(x));
    return y;
  }
  // to the nearest, ties to even; the one rounding of a bfloat16 gradient
  __device__ static inline uint32_t pair(float a, float b) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef __bf16 h2 __attribute__((ext_vector_type(2)));
    const f2 v = {a, b};
    const h2 h = __builtin_convertvector(v, h2);
    return __builtin_bit_cast(uint32_t, h);
  }
  __device__ static inline uint16_t narrow(float x) { return (uint16_t)pair(x, x); }
  __device__ static inline void pack(const float* v, uint32_t* w) {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = pair(v[2 * e], v[2 * e + 1]);
  }
};

// The rows of a call and how they are cut.
struct Rows {
  const void* z;
  int64_t stride;   // elements from row to row
  int64_t row0;     // first row of this launch
  int64_t n_rows;   // rows of the call
  int32_t C;        // values of a row
  int32_t n_seg;    // segments of a row (1: the row is kept whole)
  int32_t seg;      // values of a segment (the last may be shorter)
  float c;          // log2(e) / tau
  float inv_tau;
  float4* part;     // [n_rows, n_seg] segments' (m, S, D, R)
};

struct Stats {
  float m, S, D, R;
};

// How t_v is computed: one fused multiply-add per value, z c - M, where M = m c
// rounded; the exponents are then delta = m c - M too small, all by the same,
// which the callers take out of what they report. Where |m c| is so large that
// delta is not small (masks of the type's lowest value) the maximum is
// subtracted first and delta is 0.
struct Basis {
  float c, m, M, delta;
  bool big;
  __device__ static inline Basis of(float m, float c) {
    Basis b;
    b.c = c;
    b.m = m == kNegInf ? 0.f : m;  // no value above -inf: every term is 0
    b.M = b.m * c;
    b.big = !(__builtin_fabsf(b.M) < 65536.f);
    b.delta = b.big ? 0.f : __builtin_fmaf(b.m, c, -b.M);
    return b;
  }
  template <bool BIG>
  __device__ inline float t(float z) const {
    return BIG ? (z - m) * c : __builtin_fmaf(z, c, -M);
  }
  __device__ inline float t(float z) const { return big ? t<true>(z) : t<false>(z); }
};

__device__ __forceinline__ float exp2_fast(float t) { return __builtin_amdgcn_exp2f(t); }
// Natural logarithm of 0 or a normal number, to 1.5 units of the last place.
__device__ __forceinline__ float ln(float x) { return __builtin_amdgcn_logf(x) * kLn2; }

// max of three in one instruction; a NaN stays (a maximum that passes it over
// costs another instruction for every value loaded)
__device__ __forceinline__ float max3(float a, float b, float c) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

// ---- sums and maxima of a wave, one instruction a step: a lane without a
// source keeps its value. (A read across lanes comes two instructions after the
// write; the compiler does not look into the block, so it keeps that itself.)
#define TB_STEPS(OP1, OP2, WAIT)                                                       \
  "s_nop 1\n\t" OP1 " row_shr:1 row_mask:0xf bank_mask:0xf\n\t" OP2                   \
  " row_shr:1 row_mask:0xf bank_mask:0xf\n\t" WAIT "\n\t" OP1                         \
  " row_shr:2 row_mask:0xf bank_mask:0xf\n\t" OP2                                      \
  " row_shr:2 row_mask:0xf bank_mask:0xf\n\t" WAIT "\n\t" OP1                         \
  " row_shr:4 row_mask:0xf bank_mask:0xf\n\t" OP2                                      \
  " row_shr:4 row_mask:0xf bank_mask:0xf\n\t" WAIT "\n\t" OP1                         \
  " row_shr:8 row_mask:0xf bank_mask:0xf\n\t" OP2                                      \
  " row_shr:8 row_mask:0xf bank_mask:0xf\n\t" WAIT "\n\t" OP1                         \
  " row_bcast:15 row_mask:0xa bank_mask:0xf\n\t" OP2                                   \
  " row_bcast:15 row_mask:0xa bank_mask:0xf\n\t" WAIT "\n\t" OP1                      \
  " row_bcast:31 row_mask:0xc bank_mask:0xf\n\t" OP2                                   \
  " row_bcast:31 row_mask:0xc bank_mask:0xf\n\ts_nop 1"
#define TB_STEP(OP)                                                                     \
  "s_nop 1\n\t" OP " row_shr:1 row_mask:0xf bank_mask:0xf\n\ts_nop 1\n\t" OP          \
  " row_shr:2 row_mask:0xf bank_mask:0xf\n\ts_nop 1\n\t" OP                            \
  " row_shr:4 row_mask:0xf bank_mask:0xf\n\ts_nop 1\n\t" OP                            \
  " row_shr:8 row_mask:0xf bank_mask:0xf\n\ts_nop 1\n\t" OP                            \
  " row_bcast:15 row_mask:0xa bank_mask:0xf\n\ts_nop 1\n\t" OP                         \
  " row_bcast:31 row_mask:0xc bank_mask:0xf\n\ts_nop 1"

__device__ __forceinline__ float wave_most(float v) {  // a NaN is passed over
  asm(TB_STEP("v_max_f32_dpp %0, %0, %0") : "+v"(v));
  return bcast63_f(v);
}
__device__ __forceinline__ float wave_least(float v) {
  asm(TB_STEP("v_min_f32_dpp %0, %0, %0") : "+v"(v));
  return bcast63_f(v);
}
__device__ __forceinline__ float wave_total(float v) {
  asm(TB_STEP("v_add_f32_dpp %0, %0, %0") : "+v"(v));
  return bcast63_f(v);
}
__device__ __forceinline__ int32_t wave_total_i32(int32_t v) {
  asm(TB_STEP("v_add_u32_dpp %0, %0, %0") : "+v"(v));
  return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ void wave_totals(float& v, float& w) {
  asm(TB_STEPS("v_add_f32_dpp %0, %0, %0", "v_add_f32_dpp %1, %1, %1", "s_nop 0")
      : "+v"(v), "+v"(w));
  v = bcast63_f(v);
  w = bcast63_f(w);
}
#undef TB_STEP
#undef TB_STEPS

// Reductions over the NWR waves of a row; `box` holds NWR words (a word for
// every wave and sum) that no other reduction of the kernel uses.
template <int NWR>
__device__ __forceinline__ float row_max(float v, float* box, int q) {
  v = wave_most(v);
  if (NWR == 1) return v;
  if (__lane_id() == 0) box[q] = v;
  __syncthreads();
  float r = box[0];
#pragma unroll
  for (int i = 1; i < NWR; ++i) r = __builtin_fmaxf(r, box[i]);
  return r;
}
// Sums of v[0] and, where they are used, of v[1] or v[2].
template <int NWR, bool SECOND, bool THIRD>
__device__ __forceinline__ void row_sum(float (&v)[3], float* box, int q) {
  static_assert(!(SECOND && THIRD), "two sums at most");
  constexpr int K = SECOND ? 1 : 2;
  if (SECOND || THIRD)
    wave_totals(v[0], v[K]);
  else
    v[0] = wave_total(v[0]);
  if (NWR == 1) return;
  if (__lane_id() == 0) {
    box[q] = v[0];
    if (SECOND || THIRD) box[NWR + q] = v[K];
  }
  __syncthreads();
  float r = 0.f, r2 = 0.f;
#pragma unroll
  for (int i = 0; i < NWR; ++i) {
    r += box[i];
    if (SECOND || THIRD) r2 += box[NWR + i];
  }
  v[0] = r;
  if (SECOND || THIRD) v[K] = r2;
}

// n values of a row from `row` on, in the registers of NWR waves: NP pieces of
// PV values a lane, and what fills no piece one value per lane of wave 0. Places
// past the end hold -inf.
//
// A row of one wave starts with its first piece wherever it lies in memory, so
// that its results depend on its values alone. In longer rows of bfloat16 the
// pieces lie on whole 16 bytes and up to PV - 1 values come before them: sums
// then differ in their last bits from place to place, but a distillation with its
// gradient of 2048 rows of 131,073 takes 243 us instead of 308. Float32 rows gain
// nothing (2048 of 65,537 values, 16 alternatives: 139 and 130).
template <class LT, int NWR, int NP>
struct Tile {
  static constexpr int PV = Elem<LT>::PV;
  static constexpr bool kWhole16 = PV == 8 && NWR > 1;
  Quad<LT> w[NP];
  typename Elem<LT>::Raw rim_raw;
  int32_t lane, q;
  int32_t n, pieces;  // values, whole pieces of the row
  int32_t head;       // values before the first piece

  __device__ inline int32_t piece(int p) const { return (p * NWR + q) * 64 + lane; }
  __device__ inline bool has(int p) const { return piece(p) < pieces; }
  // Passes over the pieces, f(p): of tiles of four and more a row may need little
  // more than half, so the second half is taken by groups that are skipped where the
  // row has ended (131,072 rows of 1082 bfloat16 78 us, 70 without the unused pieces;
  // 4096 of 33,000 in segments of (4, 16) 78 and 54). Tested piece by piece
  // throughout, full tiles lose: 65,536 rows of 8193 with 32 alternatives 226 us
  // instead of 211.
  template <class F>
  __device__ inline void each(F f) const {
    constexpr int H = NP >= 4 ? NP / 2 : NP, G = NP >= 4 ? NP / 4 : 1;
#pragma unroll
    for (int p = 0; p < H; ++p) f(p);
#pragma unroll
    for (int g = H; g < NP; g += G) {
      if ((g * NWR + q) * 64 >= pieces) continue;  // uniform
#pragma unroll
      for (int p = g; p < g + G; ++p) f(p);
    }
  }
  __device__ inline int32_t first(int p) const { return head + piece(p) * PV; }
  __device__ inline int32_t rim_at() const { return lane < head ? lane : pieces * PV + lane; }
  __device__ inline bool has_rim() const { return q == 0 && lane < n - pieces * PV; }

  __device__ inline void load(const LT* row, int32_t n_, int lane_, int q_) {
    n = n_;
    lane = lane_;
    q = q_;
    head = kWhole16 ? (int32_t)((16 - ((uintptr_t)row & 15)) & 15) / (int32_t)sizeof(LT) : 0;
    if (head > n) head = n;
    pieces = (n - head) / PV;
    const LT* aligned = row + head;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      if (has(p)) {
        w[p] = *reinterpret_cast<const Quad<LT>*>(aligned + piece(p) * PV);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) w[p].w[k] = Elem<LT>::kFill;
      }
    }
    rim_raw = Elem<LT>::kRawNegInf;
    if (has_rim()) rim_raw = row[rim_at()];
  }
  __device__ inline float rim() const { return Elem<LT>::widen(rim_raw); }
  // Places of a value in membership bits: a piece's lie within one word.
  __device__ inline int32_t bit(int32_t i) const { return i + PV - head; }
  __device__ inline float at(int p, int e) const { return Elem<LT>::get(w[p].w, e); }

  // largest value of this lane's (or NaN), also of two halves of them
  __device__ inline void lane_max2(float& a, float& b) {
    a = rim();
    b = kNegInf;
    each([&](int p) {
#pragma unroll
      for (int e = 0; e < PV; e += 4) {
        a = max3(a, at(p, e), at(p, e + 1));
        b = max3(b, at(p, e + 2), at(p, e + 3));
      }
    });
  }
  __device__ inline float lane_max() {
    float a, b;
    lane_max2(a, b);
    return __builtin_elementwise_maximum(a, b);
  }

  // This lane's sums of 2^t, of 2^t t (ENT) and of 2^t outside the list whose
  // members are set in `bits` (LIST), in four chains: less rounding than in one.
  // t is held at -200, where 2^t is 0, so that -inf adds 0 to D. look(value,
  // place) sees every value, too.
  template <bool BIG, bool ENT, bool LIST, class F>
  __device__ inline void sums(const Basis& b, const uint32_t* bits, float (&s)[3], F look) {
    float a[4], d[4];
    {
      const float t = b.t<BIG>(rim()), x = exp2_fast(t);
      a[0] = x;
      a[1] = a[2] = a[3] = d[1] = d[2] = d[3] = 0.f;
      d[0] = ENT ? x * __builtin_fmaxf(t, -200.f) : 0.f;
      if (LIST) {
        const int32_t i = bit(rim_at());
        s[2] = has_rim() && ((bits[i >> 5] >> (i & 31)) & 1) ? 0.f : x;
      }
    }
    each([&](int p) {
      float v[PV], x[PV];
#pragma unroll
      for (int e = 0; e < PV; ++e) {
        v[e] = at(p, e);
        const float t = b.t<BIG>(v[e]);
        x[e] = exp2_fast(t);
        if (!LIST) a[e & 3] += x[e];
        if (ENT) d[e & 3] = __builtin_fmaf(x[e], __builtin_fmaxf(t, -200.f), d[e & 3]);
      }
      // the sums of a piece before its values are looked at and before the next
      // one's: put off, they hold registers
      if (!LIST) asm volatile("" : "+v"(a[0]), "+v"(a[1]), "+v"(a[2]), "+v"(a[3]));
      if (ENT) asm volatile("" : "+v"(d[0]), "+v"(d[1]), "+v"(d[2]), "+v"(d[3]));
#pragma unroll
      for (int e = 0; e < PV; ++e) look(v[e], first(p) + e);
      if (LIST) {
        // (also past the row's end, where 2^t is 0: no test of it)
        const int32_t f = bit(first(p));
        const uint32_t mask = bits[f >> 5] >> (f & 31) & ((1u << PV) - 1);
        float all = x[0];
#pragma unroll
        for (int e = 1; e < PV; ++e) all += x[e];
        asm volatile("" : "+v"(all));  // (as above)
        float r = all;
        if (__ballot(mask != 0) != 0) {  // few pieces hold a listed token
          r = 0.f;
#pragma unroll
          for (int e = 0; e < PV; ++e) r += (mask >> e) & 1 ? 0.f : x[e];
        }
        s[2] += r;
        a[p & 3] += all;
        asm volatile("" : "+v"(s[2]), "+v"(a[p & 3]));
      }
    });
    look(rim(), rim_at());
    s[0] = (a[0] + a[1]) + (a[2] + a[3]);
    if (ENT) s[1] = (d[0] + d[1]) + (d[2] + d[3]);
  }

  // Writes f(t, 2^t) in place of every value.
  template <bool BIG, class F>
  __device__ inline void store(LT* out, const Basis& b, F f) {
    each([&](int p) {
      float v[PV];
#pragma unroll
      for (int e = 0; e < PV; ++e) {
        const float t = b.t<BIG>(at(p, e));
        v[e] = f(t, exp2_fast(t));
      }
      Quad<LT> o;
      Elem<LT>::pack(v, o.w);
      if (PV == 8) asm volatile("" : "+v"(o.w[0]), "+v"(o.w[1]), "+v"(o.w[2]), "+v"(o.w[3]));
      if (has(p)) {
        *reinterpret_cast<Quad<LT>*>(out + first(p)) = o;
      }
    });
    if (has_rim()) {
      const float t = b.t<BIG>(rim());
      out[rim_at()] = Elem<LT>::narrow(f(t, exp2_fast(t)));
    }
  }

  __device__ inline void store_zeros(LT* out) const {
    Quad<LT> o = {{0u, 0u, 0u, 0u}};
#pragma unroll
    for (int p = 0; p < NP; ++p)
      if (has(p)) *reinterpret_cast<Quad<LT>*>(out + first(p)) = o;
    if (has_rim()) out[rim_at()] = Elem<LT>::narrow(0.f);
  }
};

// The row's statistics in the waves that hold it: relative to b's exponents (S,
// D and R are 2^-delta times too large, D also off by delta S).
// `box` holds 3 NWR words.
template <bool ENT, bool LIST, class LT, int NWR, int NP>
__device__ __forceinline__ Stats statistics(Tile<LT, NWR, NP>& x, float c, const uint32_t* bits,
                                            float* box, Basis& b) {
  const float m = row_max<NWR>(x.lane_max(), box, x.q);
  b = Basis::of(m, c);
  float s[3] = {0.f, 0.f, 0.f};
  auto look = [](float, int32_t) {};
  if (b.big)
    x.template sums<true, ENT, LIST>(b, bits, s, look);
  else
    x.template sums<false, ENT, LIST>(b, bits, s, look);
  row_sum<NWR, ENT, LIST>(s, box + NWR, x.q);
  return {m, s[0], s[1], s[2]};
}

// Statistics relative to the maximum itself, as segments are kept.
__device__ __forceinline__ float4 to_part(const Stats& s, const Basis& b) {
  const float f = exp2_fast(-b.delta);
  return make_float4(s.m, f * s.S, f * (s.D - b.delta * s.S), f * s.R);
}

// All segments' statistics of a row, joined; every lane of the wave returns
// them, relative to Basis::of(m, c).
__device__ __forceinline__ Stats join(const float4* part, int32_t n_seg, float c, int lane,
                                      Basis& b) {
  float4 v = make_float4(kNegInf, 0.f, 0.f, 0.f);
  if (lane < n_seg) v = part[lane];
  const float m = wave_most(v.x);
  b = Basis::of(m, c);
  // a segment without a value above -inf adds nothing, but its NaN
  const float a = v.x == kNegInf ? 0.f : (v.x - b.m) * c + b.delta;
  const float f = exp2_fast(a);
  const float t = __builtin_fmaxf(a, -200.f);
  Stats s;
  s.m = m;
  s.S = wave_total(f * v.y);
  s.D = f * __builtin_fmaf(t, v.y, v.z);
  s.R = f * v.w;
  wave_totals(s.D, s.R);
  return s;
}

// ln of the sum of exp(u - u_max)
__device__ __forceinline__ float log_sum(const Stats& s, const Basis& b) {
  return ln(s.S) - kLn2 * b.delta;
}
// entropy in nats; a row without a value above -inf has none
__device__ __forceinline__ float entropy(const Stats& s) {
  if (s.m == kNegInf && s.S == 0.f) return 0.f;
  const float h = ln(s.S) - kLn2 * (s.D * __builtin_amdgcn_rcpf(s.S));
  return h < 0.f ? 0.f : h;
}
__device__ __forceinline__ bool empty(const Stats& s) { return s.m == kNegInf && s.S == 0.f; }

// log probability of a value of the row
__device__ __forceinline__ float log_prob(float z, const Basis& b, float log_s, float inv_tau) {
  return z == kNegInf ? (log_s != log_s ? log_s : kNegInf) : (z - b.m) * inv_tau - log_s;
}

// ---- instances: waves per row and pieces per lane, by the values they hold

struct Shape {
  int nwr, np;
};
constexpr int capacity(Shape s, int pv) { return s.nwr * s.np * 64 * pv + pv - 1; }

constexpr int kShapes = 11;
constexpr Shape kShape[kShapes] = {{1, 1}, {1, 2},  {1, 4},  {1, 8},  {1, 16}, {2, 16},
                                   {4, 8}, {4, 16}, {16, 4}, {16, 8}, {16, 16}};
// Shapes that the segments of cut rows take.
constexpr bool cuts(Shape s) { return s.nwr == 4 && s.np >= 8; }
// bfloat16's largest shape, which plan() takes only where a gradient is written.
constexpr bool fills(Shape s, int pv) { return s.nwr == 16 && s.np == 16 && pv == 8; }

struct Plan {
  int shape;       // instance of the (whole or cut) rows
  int32_t n_seg;   // segments of a row
  int32_t seg;     // values of a segment
};
Plan plan(int32_t dtype, int64_t n_rows, int32_t C, bool grad);

// The segments' statistics, then their alternatives.
inline int64_t workspace_bytes(const Plan& p, int64_t n_rows, int32_t n_alt) {
  return p.n_seg > 1 ? n_rows * p.n_seg * (16 + 8 * (int64_t)n_alt) : 0;
}
// What suffices for any operator on up to n_rows rows.
int64_t most_workspace(int32_t dtype, int64_t n_rows, int32_t C, int32_t n_alt);

// Calls f(Int<NWR>, Int<NP>) for an instance.
template <int N>
struct Int {
  static constexpr int value = N;
};
template <class LT, int I = 0, class F>
inline void with_shape(int i, F f) {
  constexpr Shape s = kShape[I];
  if (i == I) {
    f(Int<s.nwr>(), Int<s.np>());
  } else if constexpr (I + 1 < kShapes) {
    with_shape<LT, I + 1>(i, f);
  }
}

// Launches over all rows, in ranges that one launch may hold; f(first row, grid).
template <class F>
inline void in_launches(int64_t n_rows, int rows_per_group, int threads, int32_t n_seg, F f) {
  const int64_t most = most_groups(threads) / n_seg * rows_per_group;
  for (int64_t r = 0; r < n_rows; r += most) {
    const int64_t n = n_rows - r < most ? n_rows - r : most;
    f(r, dim3((unsigned)((n + rows_per_group - 1) / rows_per_group), (unsigned)n_seg));
  }
}

// Where a wave stands: its row, its part of it.
template <int NWR>
struct Place {
  static constexpr int kWg = NWR > 1 ? NWR * 64 : kThreads;
  static constexpr int kRows = kWg / 64 / NWR;  // rows of a workgroup
  int lane, q, slot;  // slot: row of the workgroup
  int64_t row;
  int32_t c0, n;      // first value and number of values of the segment
  __device__ inline explicit Place(const Rows& a) {
    lane = __lane_id();
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    q = wv % NWR;
    slot = wv / NWR;
    row = a.row0 + (int64_t)blockIdx.x * kRows + slot;
    c0 = (int32_t)blockIdx.y * a.seg;
    n = a.C - c0 < a.seg ? a.C - c0 : a.seg;
  }
};

// Waves that a SIMD should hold at least: the largest tiles come out a few
// registers above the 96 that five waves may have (97: four, 65,536 rows of 8193
// bfloat16 with 32 alternatives 235 us instead of 217), tiles of eight pieces
// above the 64 with which two workgroups of sixteen waves fit a CU (4096 rows of
// 65,537 bfloat16, distillation with the tail and its gradient, 219 us instead of
// 240).
constexpr int least_waves(Shape s) {
  return s.nwr == 16 ? (s.np == 8 ? 8 : 4) : s.np == 16 ? 5 : 1;
}

// Orders a wave's LDS writes before its later reads (one wave's LDS operations
// are in order; this holds the compiler to it).
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ---- launchers (argument checks happen in the C ABI)

struct ScoreIO {
  const int32_t* tokens;
  int32_t J;
  float* logprob;
  float* lse;
  float* entropy;
  int32_t M;
  int32_t* alt;
  float* alt_logprob;
  int2* lists;  // [n_rows, n_seg, M] segments' alternatives: value bits, token
};
struct GradIO {
  const int32_t* tokens;
  int32_t J;
  const float* d_logprob;
  const float* d_lse;
  const float* d_entropy;
  void* grad;
  int64_t grad_stride;
};
struct DistillIO {
  const int32_t* tokens;
  const float* score;
  int32_t K;
  int32_t tail;
  const float* weight;
  float* loss;
  void* grad;
  int64_t grad_stride;
};
hipError_t score_f32(const Rows& a, const ScoreIO& io, const Plan& p, hipStream_t st);
hipError_t score_bf16(const Rows& a, const ScoreIO& io, const Plan& p, hipStream_t st);
hipError_t grad_f32(const Rows& a, const GradIO& io, const Plan& p, hipStream_t st);
hipError_t grad_bf16(const Rows& a, const GradIO& io, const Plan& p, hipStream_t st);
hipError_t distill_f32(const Rows& a, const DistillIO& io, const Plan& p, hipStream_t st);
hipError_t distill_bf16(const Rows& a, const DistillIO& io, const Plan& p, hipStream_t st);

}  // namespace rows
}  // namespace tbias
