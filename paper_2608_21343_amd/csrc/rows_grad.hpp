// Gradients of the row operators with respect to the logits: of the log
// probabilities of given tokens, the log-sum-exp and the entropy, and of the
// distillation loss from a teacher's top logits, whose value is computed here
// too (templates; instantiated in rows_grad_*.hip and rows_distill_*.hip).
//
// Every gradient is a multiple of the row's probabilities, with other values at
// the few listed tokens:
//
//   log probabilities g_j of tokens t_j, log-sum-exp g_L, entropy g_H:
//     dz_v = p_v (g_L - sum_j g_j - g_H (ln p_v + H)) / tau + sum_{t_j = v} g_j / tau
//   distillation, weight w, teacher probabilities q_k of tokens t_k:
//     dz_v = w p_v (Q - T) / tau  off the list,  w (Q p_v - sum_{t_k = v} q_k) / tau  on it,
//     Q: the teacher's mass; T = q_rest / p_rest with the tail, 0 without.
//
// So a lane writes its values from registers, then the lanes of one wave write
// the listed tokens over them (a token listed twice once, by its first place,
// with the places summed in order). A row is read once and written once, and
// the gradient may take the logits' own place.
#pragma once

#include "rows.hpp"

namespace tbias {
namespace rows {

// Words of a row's (or segment's) membership bits, one per value (Tile::bit).
template <class LT, int NWR, int NP>
constexpr int list_words() {
  return NWR * NP * 64 * Elem<LT>::PV / 32 + 1;
}

// A row's list: which lanes' tokens are the first of their kind, and the sum
// of g over the places of each. Lists of up to four places are compared place
// by place; for longer ones the lanes mark their tokens in bits, and only if one
// is found marked the places are compared.
__device__ __forceinline__ float sum_same(int32_t id, float g, int n, int lane, bool& first) {
  float sum = 0.f;
  first = true;
  for (int i = 0; i < n; ++i) {
    const int32_t other = __builtin_amdgcn_readlane(id, i);
    const float add = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(g), i));
    if (other == id) {
      sum += add;
      if (i < lane) first = false;
    }
  }
  return sum;
}
constexpr int kFewPlaces = 4;
// Marks a lane's token, at place i of the part's bits; whether two lanes have the
// same (every lane returns it).
__device__ __forceinline__ bool mark(uint32_t* bits, bool mine, int32_t i) {
  bool twice = false;
  if (mine) {
    const uint32_t one = 1u << (i & 31);
    twice = (atomicOr(&bits[i >> 5], one) & one) != 0;
  }
  return __ballot(twice) != 0;
}
__device__ __forceinline__ bool mark_fresh(uint32_t* bits, bool mine, int32_t i) {
  if (mine) bits[i >> 5] = 0u;
  wave_fence();
  return mark(bits, mine, i);
}

// The wave of a row that writes listed tokens has to come after all that the
// row's waves wrote.
template <int NWR>
__device__ __forceinline__ void row_sync() {
  if (NWR > 1)
    __syncthreads();
  else
    wave_fence();
}

enum Pass { kWhole, kStats, kApply };

// ---- gradient of log probabilities, log-sum-exp and entropy

template <class LT, int NWR, int NP, bool ENT, Pass PASS>
__global__ __launch_bounds__(Place<NWR>::kWg, least_waves(Shape{NWR, NP})) void grad_kernel(
    Rows a, GradIO io) {
  __shared__ float box[3 * NWR];
  __shared__ uint32_t bits_all[Place<NWR>::kRows][list_words<LT, NWR, NP>()];
  lds_poison(box, sizeof(box));
  lds_poison(bits_all, sizeof(bits_all));
  const Place<NWR> at(a);
  if (at.row >= a.n_rows) return;  // uniform over the row's waves
  const LT* z = static_cast<const LT*>(a.z) + at.row * a.stride;
  LT* out = static_cast<LT*>(io.grad) + at.row * io.grad_stride + at.c0;
  Tile<LT, NWR, NP> x;
  int32_t id = -1;
  typename Elem<LT>::Raw zj = Elem<LT>::kRawNegInf;
  float g = 0.f, gl = 0.f, gh = 0.f;
  if (at.lane < io.J) {
    id = io.tokens[at.row * io.J + at.lane];
    g = io.d_logprob[at.row * io.J + at.lane];
  }
  if (io.d_lse) gl = io.d_lse[at.row];
  if (ENT) gh = io.d_entropy[at.row];
  x.load(z + at.c0, at.n, at.lane, at.q);
  const bool ok = (uint32_t)id < (uint32_t)a.C;
  const bool mine = ok && id >= at.c0 && id < at.c0 + at.n;
  if (mine) zj = z[id];
  const bool bad = __ballot(!ok && id != -1) != 0;
  if (!ok) g = 0.f;
  // no gradient comes in: none goes out, whatever the row holds
  if (!bad && __ballot(g != 0.f) == 0 && gl == 0.f && gh == 0.f) {
    if (PASS != kStats) x.store_zeros(out);
    return;
  }
  Basis b;
  Stats s;
  if (PASS == kApply) {
    s = join(a.part + at.row * a.n_seg, a.n_seg, a.c, at.lane, b);
    row_sync<NWR>();  // zj is read before another wave may write there
  } else {
    s = statistics<ENT, false>(x, a.c, nullptr, box, b);
  }
  if (PASS == kStats) {
    if (at.q == 0 && at.lane == 0) a.part[at.row * a.n_seg + blockIdx.y] = to_part(s, b);
    return;
  }
  if (empty(s) && !bad) {
    x.store_zeros(out);
    return;
  }
  const float total = wave_total(g);
  const float f = a.inv_tau / s.S;
  float k0 = (gl - total) * f, k1 = 0.f;
  if (ENT) {
    k0 -= gh * (entropy(s) - ln(s.S)) * f;
    k1 = -gh * kLn2 * f;
  }
  if (bad) k0 = __builtin_nanf("");
  auto slope = [&](float t, float e) {
    return ENT ? e * __builtin_fmaf(k1, __builtin_fmaxf(t, -200.f), k0) : e * k0;
  };
  if (b.big)
    x.template store<true>(out, b, slope);
  else
    x.template store<false>(out, b, slope);
  row_sync<NWR>();
  if (at.q != 0) return;
  bool first = true;
  float sum = g;
  if (io.J <= kFewPlaces || mark_fresh(bits_all[at.slot], mine, x.bit(id - at.c0)))
    sum = sum_same(id, g, io.J, at.lane, first);
  if (mine && first) {
    const float t = b.t(Elem<LT>::widen(zj));
    out[id - at.c0] = Elem<LT>::narrow(__builtin_fmaf(sum, a.inv_tau, slope(t, exp2_fast(t))));
  }
}

// ---- distillation

// A rest of less mass than this is the rounding of the scores and of their sum:
// 64 half steps of float32, where a whole vocabulary's scores, H = -sum q s <=
// ln 64, are off by 4 H + 15 half steps of their sum and the sum of their
// exponentials by another 1.5 H + 8. (Taken as mass, it makes the loss infinite
// where the student has none outside the list.)
constexpr float kLeastRest = 0x1p-18f;

// A teacher's list, a token per lane.
struct Teacher {
  int32_t id;
  bool ok, bad;      // bad: the row has a token out of range
  bool none;         // no place is used
  float q, logq;
  float mass, rest;  // of the list and (with the tail) of all else
};
struct Places {  // as they lie in memory
  int32_t id;
  float score;
  __device__ inline Places(const DistillIO& io, int64_t row, int lane) {
    id = -1;
    score = kNegInf;
    if (lane < io.K) {
      id = io.tokens[row * io.K + lane];
      score = io.score[row * io.K + lane];
    }
  }
};
__device__ __forceinline__ Teacher teacher(const DistillIO& io, const Places& p, int32_t C,
                                           float c) {
  Teacher t;
  t.id = p.id;
  t.ok = (uint32_t)t.id < (uint32_t)C;
  t.bad = __ballot(!t.ok && t.id != -1) != 0;
  t.none = __ballot(t.ok) == 0;
  const float sc = t.ok ? p.score : kNegInf;
  t.rest = 0.f;
  if (io.tail) {
    t.q = exp2_fast(sc * kLog2e);
    t.logq = sc;
    const float sum = wave_total(t.q);
    const float rest = 1.f - sum;
    t.rest = rest < kLeastRest ? 0.f : rest;  // (a NaN stays)
    t.mass = sum + t.rest;
  } else {
    const float m = wave_most(sc);
    const float x = sc - (m == kNegInf ? 0.f : m);
    const float e = exp2_fast(x * c);
    const float sum = wave_total(e);
    t.mass = sum == 0.f ? 0.f : 1.f;
    t.q = sum == 0.f ? 0.f : e * __builtin_amdgcn_rcpf(sum);
    t.logq = x * (c * kLn2) - ln(sum);
    if (sum != sum) t.mass = sum;
  }
  return t;
}

// The sum outside the list, 0 where it is no normal number. Without a listed token
// it is that of the row, which was added up in another order: loss and gradient are
// then 0, not their difference.
__device__ __forceinline__ float sum_outside(const Teacher& t, const Stats& s) {
  return t.none ? s.S : s.R < 0x1p-126f ? 0.f : s.R;
}

__device__ __forceinline__ float distill_loss(const Teacher& t, float zk, const Stats& s,
                                              const Basis& b, float inv_tau) {
  const float log_s = log_sum(s, b);
  const float lp = log_prob(zk, b, log_s, inv_tau);
  // NaN scores give NaN terms
  float loss = wave_total(t.ok && t.q != 0.f ? t.q * (t.logq - lp) : 0.f);
  if (t.rest != 0.f) {  // nothing outside the list (or an empty row): no mass for the rest
    const float lr = s.R == 0.f ? kNegInf : ln(s.R) - ln(s.S);
    loss += t.rest * (ln(t.rest) - lr);
  }
  return t.bad ? __builtin_nanf("") : loss;
}

template <class LT, int NWR, int NP, bool TAIL, Pass PASS>
__global__ __launch_bounds__(Place<NWR>::kWg, least_waves(Shape{NWR, NP})) void distill_kernel(
    Rows a, DistillIO io) {
  constexpr int kWords = list_words<LT, NWR, NP>();
  __shared__ float box[3 * NWR];
  __shared__ uint32_t bits_all[Place<NWR>::kRows][kWords];
  lds_poison(box, sizeof(box));
  lds_poison(bits_all, sizeof(bits_all));
  const Place<NWR> at(a);
  if (at.row >= a.n_rows) return;  // uniform over the row's waves
  const LT* z = static_cast<const LT*>(a.z) + at.row * a.stride;
  LT* out = static_cast<LT*>(io.grad) + at.row * io.grad_stride + at.c0;
  // loads in the order in which they are waited for: the list, the row, and the
  // listed values, whose places the list gives while the row is on its way
  const Places places(io, at.row, at.lane);
  Tile<LT, NWR, NP> x;
  x.load(z + at.c0, at.n, at.lane, at.q);
  const bool mine = places.id >= at.c0 && places.id < at.c0 + at.n;
  typename Elem<LT>::Raw zk = Elem<LT>::kRawNegInf;
  if (mine) zk = z[places.id];
  const float w = io.weight ? io.weight[at.row] : 1.f;
  const Teacher t = teacher(io, places, a.C, a.c);
  if (w == 0.f || (t.mass == 0.f && !t.bad)) {
    if (PASS != kStats && io.grad) x.store_zeros(out);
    if (PASS == kWhole && io.loss && at.q == 0 && at.lane == 0) io.loss[at.row] = 0.f;
    return;
  }
  Basis b;
  Stats s;
  uint32_t* bits = bits_all[at.slot];
  bool twice = false;  // a token is listed twice (in the wave that writes the list)
  if (PASS == kApply) {
    s = join(a.part + at.row * a.n_seg, a.n_seg, a.c, at.lane, b);
    row_sync<NWR>();  // zk is read before another wave may write there
  } else {
    if (TAIL) {
      for (int i = at.q * 64 + at.lane; i < kWords; i += NWR * 64) bits[i] = 0u;
      row_sync<NWR>();
      if (at.q == 0) twice = mark(bits, mine, x.bit(t.id - at.c0));
      row_sync<NWR>();
    }
    s = statistics<false, TAIL>(x, a.c, bits, box, b);
  }
  if (PASS == kStats) {
    if (at.q == 0 && at.lane == 0) a.part[at.row * a.n_seg + blockIdx.y] = to_part(s, b);
    return;
  }
  if (TAIL) s.R = sum_outside(t, s);
  if (PASS == kWhole && io.loss && at.q == 0) {
    const float loss = distill_loss(t, Elem<LT>::widen(zk), s, b, a.inv_tau);
    if (at.lane == 0) io.loss[at.row] = w * loss;
  }
  if (!io.grad) return;
  if (empty(s) && !t.bad) {
    x.store_zeros(out);
    return;
  }
  const float wt = w * a.inv_tau;
  const float mass = t.bad ? __builtin_nanf("") : t.mass;
  const float k_on = mass * wt / s.S;
  float k_off = k_on, share = mass / s.S;
  if (TAIL && t.rest != 0.f && s.R != 0.f) {
    // (not by way of R / S, which may be too small a number for its inverse)
    share -= t.rest / s.R;
    k_off = share * wt;
  }
  // The quotient by R is up to 2^126 and wt 1e4 by the temperature alone: where their
  // product overflows, the exponential comes between them (a multiplication more a
  // value, so not in all rows: 7511 of 612 bfloat16 9.59 us, so 9.53).
  const bool fits = !TAIL || !__builtin_isinf(k_off);
  auto slope = [&](float, float e) { return e * k_off; };
  auto steep = [&](float, float e) { return e * share * wt; };
  if (!fits && b.big)
    x.template store<true>(out, b, steep);
  else if (!fits)
    x.template store<false>(out, b, steep);
  else if (b.big)
    x.template store<true>(out, b, slope);
  else
    x.template store<false>(out, b, slope);
  row_sync<NWR>();
  if (at.q != 0) return;
  if (!TAIL || PASS == kApply)
    twice = io.K <= kFewPlaces || mark_fresh(bits, mine, x.bit(t.id - at.c0));
  bool first = true;
  float sum = t.q;
  if (twice) sum = sum_same(t.id, t.q, io.K, at.lane, first);
  if (mine && first) {
    const float e = exp2_fast(b.t(Elem<LT>::widen(zk)));
    out[t.id - at.c0] = Elem<LT>::narrow(__builtin_fmaf(-sum, wt, e * k_on));
  }
}

// The loss of rows in segments: one wave per row, before the gradient may take
// the logits' place.
template <class LT>
__global__ __launch_bounds__(kThreads) void distill_loss_kernel(Rows a, DistillIO io) {
  const int lane = __lane_id();
  const int64_t row = a.row0 + (int64_t)blockIdx.x * (kThreads / 64) +
                      __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= a.n_rows) return;
  const LT* z = static_cast<const LT*>(a.z) + row * a.stride;
  const float w = io.weight ? io.weight[row] : 1.f;
  const Teacher t = teacher(io, Places(io, row, lane), a.C, a.c);
  float loss = 0.f;
  if (w != 0.f && (t.mass != 0.f || t.bad)) {
    Basis b;
    Stats s = join(a.part + row * a.n_seg, a.n_seg, a.c, lane, b);
    s.R = sum_outside(t, s);
    loss = w * distill_loss(t, t.ok ? Elem<LT>::widen(z[t.id]) : kNegInf, s, b, a.inv_tau);
  }
  if (lane == 0) io.loss[row] = loss;
}

// ---- launches

template <class LT, class F>
hipError_t in_shape(Rows a, const Plan& p, F launch) {
  with_shape<LT>(p.shape, [&](auto nwr, auto np) {
    constexpr int NWR = decltype(nwr)::value;
    typedef Place<NWR> Pl;
    in_launches(a.n_rows, Pl::kRows, Pl::kWg, p.n_seg, [&](int64_t r, dim3 grid) {
      a.row0 = r;
      launch(a, grid, dim3(Pl::kWg), nwr, np);
    });
  });
  return hipGetLastError();
}

template <class LT>
hipError_t grad_t(const Rows& all, const GradIO& io, const Plan& p, hipStream_t st) {
  auto pass = [&](const Rows& rows, auto pass_) {
    constexpr Pass PASS = (Pass) decltype(pass_)::value;
    return in_shape<LT>(rows, p, [&](const Rows& a, dim3 grid, dim3 wg, auto nwr, auto np) {
      constexpr int NWR = decltype(nwr)::value, NP = decltype(np)::value;
      if constexpr (PASS == kWhole || cuts(Shape{NWR, NP})) {
        if (io.d_entropy)
          grad_kernel<LT, NWR, NP, true, PASS><<<grid, wg, 0, st>>>(a, io);
        else
          grad_kernel<LT, NWR, NP, false, PASS><<<grid, wg, 0, st>>>(a, io);
      }
    });
  };
  if (p.n_seg == 1) return pass(all, Int<kWhole>());
  const hipError_t e = pass(all, Int<kStats>());
  return e == hipSuccess ? pass(all, Int<kApply>()) : e;
}

template <class LT>
hipError_t distill_t(const Rows& all, const DistillIO& io, const Plan& p, hipStream_t st) {
  auto pass = [&](const Rows& rows, auto pass_) {
    constexpr Pass PASS = (Pass) decltype(pass_)::value;
    return in_shape<LT>(rows, p, [&](const Rows& a, dim3 grid, dim3 wg, auto nwr, auto np) {
      constexpr int NWR = decltype(nwr)::value, NP = decltype(np)::value;
      if constexpr (PASS == kWhole || cuts(Shape{NWR, NP})) {
        if (io.tail)
          distill_kernel<LT, NWR, NP, true, PASS><<<grid, wg, 0, st>>>(a, io);
        else
          distill_kernel<LT, NWR, NP, false, PASS><<<grid, wg, 0, st>>>(a, io);
      }
    });
  };
  if (p.n_seg == 1) return pass(all, Int<kWhole>());
  hipError_t e = pass(all, Int<kStats>());
  if (e == hipSuccess && io.loss) {
    Rows a = all;
    in_launches(a.n_rows, kThreads / 64, kThreads, 1, [&](int64_t r, dim3 grid) {
      a.row0 = r;
      distill_loss_kernel<LT><<<grid, kThreads, 0, st>>>(a, io);
    });
    e = hipGetLastError();
  }
  return e == hipSuccess && io.grad ? pass(all, Int<kApply>()) : e;
}

}  // namespace rows
}  // namespace tbias
