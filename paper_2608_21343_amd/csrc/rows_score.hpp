// Log probabilities of given tokens, log-sum-exp, entropy and the M best
// alternatives of every row (templates; instantiated in rows_score_*.hip).
#pragma once

#include "rows.hpp"

namespace tbias {
namespace rows {

// Writes what follows from a row's statistics; one wave. (The given tokens are read
// here: read before the row they are waited for together with it, which gains
// nothing: 7511 rows of 612 bfloat16 9.5 us instead of 9.2.)
template <class LT>
__device__ __forceinline__ void write_scores(const Rows& a, const ScoreIO& io, int64_t row,
                                             const LT* z, const Stats& s, const Basis& b,
                                             float log_s, int lane) {
  if (lane == 0) {
    if (io.lse) io.lse[row] = b.m * a.inv_tau + (empty(s) ? kNegInf : log_s);
    if (io.entropy) io.entropy[row] = entropy(s);
  }
  if (lane < io.J) {
    const int32_t id = io.tokens[row * io.J + lane];
    float lp = 0.f;  // -1: no token
    if ((uint32_t)id < (uint32_t)a.C)
      lp = log_prob(Elem<LT>::widen(z[id]), b, log_s, a.inv_tau);
    else if (id != -1)
      lp = __builtin_nanf("");
    io.logprob[row * io.J + lane] = lp;
  }
}

// Where a row's (or segment's) alternatives are written.
template <bool PART>
struct AltRow {
  int32_t* id;
  float* logprob;
  int2* list;
  float log_s, m, inv_tau;
  __device__ inline AltRow(const Rows& a, const ScoreIO& io, int64_t row, const Basis& b,
                           float log_s_) {
    if (PART) {
      list = io.lists + (row * a.n_seg + blockIdx.y) * io.M;
    } else {
      id = io.alt + row * io.M;
      logprob = io.alt_logprob + row * io.M;
    }
    log_s = log_s_;
    m = b.m;
    inv_tau = a.inv_tau;
  }
  __device__ inline void write(int i, float z, int32_t token) const {
    if (PART) {
      list[i] = make_int2(__float_as_int(z), token);
    } else {
      id[i] = token;
      logprob[i] = (z - m) * inv_tau - log_s;
    }
  }
  __device__ inline void none(int i) const {
    if (PART) {
      list[i] = make_int2(__float_as_int(kNegInf), -1);
    } else {
      id[i] = -1;
      logprob[i] = kNegInf;
    }
  }
};

// Best (z, id) over the row's waves of every wave's own best.
template <int NWR>
__device__ __forceinline__ void row_best(float& z, int32_t& id, float* box_z, int32_t* box_id,
                                         int q, int lane) {
  float bz;
  int32_t bi;
  wave_argmax_dpp(z, id, bz, bi);
  if (NWR > 1) {
    __syncthreads();  // the boxes' last readers are done
    if (lane == 0) {
      box_z[q] = bz;
      box_id[q] = bi;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NWR; ++i)
      if (better(box_z[i], box_id[i], bz, bi)) {
        bz = box_z[i];
        bi = box_id[i];
      }
  }
  z = bz;
  id = bi;
}

// ---- the M best values of a row
//
// A value t that M values reach bounds the M-th best from below. The maxima of
// 64 (M > 16: 128) groups of the row's values supply it: t is the M-th best of
// them, and some 1.1 to 1.4 M values reach it. Those are collected in LDS and
// ranked against each other. The maxima are needed for the softmax anyway; the
// rest costs a test per value, some six operations per place of a lane at which
// candidates lie and two per candidate, where one argmax after the other costs
// four operations per value and alternative.

// Floats in an order of whole numbers (-0 as 0), and back.
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_order(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// Lanes that share a group, as a power of two; -1: a lane holds two groups.
template <int NWR>
__device__ __forceinline__ int group_log2(int M) {
  return (NWR == 1 ? 0 : NWR == 2 ? 1 : NWR == 4 ? 2 : 4) - (M > 16 ? 1 : 0);
}
__device__ __forceinline__ float group_max(float v, int log2) {
  if (log2 > 0) v = __builtin_fmaxf(v, dpp_f<0xB1, 0xf>(v, v));   // pairs
  if (log2 > 1) v = __builtin_fmaxf(v, dpp_f<0x4E, 0xf>(v, v));   // quads
  if (log2 > 2) v = __builtin_fmaxf(v, dpp_f<0x141, 0xf>(v, v));  // 8 lanes, mirrored
  if (log2 > 3) v = __builtin_fmaxf(v, dpp_f<0x140, 0xf>(v, v));  // 16 lanes, mirrored
  return v;
}
__device__ __forceinline__ float no_nan(float v) { return v == v ? v : kNegInf; }

// A value that at least `need` (at most 64) of the lanes' a (and, with two, b)
// reach, and few more if it can be: bisection between their least and greatest
// in the order of whole numbers.
__device__ __forceinline__ float reached_by(float a, float b, bool two, int need, float most) {
  if (need == 1) return most;
  const uint32_t ka = order_of(a), kb = order_of(b);
  uint32_t lo = order_of(wave_least(a)), hi = order_of(most);
  while (lo < hi) {  // need values reach lo
    const uint32_t mid = lo + (hi - lo) / 2 + 1;
    int n = __builtin_popcountll(__ballot(ka >= mid));
    if (two) n += __builtin_popcountll(__ballot(kb >= mid));
    if (n < need) {
      hi = mid - 1;
    } else {
      lo = mid;
      if (n == need) break;
    }
  }
  return of_order(lo);
}

// Candidates of a row: those of its waves (value, place), each in its own part
// of the list.
template <int NWR>
struct Found {
  static constexpr int kCap = NWR <= 2 ? 256 : NWR == 4 ? 128 : 64;  // of a wave
  static constexpr int kMost = 256;                                  // of a row
  static constexpr int kKeys = 128;  // ranked by words of 32 bits
  int2 at[NWR][kCap];
  uint4 key[kKeys / 4];
  int32_t n[NWR];
};

// Writes the M best of the row's candidates; one wave. The order is that of
// (value, lower place) as one whole number: of 32 bits for bfloat16 rows of up
// to 2^16 values, also for float32 where no two candidates are equal (which
// shows in the sum of the ranks), else of 64.
template <class LT, int NWR, bool PART>
__device__ __forceinline__ void rank(Found<NWR>& f, const AltRow<PART>& out, int M, int32_t c0,
                                     int32_t n, int lane) {
  int32_t total = 0, count[NWR];
#pragma unroll
  for (int w = 0; w < NWR; ++w) {
    count[w] = __builtin_amdgcn_readfirstlane(f.n[w]);
    total += count[w];
  }
  auto candidate = [&](int32_t i) {  // of all waves'
    int2 c = make_int2(0, 0);
#pragma unroll
    for (int w = 0; w < NWR; ++w) {
      if (i >= 0 && i < count[w]) c = f.at[w][i];
      i -= count[w];
    }
    return c;
  };
  auto write = [&](int2 c, int at) {
    if (at < M) out.write(at, __int_as_float(c.x), c0 + c.y);
  };
  if (total < M && lane >= total && lane < M) out.none(lane);
  constexpr bool kShort = sizeof(LT) == 2;
  if (total <= Found<NWR>::kKeys && (!kShort || n <= 65536)) {
    auto key_of = [&](int2 c) {
      const uint32_t o = order_of(__int_as_float(c.x));
      return kShort ? (o & 0xffff0000u) | (0xffff - c.y) : o;
    };
    uint32_t* keys = reinterpret_cast<uint32_t*>(f.key);
    const int2 c = candidate(lane);
    const uint32_t key = lane < total ? key_of(c) : 0;
    keys[lane] = key;
    bool ties = false;
    if (total <= 64) {
      int at = 0;
      wave_fence();
      for (int j = 0; j < total; j += 4) {
        const uint4 k = f.key[j / 4];
        at += (k.x > key) + (k.y > key) + (k.z > key) + (k.w > key);
      }
      if (!kShort) ties = wave_total_i32(lane < total ? at : 0) != total * (total - 1) / 2;
      if (!ties && lane < total) write(c, at);
    } else {
      const int2 c2 = candidate(64 + lane);
      const uint32_t key2 = 64 + lane < total ? key_of(c2) : 0;
      keys[64 + lane] = key2;
      int at = 0, at2 = 0;
      wave_fence();
      for (int j = 0; j < total; j += 4) {
        const uint4 k = f.key[j / 4];
        at += (k.x > key) + (k.y > key) + (k.z > key) + (k.w > key);
        at2 += (k.x > key2) + (k.y > key2) + (k.z > key2) + (k.w > key2);
      }
      if (!kShort)
        ties = wave_total_i32(at + (64 + lane < total ? at2 : 0)) != total * (total - 1) / 2;
      if (!ties) {
        write(c, at);
        if (64 + lane < total) write(c2, at2);
      }
    }
    if (!ties) return;
  }
  auto whole = [](int2 c) {
    return (uint64_t)order_of(__int_as_float(c.x)) << 32 | (uint32_t)~c.y;
  };
  for (int base = 0; base < total; base += 64) {
    const int2 own = candidate(base + lane);
    const uint64_t key = whole(own);
    int at = 0;
#pragma unroll
    for (int w = 0; w < NWR; ++w)
      for (int j = 0; j < count[w]; ++j) at += whole(f.at[w][j]) > key;
    if (base + lane < total) write(own, at);
  }
}

template <class LT, int NWR, int NP, bool TOP, bool PART>
__global__ __launch_bounds__(Place<NWR>::kWg, least_waves(Shape{NWR, NP})) void score_kernel(
    Rows a, ScoreIO io) {
  typedef Tile<LT, NWR, NP> T;
  constexpr int PV = T::PV;
  __shared__ float box[3 * NWR], box_z[NWR];
  __shared__ int32_t box_id[NWR];
  __shared__ float group[TOP && NWR > 1 ? 128 : 1];
  __shared__ Found<TOP ? NWR : 1> found_all[TOP ? Place<NWR>::kRows : 1];
  lds_poison(box, sizeof(box));
  lds_poison(group, sizeof(group));
  lds_poison(found_all, sizeof(found_all));
  const Place<NWR> at(a);
  if (at.row >= a.n_rows) return;  // uniform over the row's waves
  const LT* z = static_cast<const LT*>(a.z) + at.row * a.stride;
  T x;
  x.load(z + at.c0, at.n, at.lane, at.q);
  Basis b;
  Stats s;
  auto finish = [&](float log_s) {  // one wave
    if (PART) {
      if (at.lane == 0) a.part[at.row * a.n_seg + blockIdx.y] = to_part(s, b);
    } else {
      write_scores(a, io, at.row, z, s, b, log_s, at.lane);
    }
  };
  if constexpr (!TOP) {
    s = PART || io.entropy
            ? statistics<true, false>(x, a.c, nullptr, box, b)
            : statistics<false, false>(x, a.c, nullptr, box, b);
    if (at.q == 0) finish(log_sum(s, b));
  } else {
    // the row's maximum and a bound of its M-th best value
    Found<NWR>& found = found_all[at.slot];
    const int log2 = group_log2<NWR>(io.M);
    const bool two = io.M > 16;
    float g0, g1;
    x.lane_max2(g0, g1);
    g0 = no_nan(g0);
    g1 = no_nan(g1);
    if (log2 >= 0) g0 = group_max(__builtin_fmaxf(g0, g1), log2);
    if (NWR > 1) {
      if ((at.lane & ((1 << log2) - 1)) == 0) group[at.q * (64 >> log2) + (at.lane >> log2)] = g0;
      __syncthreads();
      g0 = group[at.lane];
      if (two) g1 = group[64 + at.lane];
    }
    s.m = wave_most(two ? __builtin_fmaxf(g0, g1) : g0);
    b = Basis::of(s.m, a.c);
    float bound = reached_by(g0, g1, two, io.M, s.m);
    if (bound == kNegInf) bound = -__FLT_MAX__;  // only tokens above -inf
    int32_t n = 0;
    auto see = [&](float val, int32_t id) {
      const uint64_t hit = __ballot(val >= bound);
      if (hit == 0) return;
      const int32_t more = n + __builtin_popcountll(hit);
      if (more <= Found<NWR>::kCap && val >= bound) {
        const int32_t i = __builtin_amdgcn_mbcnt_hi((uint32_t)(hit >> 32),
                                                    __builtin_amdgcn_mbcnt_lo((uint32_t)hit, n));
        found.at[at.q][i] = make_int2(__float_as_int(val), id);
      }
      n = more;
    };
    float v[3] = {0.f, 0.f, 0.f};
    if (b.big)
      x.template sums<true, true, false>(b, nullptr, v, see);
    else
      x.template sums<false, true, false>(b, nullptr, v, see);
    if (at.lane == 0) found.n[at.q] = n;
    if (NWR == 1) wave_fence();
    row_sum<NWR, true, false>(v, box, at.q);  // the waves' candidates are in LDS then, too
    s.S = v[0];
    s.D = v[1];
    s.R = 0.f;
    const float log_s = log_sum(s, b);
    if (at.q == 0) finish(log_s);
    bool over = false;
    int32_t total = 0;
#pragma unroll
    for (int w = 0; w < NWR; ++w) {
      const int32_t k = __builtin_amdgcn_readfirstlane(found.n[w]);
      over |= k > Found<NWR>::kCap;
      total += k;
    }
    const AltRow<PART> out(a, io, at.row, b, log_s);
    if (!over && total <= Found<NWR>::kMost) {
      if (at.q == NWR - 1) rank<LT, NWR, PART>(found, out, io.M, at.c0, at.n, at.lane);
      return;
    }
    // Too many for the list (rows of few different values): one alternative after
    // the other, the best of those that come after the last.
    float lz = __builtin_huge_valf();
    int32_t li = -1;
    for (int i = 0; i < io.M; ++i) {
      float bz = kNegInf;
      int32_t bi = INT_MAX;
      // the places are formed anew in each turn: held, they take a register a value
      int32_t place = x.head + at.lane * PV;
      asm volatile("" : "+v"(place));
      auto best = [&](float val, int32_t id) {
        if ((val < lz || (val == lz && id > li)) && better(val, id, bz, bi) && val > kNegInf) {
          bz = val;
          bi = id;
        }
      };
      x.each([&](int p) {
#pragma unroll
        for (int e = 0; e < PV; ++e)
          best(x.at(p, e), place + (p * NWR + at.q) * 64 * PV + e);
      });
      best(x.rim(), x.rim_at());
      row_best<NWR>(bz, bi, box_z, box_id, at.q, at.lane);
      if (at.q == 0 && at.lane == 0) {
        if (bz == kNegInf)
          out.none(i);
        else
          out.write(i, bz, at.c0 + bi);
      }
      lz = bz;
      li = bi;
    }
  }
}

// Joins the segments of a row: one workgroup of one wave per row, the segments'
// lists in its LDS. The best of them are found as those of a row are: the first
// J places of the n_seg lists hold at least M values, whose M-th best bounds the
// row's. (Merged place by place, each place waits for the last: 8 rows of 131,073
// float32 with 64 alternatives 24.7 us; so 18.4.)
template <class LT>
__global__ __launch_bounds__(64) void score_join_kernel(Rows a, ScoreIO io) {
  extern __shared__ int2 lists[];  // [n_seg, M]
  __shared__ Found<1> found;
  lds_poison(lists, sizeof(int2) * a.n_seg * io.M);
  lds_poison(&found, sizeof(found));
  const int lane = __lane_id();
  const int64_t row = a.row0 + blockIdx.x;
  if (row >= a.n_rows) return;
  const LT* z = static_cast<const LT*>(a.z) + row * a.stride;
  const int M = io.M, n = a.n_seg * M;
  const int2* all = io.lists + row * n;
  for (int i = lane; i < n; i += 64) lists[i] = all[i];
  Basis b;
  const Stats s = join(a.part + row * a.n_seg, a.n_seg, a.c, lane, b);
  const float log_s = log_sum(s, b);
  write_scores(a, io, row, z, s, b, log_s, lane);
  if (M == 0) return;
  wave_fence();
  // place i of list k is value i * n_seg + k of the first J places
  const int J = M < 128 / a.n_seg ? M : 128 / a.n_seg, G = J * a.n_seg;
  auto value = [&](int e) {
    return e < G ? __int_as_float(lists[e % a.n_seg * M + e / a.n_seg].x) : kNegInf;
  };
  const float g0 = value(lane), g1 = value(64 + lane);
  float bound = reached_by(g0, g1, true, M, wave_most(__builtin_fmaxf(g0, g1)));
  if (bound == kNegInf) bound = -__FLT_MAX__;  // only tokens above -inf
  int32_t count = 0;
  for (int base = 0; base < n; base += 64) {
    const int2 c = base + lane < n ? lists[base + lane] : make_int2(__float_as_int(kNegInf), -1);
    const bool in = __int_as_float(c.x) >= bound;
    const uint64_t hit = __ballot(in);
    const int32_t more = count + __builtin_popcountll(hit);
    if (more <= Found<1>::kCap && in)
      found.at[0][__builtin_amdgcn_mbcnt_hi((uint32_t)(hit >> 32),
                                            __builtin_amdgcn_mbcnt_lo((uint32_t)hit, count))] = c;
    count = more;
  }
  if (lane == 0) found.n[0] = count;
  wave_fence();
  const AltRow<false> out(a, io, row, b, log_s);
  if (count <= Found<1>::kCap) {
    rank<LT, 1, false>(found, out, M, 0, a.C, lane);
    return;
  }
  // too many equal values: every lane holds the best that its list has left
  const int2 end = make_int2(__float_as_int(kNegInf), -1);
  const int2* head = lists + lane * M;
  const int2* last = head + M;
  int2 best = lane < a.n_seg ? *head : end;
  for (int i = 0; i < M; ++i) {  // (there are more than M)
    const float v = __int_as_float(best.x), top = wave_most(v);
    const int32_t id = wave_min_i32_dpp(v == top ? best.y : INT_MAX);
    if (v == top && best.y == id) {
      out.write(i, top, id);
      best = ++head < last ? *head : end;
    }
  }
}

template <class LT>
hipError_t score_t(const Rows& a0, const ScoreIO& io, const Plan& p, hipStream_t st) {
  Rows a = a0;
  with_shape<LT>(p.shape, [&](auto nwr, auto np) {
    constexpr int NWR = decltype(nwr)::value, NP = decltype(np)::value;
    typedef Place<NWR> Pl;
    in_launches(a.n_rows, Pl::kRows, Pl::kWg, p.n_seg, [&](int64_t r, dim3 grid) {
      a.row0 = r;
      if (p.n_seg > 1) {
        if constexpr (cuts(Shape{NWR, NP})) {
          if (io.M > 0)
            score_kernel<LT, NWR, NP, true, true><<<grid, Pl::kWg, 0, st>>>(a, io);
          else
            score_kernel<LT, NWR, NP, false, true><<<grid, Pl::kWg, 0, st>>>(a, io);
        }
      } else if constexpr (!fills(Shape{NWR, NP}, Elem<LT>::PV)) {
        if (io.M > 0)
          score_kernel<LT, NWR, NP, true, false><<<grid, Pl::kWg, 0, st>>>(a, io);
        else
          score_kernel<LT, NWR, NP, false, false><<<grid, Pl::kWg, 0, st>>>(a, io);
      }
    });
  });
  if (p.n_seg > 1)
    in_launches(a.n_rows, 1, 64, 1, [&](int64_t r, dim3 grid) {
      a.row0 = r;
      score_join_kernel<LT><<<grid, 64, sizeof(int2) * p.n_seg * io.M, st>>>(a, io);
    });
  return hipGetLastError();
}

}  // namespace rows
}  // namespace tbias
