// Log probabilities of given tokens, log-sum-exp, entropy and the M best
// alternatives of every row (templates; instantiated in rows_score_*.hip).
#pragma once

#include "rows.hpp"

namespace tbias {
namespace rows {

// Writes what follows from a row's statistics; one wave.
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

// The i-th alternative of a row (or segment).
template <bool PART>
__device__ __forceinline__ void write_alt(const Rows& a, const ScoreIO& io, int64_t row, int i,
                                          float z, int32_t id, const Basis& b, float log_s) {
  if (PART) {
    io.lists[(row * a.n_seg + blockIdx.y) * io.M + i] = make_int2(__float_as_int(z), id);
  } else {
    io.alt[row * io.M + i] = id;
    io.alt_logprob[row * io.M + i] = id < 0 ? kNegInf : log_prob(z, b, log_s, a.inv_tau);
  }
}

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

template <class LT, int NWR, int NP, bool TOP, bool PART>
__global__ __launch_bounds__(Place<NWR>::kWg) void score_kernel(Rows a, ScoreIO io) {
  typedef Tile<LT, NWR, NP> T;
  constexpr int PV = T::PV;
  __shared__ float box[4 * NWR], box_z[NWR];
  __shared__ int32_t box_id[NWR];
  lds_poison(box, sizeof(box));
  const Place<NWR> at(a);
  if (at.row >= a.n_rows) return;  // uniform over the row's waves
  const LT* z = static_cast<const LT*>(a.z) + at.row * a.stride;
  T x;
  x.load(z + at.c0, at.n, at.lane, at.q);
  Basis b;
  const float lm = x.lane_max();
  const Stats s = PART || io.entropy
                      ? statistics<true, false>(x, a.c, lm, nullptr, box, b)
                      : statistics<false, false>(x, a.c, lm, nullptr, box, b);
  const float log_s = log_sum(s, b);
  if (at.q == 0) {
    if (PART) {
      if (at.lane == 0) a.part[at.row * a.n_seg + blockIdx.y] = to_part(s, b);
    } else {
      write_scores(a, io, at.row, z, s, b, log_s, at.lane);
    }
  }
  if (!TOP) return;
  // one alternative after the other: the best of those that come after the last
  float lz = __builtin_huge_valf();
  int32_t li = -1;
  for (int i = 0; i < io.M; ++i) {
    float bz = kNegInf;
    int32_t bi = INT_MAX;
    auto see = [&](float v, int32_t id) {
      if ((v < lz || (v == lz && id > li)) && v > bz) {
        bz = v;
        bi = id;
      }
    };
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int e = 0; e < PV; ++e) see(x.at(p, e), x.first(p) + e);
    see(x.tail, x.tail_at());
    x.repack();
    row_best<NWR>(bz, bi, box_z, box_id, at.q, at.lane);
    if (at.q == 0 && at.lane == 0)
      write_alt<PART>(a, io, at.row, i, bz, bz == kNegInf ? -1 : at.c0 + bi, b, log_s);
    lz = bz;
    li = bi;
  }
}

// Joins the segments of a row: one wave per row.
template <class LT>
__global__ __launch_bounds__(kThreads) void score_join_kernel(Rows a, ScoreIO io) {
  const int lane = __lane_id();
  const int64_t row = a.row0 + (int64_t)blockIdx.x * (kThreads / 64) +
                      __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= a.n_rows) return;
  const LT* z = static_cast<const LT*>(a.z) + row * a.stride;
  Basis b;
  const Stats s = join(a.part + row * a.n_seg, a.n_seg, a.c, lane, b);
  const float log_s = log_sum(s, b);
  write_scores(a, io, row, z, s, b, log_s, lane);
  // merge: every lane holds the best that its segment's list has left
  const int2* list = io.lists + (row * a.n_seg + lane) * io.M;
  int at = 0;
  int2 head = make_int2(__float_as_int(kNegInf), INT_MAX);
  if (io.M > 0 && lane < a.n_seg) head = list[0];
  for (int i = 0; i < io.M; ++i) {
    float bz;
    int32_t bi;
    const int own = wave_argmax_dpp(__int_as_float(head.x), head.y < 0 ? INT_MAX : head.y, bz, bi);
    if (lane == 0)
      write_alt<false>(a, io, row, i, bz, bz == kNegInf ? -1 : bi, b, log_s);
    if (lane == own) {
      ++at;
      head = at < io.M && lane < a.n_seg ? list[at] : make_int2(__float_as_int(kNegInf), INT_MAX);
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
      } else if (io.M > 0) {
        score_kernel<LT, NWR, NP, true, false><<<grid, Pl::kWg, 0, st>>>(a, io);
      } else {
        score_kernel<LT, NWR, NP, false, false><<<grid, Pl::kWg, 0, st>>>(a, io);
      }
    });
  });
  if (p.n_seg > 1)
    in_launches(a.n_rows, kThreads / 64, kThreads, 1, [&](int64_t r, dim3 grid) {
      a.row0 = r;
      score_join_kernel<LT><<<grid, kThreads, 0, st>>>(a, io);
    });
  return hipGetLastError();
}

}  // namespace rows
}  // namespace tbias
