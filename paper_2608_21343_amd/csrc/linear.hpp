// Cross entropy of a linear layer without its logits: what the kernels share.
//
//   z = x w^T + b, lse_i = log sum_c exp z_ic, loss_i = weight_i (lse_i - z_i,t(i)),
//   G_ic = a_i exp(z_ic - lse_i) - b_i [c = t(i)], dx = G w, dw = G^T x, db = sum_i G_i
//
// with b_i = weight_i d_loss_i and a_i = b_i + d_lse_i. All four products run on the
// matrix cores as 16-bit operands with float32 sums (linear_gemm.hpp).
//
// bfloat16 operands are taken as they are, and G is rounded to bfloat16. Up to 32 rows leave
// room in a tile for what that rounding left, as rows of their own: with many rows the
// roundings of G average out, but a few rows' would show in their gradients (two rows of 127
// against 339 tokens: dx off by 2.7e-3 of its norm, and 1.6e-3, the rounding of dx itself,
// with them; a step of 8 rows of 512 against 1025 tokens takes 39 us and 35 without).
//
// A float32 operand is the sum of two float16 planes, the second the rounding of what
// the first leaves: 22 bits and a second sign, so up to 2^-23 of a value is lost. A product
// of two such operands is the sum of three products of planes; the fourth is at most 2^-22
// of it. (Three bfloat16 planes hold a little more but take six products: forward and
// backward of 2048 x 1024 features against 32,769 tokens took 3.4 ms with them and 1.9 with
// these, when the rest was the same.)
//
// What float16 lacks is range: 2^-14 to 2^16, and absolute steps of 2^-24 below. So rows of x
// are divided by powers of two r_i, and all of w by one, S, that bring their largest value
// to 2^14..2^15. A value below 2^-16 of that largest loses precision, at most 2^-39 of it;
// an entry of G below 2^-16 of its row's weight at most 2^-39 of that weight:
//
//   z_ic  = (x_i / r_i) (w_c / S) r_i S
//   G'_ic = G_ic / m_i * 2^14,  m_i = max(|a_i|, |b_i|)
//   dx_i  = G'_i (w / S) * m_i S 2^-14
//   dw_c  = G'_c^T (x_i m_i / T) * T 2^-14,  T a power of two for all rows
//
// so that a row's gradient is as exact as if it were alone, whatever the others weigh. (With
// a unit for each token G' would have to carry it too, and a token of small weights would
// lose its gradient.) Tokens that the bias masks have no say in S, whatever they hold.
//
// lse_i is the sum of a row's maximum and a logarithm, and its rounding would be a relative
// error of p that shows in p - 1 where p is near 1. Where the statistics are of the same
// call, a_i is divided by the sum and the maximum taken for lse_i; else the caller may hand
// over what the rounding left.
//
// Rows that take part (target not -1, weight not 0) are gathered first, so that the
// others cost nothing and whatever they hold reaches no sum. Rows of the gathered
// matrix end at a multiple of 64 values, and its rows at one of 64, with zeros.
#pragma once

#include "device.hpp"
#include "launch.hpp"

namespace tbias {
namespace linear {

constexpr int kStep = 64;    // values of the summed axis that a tile takes at a time
constexpr int kTile = 256;   // rows and columns of the largest tile
constexpr int kPair = 32;    // bfloat16 rows whose gradients may be kept twice
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__host__ __device__ inline int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// Left by the gathering of the rows, read by every later kernel.
struct Meta {
  int32_t n;  // gathered rows
  // bfloat16: G is kept divided by the largest finite |a_i|, |b_i|. With equal weights, as
  // the mean over a batch has, the target's entry p - 1 is then rounded near 1 and not
  // every row's by the same part of the weight (up to 2^-8, which no sum averages out).
  float scale, inverse;
  float S;        // float32 only, as is
  uint32_t T;     // the bits of the largest |x_i m_i|
};

// A matrix as 16-bit planes. Element (i, k), k the summed axis, lies in row i at value k,
// or (transposed) in row k at value i; ld: 16-bit values from row to row. i < n and
// k < kn are in memory; a row ends at a multiple of 8 values, 16-byte aligned. Two planes
// lie in turns of 32 values, so that 64 of a row's are 32 of the matrix's, whole.
struct Operand {
  const uint16_t* p;
  int64_t ld;
  int32_t n, kn;
};

// Where value c of a row's first plane lies, and how much further on the next plane's.
constexpr int kTurn = 32;
template <int PLANES>
__host__ __device__ inline int64_t place(int64_t c) {
  return PLANES == 1 ? c : 2 * c - (c & (kTurn - 1));
}

// Per gathered row.
struct RowArgs {
  const int32_t* target;  // -1: none in range
  const float *a, *b, *lse;  // float32: a and b divided by m
  const float *r, *m;        // float32 only
};

struct Gemm {
  Operand P, Q;  // result element (p, q): sum over k of P(p, k) Q(q, k)
  const Meta* meta;
  int32_t tile, tp, tq, splits;  // size of a tile (256, 128, 64), and their numbers
  int32_t k;       // length of the summed axis, a multiple of kStep
  int32_t n_q;     // columns of the result that are kept
  // statistics and gradients of the logits
  const void* bias;
  int32_t C, c0;   // tokens, and the first of P
  RowArgs row;
  float2* part;    // [gathered row, n_part]: maximum, sum
  int32_t n_part;
  float* hit;      // logit of the row's target
  float* z;        // [gathered row, ldg] the logits, where they are kept
  uint16_t* G;     // planes of [row, ldg]
  int32_t ldg;
  float* col;      // [row tiles, ldg], or NULL
  // products with the gradients
  float* acc;      // [split, n_q, lda]
  int64_t acc_split;
  int32_t lda, add;  // add: to what is there
  bool paired;       // dx: rows and, kPair further on, what their gradients' rounding left
  void* out;         // or the result itself: [q, ldo] (dx: [idx[q], ldo]), D values
  const int32_t* idx;
  int64_t ldo;
  int32_t D;
};

enum { kStats, kLogitGrad, kDx, kDw };

// Statistics of the logits of few rows (linear_few.hip), by their place in x.
struct Few {
  const void *x, *w, *bias;
  int64_t x_stride, w_stride;
  int32_t n, D, C;
  const int32_t* target;
  int32_t parts, each;  // waves that share the tokens, and units of 16 tokens of a wave
  float2* part;   // [n, parts]
  float* hit;     // [n]
  float* z;       // [n, ldz] the logits, -inf up to a multiple of 16 tokens; or NULL
  int32_t ldz;
};
int32_t few_each(int32_t C);
int32_t few_parts(int32_t C);
hipError_t few(const Few& f, int32_t dtype, hipStream_t st);

// One launch over tp * tq * splits tiles.
hipError_t stats_bf16(const Gemm& g, hipStream_t st);
hipError_t stats_f32(const Gemm& g, hipStream_t st);
hipError_t logit_grad_bf16(const Gemm& g, hipStream_t st);
hipError_t logit_grad_f32(const Gemm& g, hipStream_t st);
hipError_t dx_bf16(const Gemm& g, hipStream_t st);
hipError_t dx_f32(const Gemm& g, hipStream_t st);
hipError_t dw_bf16(const Gemm& g, hipStream_t st);
hipError_t dw_f32(const Gemm& g, hipStream_t st);

// A call, after its checks.
struct Call {
  const void *x, *w, *bias;
  int32_t dtype;
  int64_t n;
  int32_t D, C;
  int64_t x_stride, w_stride;
  const int32_t* target;
  const float *weight, *d_loss, *d_lse;
  int32_t d_step;    // from row to row of d_loss: 1, or 0 for one value
  const float *lse, *lse_low;  // of an earlier call, or NULL: computed here
  float *out_loss, *out_lse, *out_low;
  void *dx, *dw, *db;
  int64_t dx_stride, dw_stride;
};

// How a product is cut into tiles, and in which parts of the summed axis.
struct Cut {
  int32_t tile, parts;
  double cost;
};
// The tokens of a product: those in whole tiles of 256, and the few behind them.
struct Strips {
  int32_t main;  // tokens of the first
  Cut cut[2];
};
// How a call is done, and where its buffers lie in the workspace.
struct Layout {
  int64_t np, dp, planes;      // gathered rows and values a row, rounded up
  int64_t rows_g, rows_x;      // rows of the logits' gradients, and of dx's sums
  bool copy_w, few, gather, paired;
  bool kept;                   // the logits, from the statistics to their gradients
  int32_t n_part;
  // tokens of a piece of the vocabulary (of all but the last), and of a row of gradients
  int32_t piece, pieces, ldg;
  Strips stats, grad, w;       // of the products with tokens of their own ...
  Cut grad_all, w_all;         // (pieces but the last)
  Cut x;                       // ... and that which sums over them
  int32_t kept_rows;           // of a workgroup that makes gradients of kept logits
  bool direct;                 // dx leaves its product's sums as it is
  int64_t meta, counts, tops, idx, inv, tgt, a, b, lse, r, m, most, hit, part, px, pxm, pw;
  int64_t z, G, acc_x, acc_w, col, total;
};

// The plan of a call (its workspace: `total` bytes); the bytes that suffice for every x of
// a call's sizes; the launches.
Layout plan(const Call& c);
int64_t most_workspace(Call c);
hipError_t run(const Call& c, const Layout& L, void* workspace, hipStream_t st);

}  // namespace linear
}  // namespace tbias
