// AdamW over many tensors. A value costs its bytes: parameter, gradient and moments
// are read once and written once, with the arithmetic between in registers.
//
// Moments in 8 bits are sizes times a unit that 256 neighbouring values share (two
// floats for 512 bytes of codes). A size has runs of 2^P codes whose step doubles from
// the second run on, so its error is about even over three decades: P = 4 and a sign
// for the first moment, sizes up to 1984; P = 5 for the root of the second, up to
// 4032 (the second moment itself is size^2 times the unit). A step changes a second
// moment by one part in a thousand, far less than half a code: rounded to the nearest
// one it would never move. So a moment goes to either neighbour with the probability
// that keeps its mean, from 16 bits that a hash makes of seed, step, tensor and place.
// A second moment above 0 never becomes 0, which would make the next step a large one.
//
// What bounds it, in 235 million bfloat16 values of 290 tensors: with 32-bit states and copies
// its bytes (28 a value, 1.35 ms, 4.9 TB/s; a large copy runs at 5.3), with 8-bit states (10 a
// value) its instructions (0.62 ms, 3.8 TB/s), reading the moments their bytes (0.45 ms for 10
// a value, 5.2 TB/s). Up to 52 tensors go into a launch, since their records fit its
// arguments, so that a table need not be copied to the device first, which a captured graph
// could not do again. A lane takes 8 values at a time, 16-byte loads at any address, the next
// ones in flight while it works: without that 1.40 ms and 0.78. Loads and stores that leave
// the caches alone were slower (1.66 ms; 5 million float32 values 38 us instead of 25).
//
// The moments' products and sums are rounded one by one, in float32, as the interface
// states them, so the codes are the same wherever the same arithmetic runs.
#include "adamw.hpp"

#include <cmath>

namespace tbias {
namespace adamw {

namespace {

constexpr int kThreads = 256, kEach = 8;           // values of a lane at a time
constexpr int kChunk = kThreads * kEach * 4;       // values of a workgroup
constexpr float kTopM = 1.f / 1984.f, kTopV = 1.f / 16257024.f;  // 1 / largest size, 1 / its square

struct Rec {
  void* param;
  const void* grad;
  void *m, *v;
  float *m_unit, *v_unit;
  float* master;
  int64_t n;
};

struct Args {
  Rec rec[kMost];
  int32_t end[kMost];    // chunks up to and with a tensor
  int32_t index[kMost];  // of a tensor in the call
  int32_t count;
  float decay, size, root, b1, c1, b2, c2, eps;
  uint32_t key;
  double lr, beta1, beta2, weight_decay;
  const float* lr_dev;
  const int64_t* step_dev;
  const float* grad_scale;
  int64_t step;
  uint32_t seed;
};
static_assert(sizeof(Args) <= 4096, "kernel arguments");

__host__ __device__ inline uint32_t mix(uint32_t h) {
  h ^= h >> 16;
  h *= 0x7feb352du;
  h ^= h >> 15;
  h *= 0x846ca68bu;
  return h ^ (h >> 16);
}

typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

__device__ __forceinline__ uint16_t to_bf16(float v) {
  return __builtin_bit_cast(uint16_t, (__bf16)v);
}

// Sixteen (eight) bytes at the alignment of one element: the memory takes them anywhere.
typedef uint32_t Words4 __attribute__((ext_vector_type(4)));
typedef uint32_t Words2 __attribute__((ext_vector_type(2)));
typedef Words4 Quad4 __attribute__((aligned(4)));
typedef Words4 Quad2 __attribute__((aligned(2)));
typedef Words2 Pair1 __attribute__((aligned(1)));

// Eight values, or (FULL false) the `left` there are.
template <bool FULL>
__device__ __forceinline__ void load8(const float* p, int left, float* v) {
  if (FULL || left >= 8) {
    const Words4 a = reinterpret_cast<const Quad4*>(p)[0], b = reinterpret_cast<const Quad4*>(p)[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = __uint_as_float(a[e]);
      v[4 + e] = __uint_as_float(b[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < left ? p[e] : 0.f;
  }
}
template <bool FULL>
__device__ __forceinline__ void load8(const uint16_t* p, int left, float* v) {
  if (FULL || left >= 8) {
    const Words4 a = *reinterpret_cast<const Quad2*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(a[e] << 16);
      v[2 * e + 1] = __uint_as_float(a[e] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < left ? __uint_as_float((uint32_t)p[e] << 16) : 0.f;
  }
}
template <bool FULL>
__device__ __forceinline__ void store8(float* p, int left, const float* v) {
  if (FULL || left >= 8) {
    Words4 a, b;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      a[e] = __float_as_uint(v[e]);
      b[e] = __float_as_uint(v[4 + e]);
    }
    reinterpret_cast<Quad4*>(p)[0] = a;
    reinterpret_cast<Quad4*>(p)[1] = b;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) p[e] = v[e];
  }
}
template <bool FULL>
__device__ __forceinline__ void store8(uint16_t* p, int left, const float* v) {
  if (FULL || left >= 8) {
    Words4 a;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x2 x = {v[2 * e], v[2 * e + 1]};
      a[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
    }
    *reinterpret_cast<Quad2*>(p) = a;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) p[e] = to_bf16(v[e]);
  }
}
template <bool FULL>
__device__ __forceinline__ void load8(const uint8_t* p, int left, uint32_t* c) {
  if (FULL || left >= 8) {
    const Words2 a = *reinterpret_cast<const Pair1*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      c[e] = (a[0] >> (8 * e)) & 255;
      c[e + 4] = (a[1] >> (8 * e)) & 255;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = e < left ? p[e] : 0;
  }
}
template <bool FULL>
__device__ __forceinline__ void store8(uint8_t* p, int left, const uint32_t* c) {
  if (FULL || left >= 8) {
    Words2 a = {0, 0};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      a[0] |= c[e] << (8 * e);
      a[1] |= c[e + 4] << (8 * e);
    }
    *reinterpret_cast<Pair1*>(p) = a;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) p[e] = (uint8_t)c[e];
  }
}

// A code as bits of a float: its run in the exponent, its place in the run in the mantissa,
// and the first run among the denormals, so that one product (a denormal operand is exact)
// gives its size times 2^-P.
template <int P>
__device__ __forceinline__ float size_of(uint32_t code) {
  return __uint_as_float(code << (23 - P)) * 0x1p126f;
}
// `unit` is the block's times 2^4 and 2^10, which undoes the 2^-P: exact powers of two.
__device__ __forceinline__ float decode_m(uint32_t code, float unit) {
  const float s = size_of<4>(code & 127) * unit;
  return __uint_as_float(__float_as_uint(s) | (code << 24 & 0x80000000u));
}
__device__ __forceinline__ float decode_v(uint32_t code, float unit) {
  const float s = size_of<5>(code);
  return s * s * unit;
}

// The run of a size below 2^(P + 7): e with size * 2^-e below 2^(P + 1).
template <int P>
__device__ __forceinline__ int run_of(float size) {
  return max(__builtin_amdgcn_frexp_expf(size) - (P + 1), 0);
}

// A block's largest value is at most 4 * 2^-24 of itself above the largest size (the
// roundings of 1 / top, unit, 1 / unit and the product), which is less than the smallest
// rnd of 2^-17 lets round up: no code is above the last one.
__device__ __forceinline__ uint32_t encode_m(float m, float inverse, float rnd) {
  const float y = fabsf(m) * inverse;
  const int e = run_of<4>(y);
  const float q = __builtin_amdgcn_ldexpf(y, -e);
  const uint32_t code = (e << 4) + (uint32_t)q + (__builtin_amdgcn_fractf(q) > rnd ? 1 : 0);
  return code | (m < 0.f ? 128u : 0u);
}
// The square root may be off by some steps: where that moves it over a whole number i, the
// value lies within i^2 2^-22 of i^2, and the comparison takes it to i from either
// side (its right side is at least (2 i - 1) 2^-17 from both ends, and i is below 64).
__device__ __forceinline__ uint32_t encode_v(float v, float inverse, float rnd) {
  const float y = v * inverse, root = __builtin_amdgcn_sqrtf(y);
  const int e = run_of<5>(root);
  const float low = floorf(__builtin_amdgcn_ldexpf(root, -e));
  const float over = __builtin_fmaf(-low, low, __builtin_amdgcn_ldexpf(y, -2 * e));
  const bool up = over > __builtin_fmaf(2.f, low, 1.f) * rnd;
  const uint32_t code = (e << 5) + (uint32_t)low + (up ? 1 : 0);
  return max(code, min(__float_as_uint(v), 1u));
}

// 2^-16 (r + 1 / 2)
__device__ __forceinline__ float fraction(uint32_t r) {
  return __builtin_fmaf((float)r, 0x1p-16f, 0x1p-17f);
}

// Largest of the 32 lanes that hold a block, of bits of floats without their signs: those
// of infinity and NaN lie above all others.
__device__ __forceinline__ uint32_t block_max(uint32_t v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d));
  return v;
}

// The unit of a block; NaN where it holds a value that is not finite.
__device__ __forceinline__ float unit_of(uint32_t most, float top) {
  const float unit = __uint_as_float(most) * top;
  return most >= 0x7f800000u ? __builtin_nanf("") : unit >= 0x1p-100f ? unit : 0.f;
}

// The tensor of a chunk: the first whose end is behind it.
template <class A>
__device__ __forceinline__ int find(const A& a, int chunk) {
  const int lane = threadIdx.x & 63;
  const bool before = lane < a.count && a.end[min(lane, kMost - 1)] <= chunk;
  return __builtin_amdgcn_readfirstlane(__popcll(__ballot(before)));
}

struct Consts {
  float decay, size, root;
  uint32_t key;
};

__host__ __device__ inline Consts consts(double lr, double beta1, double beta2, double wd,
                                         int64_t step, uint32_t seed) {
  Consts c;
  c.decay = (float)(1.0 - lr * wd);
  c.size = (float)(lr / (1.0 - pow(beta1, (double)step)));
  c.root = (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step)));
  c.key = mix(seed ^ mix((uint32_t)step));
  return c;
}

// What a lane holds of its eight values.
template <class T, int BITS>
struct Eight {
  float p[8], g[8];
  float m[8], v[8];   // 32 bits
  uint32_t cm[8], cv[8];  // 8 bits
  float um, uv;
};

// Eight values from i on, or (FULL false) the `left` there are.
template <class T, int BITS, bool MASTER, bool FULL>
__device__ __forceinline__ void load(const Rec& r, int64_t i, int left, Eight<T, BITS>* x) {
  if (MASTER) load8<FULL>(r.master + i, left, x->p);
  else load8<FULL>(static_cast<const T*>(r.param) + i, left, x->p);
  load8<FULL>(static_cast<const T*>(r.grad) + i, left, x->g);
  if constexpr (BITS == 32) {
    load8<FULL>(static_cast<const float*>(r.m) + i, left, x->m);
    load8<FULL>(static_cast<const float*>(r.v) + i, left, x->v);
  } else {
    load8<FULL>(static_cast<const uint8_t*>(r.m) + i, left, x->cm);
    load8<FULL>(static_cast<const uint8_t*>(r.v) + i, left, x->cv);
    x->um = r.m_unit[i / kBlock];
    x->uv = r.v_unit[i / kBlock];
  }
}

template <class T, int BITS, bool MASTER, bool FULL>
__device__ __forceinline__ void update(const Args& a, const Rec& r, const Consts& c, float gs,
                                       uint32_t key, int64_t i, int left, Eight<T, BITS>* x) {
  if constexpr (BITS == 8) {
    const float um = x->um * 0x1p4f, uv = x->uv * 0x1p10f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x->m[e] = decode_m(x->cm[e], um);
      x->v[e] = decode_v(x->cv[e], uv);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float g = x->g[e] * gs;
    x->m[e] = x->m[e] * a.b1 + g * a.c1;
    x->v[e] = x->v[e] * a.b2 + g * a.c2 * g;
    const float n = x->m[e] * c.size;
    if constexpr (BITS == 32) {
      x->p[e] = x->p[e] * c.decay - n / (sqrtf(x->v[e]) * c.root + a.eps);
    } else {
      // root and reciprocal to a step each: their last bits would take a fifth of the
      // kernel's instructions, which with 8-bit states bound it
      const float d = __builtin_amdgcn_sqrtf(x->v[e]) * c.root + a.eps;
      x->p[e] = x->p[e] * c.decay - n * __builtin_amdgcn_rcpf(d);
    }
  }
  store8<FULL>(static_cast<T*>(r.param) + i, left, x->p);
  if (MASTER) store8<FULL>(r.master + i, left, x->p);
  if constexpr (BITS == 32) {
    store8<FULL>(static_cast<float*>(r.m) + i, left, x->m);
    store8<FULL>(static_cast<float*>(r.v) + i, left, x->v);
  } else {
    uint32_t top_m = 0, top_v = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (e >= left) x->m[e] = x->v[e] = 0.f;
      top_m = max(top_m, __float_as_uint(x->m[e]) & 0x7fffffffu);
      top_v = max(top_v, __float_as_uint(x->v[e]) & 0x7fffffffu);
    }
    const float um = unit_of(block_max(top_m), kTopM), uv = unit_of(block_max(top_v), kTopV);
    const float im = um > 0.f ? 1.f / um : 0.f, iv = uv > 0.f ? 1.f / uv : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t bits = mix((uint32_t)(i + e) + key);
      x->cm[e] = encode_m(x->m[e], im, fraction(bits & 0xffff));
      x->cv[e] = encode_v(x->v[e], iv, fraction(bits >> 16));
    }
    store8<FULL>(static_cast<uint8_t*>(r.m) + i, left, x->cm);
    store8<FULL>(static_cast<uint8_t*>(r.v) + i, left, x->cv);
    if ((threadIdx.x & 31) == 0 && left > 0) {
      r.m_unit[i / kBlock] = um;
      r.v_unit[i / kBlock] = uv;
    }
  }
}

// A whole chunk takes no checks, and its next values are loaded before the present ones
// are worked on.
template <class T, int BITS, bool MASTER>
__global__ void __launch_bounds__(kThreads) step_kernel(const Args a) {
  constexpr int kStep = kThreads * kEach;
  const int chunk = blockIdx.x;
  const int k = find(a, chunk);
  const Rec r = a.rec[k];
  const int64_t begin = (int64_t)(chunk - (k ? a.end[k - 1] : 0)) * kChunk;

  Consts c = {a.decay, a.size, a.root, a.key};
  if (a.lr_dev || a.step_dev) {
    __shared__ Consts shared;
    if (threadIdx.x == 0)
      shared = consts(a.lr_dev ? (double)*a.lr_dev : a.lr, a.beta1, a.beta2, a.weight_decay,
                      a.step_dev ? *a.step_dev : a.step, a.seed);
    __syncthreads();
    c = shared;
  }
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  const uint32_t key = mix(c.key + (uint32_t)a.index[k]);
  const int64_t first = begin + (int64_t)threadIdx.x * kEach;
  if (begin + kChunk <= r.n) {
    Eight<T, BITS> x[2];
    load<T, BITS, MASTER, true>(r, first, 8, &x[0]);
#pragma unroll
    for (int it = 0; it < kChunk / kStep; ++it) {
      if (it + 1 < kChunk / kStep)
        load<T, BITS, MASTER, true>(r, first + (it + 1) * kStep, 8, &x[(it + 1) & 1]);
      update<T, BITS, MASTER, true>(a, r, c, gs, key, first + it * kStep, 8, &x[it & 1]);
    }
    return;
  }
#pragma unroll 1
  for (int it = 0; it < kChunk / kStep; ++it) {
    const int64_t i = first + it * kStep;
    const int left = (int)min((int64_t)kEach, max((int64_t)0, r.n - i));
    const int64_t at = left > 0 ? i : 0;  // (no address behind the end)
    Eight<T, BITS> x;
    load<T, BITS, MASTER, false>(r, at, left, &x);
    update<T, BITS, MASTER, false>(a, r, c, gs, key, at, left, &x);
  }
}

struct ReadRec {
  const uint8_t *m, *v;
  const float *m_unit, *v_unit;
  float *out_m, *out_v;
  int64_t n;
};
struct ReadArgs {
  ReadRec rec[kMost];
  int32_t end[kMost];
  int32_t count;
};
static_assert(sizeof(ReadArgs) <= 4096, "kernel arguments");

typedef uint32_t __attribute__((aligned(1))) Four;  // codes, at any address

// Four values a lane, so that the stores fill whole lines.
__global__ void __launch_bounds__(kThreads) moments_kernel(const ReadArgs a) {
  const int chunk = blockIdx.x;
  const int k = find(a, chunk);
  const ReadRec r = a.rec[k];
  const int64_t begin = (int64_t)(chunk - (k ? a.end[k - 1] : 0)) * kChunk;
  if (begin + kChunk <= r.n) {
    // a whole chunk: the loads of four rounds before their stores
    constexpr int kRounds = 4, kEach = kThreads * 4;
#pragma unroll
    for (int half = 0; half < kChunk / (kRounds * kEach); ++half) {
      const int64_t first = begin + half * (kRounds * kEach) + threadIdx.x * 4;
      uint32_t cm[kRounds], cv[kRounds];
      float um[kRounds], uv[kRounds];
#pragma unroll
      for (int it = 0; it < kRounds; ++it) {
        const int64_t i = first + it * kEach;
        cm[it] = *reinterpret_cast<const Four*>(r.m + i);
        cv[it] = *reinterpret_cast<const Four*>(r.v + i);
        um[it] = r.m_unit[i / kBlock] * 0x1p4f;
        uv[it] = r.v_unit[i / kBlock] * 0x1p10f;
      }
#pragma unroll
      for (int it = 0; it < kRounds; ++it) {
        Words4 m, v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          m[e] = __float_as_uint(decode_m(cm[it] >> (8 * e) & 255, um[it]));
          v[e] = __float_as_uint(decode_v(cv[it] >> (8 * e) & 255, uv[it]));
        }
        *reinterpret_cast<Quad4*>(r.out_m + first + it * kEach) = m;
        *reinterpret_cast<Quad4*>(r.out_v + first + it * kEach) = v;
      }
    }
    return;
  }
  for (int64_t i = begin + threadIdx.x * 4; i < r.n; i += kThreads * 4) {
    const float um = r.m_unit[i / kBlock] * 0x1p4f, uv = r.v_unit[i / kBlock] * 0x1p10f;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < r.n) {
        r.out_m[i + e] = decode_m(r.m[i + e], um);
        r.out_v[i + e] = decode_v(r.v[i + e], uv);
      }
  }
}

template <class T, int BITS, bool MASTER>
void launch(const Args& a, int64_t chunks, hipStream_t st) {
  step_kernel<T, BITS, MASTER><<<dim3((unsigned)chunks), dim3(kThreads), 0, st>>>(a);
}

// Groups of up to kMost tensors whose chunks make a launch: put(k, i) takes tensor i as
// the k-th of a group, go(k, chunks) launches it.
template <class Put, class Go>
hipError_t groups(const tb_adamw_tensor* t, int32_t n, Put put, Go go) {
  const int64_t most = most_groups(kThreads);
  int32_t k = 0;
  int64_t chunks = 0;
  for (int32_t i = 0; i < n; ++i) {
    if (t[i].n == 0) continue;
    const int64_t c = (t[i].n + kChunk - 1) / kChunk;
    if (k == kMost || chunks + c > most) {
      if (k > 0) go(k, chunks);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      k = 0;
      chunks = 0;
    }
    chunks += c;
    put(k++, i, (int32_t)chunks);
  }
  if (k > 0) go(k, chunks);
  return hipGetLastError();
}

}  // namespace

hipError_t step(const tb_adamw_tensor* t, int32_t n, const Step& s, hipStream_t st) {
  Args a = {};
  const Consts c = consts(s.lr, s.beta1, s.beta2, s.weight_decay, s.step, s.seed);
  a.decay = c.decay;
  a.size = c.size;
  a.root = c.root;
  a.key = c.key;
  a.b1 = (float)s.beta1;
  a.c1 = (float)(1.0 - s.beta1);
  a.b2 = (float)s.beta2;
  a.c2 = (float)(1.0 - s.beta2);
  a.eps = (float)s.eps;
  a.lr = s.lr;
  a.beta1 = s.beta1;
  a.beta2 = s.beta2;
  a.weight_decay = s.weight_decay;
  a.lr_dev = s.lr_dev;
  a.step_dev = s.step_dev;
  a.grad_scale = s.grad_scale;
  a.step = s.step;
  a.seed = s.seed;
  return groups(
      t, n,
      [&](int32_t k, int32_t i, int32_t end) {
        a.rec[k] = {t[i].param, t[i].grad, t[i].m, t[i].v, t[i].m_unit, t[i].v_unit,
                    t[i].master, t[i].n};
        a.end[k] = end;
        a.index[k] = i;
      },
      [&](int32_t k, int64_t chunks) {
        a.count = k;
        if (s.dtype == TB_F32) {
          if (s.bits == 32) launch<float, 32, false>(a, chunks, st);
          else launch<float, 8, false>(a, chunks, st);
        } else if (s.master) {
          if (s.bits == 32) launch<uint16_t, 32, true>(a, chunks, st);
          else launch<uint16_t, 8, true>(a, chunks, st);
        } else {
          if (s.bits == 32) launch<uint16_t, 32, false>(a, chunks, st);
          else launch<uint16_t, 8, false>(a, chunks, st);
        }
      });
}

hipError_t moments(const tb_adamw_tensor* t, int32_t n, float* const* out_m, float* const* out_v,
                   hipStream_t st) {
  ReadArgs a = {};
  return groups(
      t, n,
      [&](int32_t k, int32_t i, int32_t end) {
        a.rec[k] = {static_cast<const uint8_t*>(t[i].m), static_cast<const uint8_t*>(t[i].v),
                    t[i].m_unit, t[i].v_unit, out_m[i], out_v[i], t[i].n};
        a.end[k] = end;
      },
      [&](int32_t k, int64_t chunks) {
        a.count = k;
        moments_kernel<<<dim3((unsigned)chunks), dim3(kThreads), 0, st>>>(a);
      });
}

}  // namespace adamw
}  // namespace tbias
