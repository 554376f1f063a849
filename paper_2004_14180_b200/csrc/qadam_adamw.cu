// AdamW over many tensors at once, moments in 32 or in 8 bits: qadam_adamw_*.
//
//   m = b1 m + c1 g',  v = b2 v + c2 g'^2,  x = x k - a (m / (sqrt(v) b + eps))
//
// One read of gradient, weight and moments, one write of weight and moments, 15 operations an
// element.  With 32-bit moments bound by HBM: 109.5 x 10^6 elements with bf16 gradients and weights and
// master weights, 28 bytes each, in 450 us, 6.8 TB/s.  One launch for all tensors of all types.
#include "qadam.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "qadam_tensors.cuh"

using namespace qadam;

namespace {

constexpr int kAdamThreads = 128;
constexpr int kPair = 256;                                     // elements of two rows: what a warp takes at a time
constexpr int kAdamTile = kAdamThreads / 32 * kPair;           // 1024 elements per CTA
constexpr float kLeastEps = 7.888609052210118e-31f;            // 2^-100: 1 / (root b + eps) is then an ordinary number
constexpr unsigned kLeastScale = 0x00800000u;                  // 2^-126

// A run of at most kAdamTile elements of one tensor.
struct __align__(16) AdamTile {
  void* w;                     // the tensor
  long long begin, at;         // the run's first element: inside the tensor, in the padded layout
  int left;                    // elements of the tensor from there on (no more than 2^30 are counted)
  int seg;
  float decay;
  short wtype, gtype;
  int reserved[2];
};
static_assert(sizeof(AdamTile) == 48, "three 16-byte words");

// What depends on the step, rounded once from binary64.
struct StepScalars {
  double lr;
  float a, b;                  // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
  long long t;
};

__host__ __device__ inline StepScalars step_scalars(double lr, float beta1, float beta2, long long t) {
  StepScalars s;
  s.lr = lr;
  s.a = (float)(lr / (1.0 - pow((double)beta1, (double)t)));
  s.b = (float)(1.0 / sqrt(1.0 - pow((double)beta2, (double)t)));
  s.t = t;
  return s;
}

// Keys of the ten rounds of Philox4x32-10.
struct RoundKeys {
  unsigned k[20];
};

struct AdamParams {
  const AdamTile* tiles;
  int first, num_tiles;        // of this launch
  int pairs;                   // of rows that a warp takes one after the other (8-bit moments)
  int tensor_base;             // tensor of the first gradient pointer
  float beta1, beta2, c1, c2, eps;
  StepScalars now;
  const StepScalars* counted;  // in place of `now` if not NULL
  const float* grad_scale;
  float* master;
  void* m;
  void* v;
  float* m_scale;
  float* r_scale;
  RoundKeys keys;
  unsigned* status;
};

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }

// A code c >= 1 stands for the floating-point number whose leading bits (MANTISSA of the fraction) are c + kBase; the
// top code is 1.0, code 0 is zero.  Four codes lie in a word: the bits of number k go straight from their byte to
// their place in the float, and back.
template <int MANTISSA>
struct Code {
  static constexpr int kDrop = 23 - MANTISSA;
  static constexpr unsigned kTop = MANTISSA == 3 ? 127u : 255u;
  static constexpr unsigned kBase = ((127u << MANTISSA) - kTop) << kDrop;
  __device__ __forceinline__ static unsigned shifted(unsigned word, int left) { return left >= 0 ? word << left : word >> -left; }
  // magnitude of the code in byte k
  __device__ __forceinline__ static float value(unsigned word, int k) {
    const unsigned c = shifted(word, kDrop - 8 * k) & (kTop << kDrop);
    return c == 0u ? 0.0f : __uint_as_float(c + kBase);
  }
  // the code of y in [0, 1], in byte k: `add` < 2^kDrop, then what does not fit is cut off; at least `least` (a code
  // in its float's place)
  __device__ __forceinline__ static unsigned of(float y, unsigned add, unsigned least, int k) {
    const int c = max((int)(__float_as_uint(y) + add - kBase), (int)least);
    return shifted((unsigned)c, 8 * k - kDrop) & (kTop << (8 * k));
  }
};
using CodeM = Code<3>;
using CodeR = Code<4>;

// The largest bit pattern of four numbers without their signs: a NaN's is above all others'.
__device__ __forceinline__ unsigned largest4(const float (&x)[4]) {
  unsigned top = 0u;
#pragma unroll
  for (int k = 0; k < 4; ++k) top = max(top, __float_as_uint(x[k]) & 0x7FFFFFFFu);
  return top;
}

__device__ __forceinline__ uint4 philox(uint4 c, const RoundKeys& keys) {
#pragma unroll
  for (int round = 0; round < 10; ++round) {
    const unsigned long long a = (unsigned long long)0xD2511F53u * c.x, b = (unsigned long long)0xCD9E8D57u * c.z;
    c = make_uint4((unsigned)(b >> 32) ^ c.y ^ keys.k[2 * round], (unsigned)b, (unsigned)(a >> 32) ^ c.w ^ keys.k[2 * round + 1],
                   (unsigned)a);
  }
  return c;
}

// One element's moments and its root.
__device__ __forceinline__ void moments(const AdamParams& p, float g, float& m, float& v, float& root) {
  m = __fadd_rn(__fmul_rn(p.beta1, m), __fmul_rn(p.c1, g));
  v = __fadd_rn(__fmul_rn(p.beta2, v), __fmul_rn(p.c2, __fmul_rn(g, g)));
  root = __fsqrt_rn(v);
}

__device__ __forceinline__ StepScalars scalars_of(const AdamParams& p) { return p.counted != nullptr ? *p.counted : p.now; }

// Whether the step is taken at all, and the factor of its gradients.
__device__ __forceinline__ bool gradient_factor(const AdamParams& p, float& c) {
  c = 1.0f;
  if (p.grad_scale != nullptr) {
    c = *p.grad_scale;
    if (!finite(c)) {
      if (threadIdx.x == 0) atomicOr(p.status, QADAM_ST_NONFINITE);
      return false;
    }
  }
  return true;
}

template <int CAP>
__global__ void __launch_bounds__(kAdamThreads) adamw_kernel(const __grid_constant__ AdamParams p,
                                                             const __grid_constant__ Pointers<CAP> grads) {
  wait_for_previous_launch();
  const AdamTile T = p.tiles[p.first + blockIdx.x];
  const void* g = grads.at[T.seg - p.tensor_base];
  float c;
  if (!gradient_factor(p, c) || g == nullptr) return;
  const int lane = threadIdx.x % 32;
  const int i0 = threadIdx.x / 32 * kPair;                   // of the warp's two rows, inside the tile
  const int rows = i0 >= T.left ? 0 : i0 + 128 >= T.left ? 1 : 2;
  if (rows == 0) return;
  const bool gfits = aligned4(g, T.gtype), wfits = aligned4(T.w, T.wtype);

  Raw4 rg[2], rx[2];
  float4 rm[2], rv[2];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    if (r >= rows) break;
    const int i = i0 + 128 * r + 4 * lane;
    rg[r] = load_raw4(g, T.gtype, T.begin + i, T.begin + T.left, gfits && i + 4 <= T.left);
    if (p.master != nullptr) rx[r] = load_raw4(p.master + T.at, QADAM_F32, i, T.left, true);
    else rx[r] = load_raw4(T.w, T.wtype, T.begin + i, T.begin + T.left, wfits && i + 4 <= T.left);
    rm[r] = *reinterpret_cast<const float4*>(static_cast<const float*>(p.m) + T.at + i);
    rv[r] = *reinterpret_cast<const float4*>(static_cast<const float*>(p.v) + T.at + i);
  }
  const StepScalars now = scalars_of(p);
  const float keep = (float)(1.0 - now.lr * (double)T.decay);
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    if (r >= rows) break;
    const int i = i0 + 128 * r + 4 * lane;
    float gx[4], x[4], m[4] = {rm[r].x, rm[r].y, rm[r].z, rm[r].w}, v[4] = {rv[r].x, rv[r].y, rv[r].z, rv[r].w};
    to_floats(rg[r], T.gtype, gx);
    to_floats(rx[r], p.master != nullptr ? (int)QADAM_F32 : T.wtype, x);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float root;
      moments(p, __fmul_rn(gx[k], c), m[k], v[k], root);
      const float d = __fadd_rn(__fmul_rn(root, now.b), p.eps);
      x[k] = __fsub_rn(__fmul_rn(x[k], keep), __fmul_rn(now.a, __fdiv_rn(m[k], d)));
    }
    if (p.master != nullptr) *reinterpret_cast<float4*>(p.master + T.at + i) = make_float4(x[0], x[1], x[2], x[3]);
    store_raw4(T.w, T.wtype, T.begin + i, T.begin + T.left, wfits && i + 4 <= T.left, from_floats(x, T.wtype));
    *reinterpret_cast<float4*>(static_cast<float*>(p.m) + T.at + i) = make_float4(m[0], m[1], m[2], m[3]);
    *reinterpret_cast<float4*>(static_cast<float*>(p.v) + T.at + i) = make_float4(v[0], v[1], v[2], v[3]);
  }
}

// ---------------------------------------------------------------- 8-bit moments
//
// 16 bytes an element with binary32 master weights or weights, 10 with 16-bit weights, and 79 instructions: codes
// in and out, a root, a reciprocal, ten Philox rounds per 8 elements.  That is more than the time of the bytes leaves
// for: bound by instruction issue, so types are the kernel's and not the row's, products go two at a time, and
// what a row or a pair of rows needs once is worked out by different lanes of one instruction.

// The BERT-shaped set with master weights (109.5 x 10^6 elements, floor 269 us): 4 warps to a CTA, 4 pairs of rows to a
// warp one after the other, 10 CTAs to an SM (48 registers, some 50 bytes of them spilt) 336 us, 9 (56 registers) 338; 9 with 2
// pairs 355, 10 with 8 pairs 330: pairs share what is worked out once per warp.  A warp has fewer pairs where there
// would be less than about one wave of warps.
constexpr int kEightCtas = 10;
constexpr int kEightPairs = 8;
constexpr int64_t kEightWave = 5000;

// What m is multiplied by in place of a division, the one operation of the step that is not rounded as stated: less than 3
// units in the last place of the quotient (one of the reciprocal's, at most two of the quotient's, and half a unit for the
// product and for the rounded quotient).  It enters a step of about lr and neither moment.  Divisions take 44.2 us in place of 40.9 on
// 11.7 x 10^6 binary32 elements, 361 in place of 345 on the BERT-shaped set with master weights.
__device__ __forceinline__ float reciprocal(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// Two products at a time; what they feed is added one by one, so that every operation is rounded.
__device__ __forceinline__ void mul4(float (&out)[4], const float (&a)[4], const float (&b)[4]) {
#pragma unroll
  for (int k = 0; k < 4; k += 2) {
    const float2 r = mul2_rn(make_float2(a[k], a[k + 1]), make_float2(b[k], b[k + 1]));
    out[k] = r.x;
    out[k + 1] = r.y;
  }
}
__device__ __forceinline__ void mul4(float (&out)[4], const float (&a)[4], float b) {
  const float bb[4] = {b, b, b, b};
  mul4(out, a, bb);
}

// A lane's four elements of a row: the step, but for the moments' codes.  g: scaled.
__device__ __forceinline__ void step_row(const AdamParams& p, float step_a, float step_b, float keep, const float (&g)[4], float (&x)[4],
                                         uint32_t cm, uint32_t cr, float sm, float sr, float (&m)[4], float (&root)[4]) {
  float v[4], a[4], b[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    m[k] = CodeM::value(cm, k);
    v[k] = CodeR::value(cr, k);
  }
  mul4(m, m, sm);
  mul4(v, v, sr);
#pragma unroll
  for (int k = 0; k < 4; ++k) m[k] = __uint_as_float(__float_as_uint(m[k]) | ((cm << (24 - 8 * k)) & 0x80000000u));
  mul4(v, v, v);
  mul4(a, m, p.beta1);
  mul4(b, g, p.c1);
#pragma unroll
  for (int k = 0; k < 4; ++k) m[k] = __fadd_rn(a[k], b[k]);
  mul4(a, v, p.beta2);
  mul4(b, g, g);
  mul4(b, b, p.c2);
#pragma unroll
  for (int k = 0; k < 4; ++k) root[k] = __fsqrt_rn(__fadd_rn(a[k], b[k]));
  mul4(a, root, step_b);
#pragma unroll
  for (int k = 0; k < 4; ++k) b[k] = reciprocal(__fadd_rn(a[k], p.eps));
  mul4(b, m, b);
  mul4(b, b, step_a);
  mul4(x, x, keep);
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = __fsub_rn(x[k], b[k]);
}

// A lane's codes of a row.  w0, w1: the elements' random bits, the low half of a word for k = 0, 2, the high half for 1, 3.
__device__ __forceinline__ uint2 codes_of(const float (&m)[4], const float (&root)[4], float im, float ir, unsigned w0, unsigned w1) {
  float a[4], b[4];
  mul4(a, m, im);
  mul4(b, root, ir);
  uint2 out = make_uint2(0u, 0u);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const unsigned word = k < 2 ? w0 : w1;
    const unsigned add_m = ((k % 2 == 0 ? word << 14 : word >> 2) & (63u << 14)) | (1u << 13);
    const unsigned add_r = ((k % 2 == 0 ? word << 3 : word >> 13) & (1023u << 9)) | (1u << 8);
    out.x |= CodeM::of(fabsf(a[k]), add_m, 0u, k) | (CodeM::shifted(__float_as_uint(m[k]), 8 * k - 24) & (128u << (8 * k)));
    // at least code 1 unless the root is 0: the root of the smallest binary32 number is far above 2^-126
    out.y |= CodeR::of(b[k], add_r, min(__float_as_uint(root[k]), 1u << CodeR::kDrop), k);
  }
  return out;
}

// Both rows' codes, and scales.  Lane l works out the reciprocal of scale l mod 4: m's and r's of the first row, of
// the second.  at: the lane's first element.
__device__ __forceinline__ void put_moments(const AdamParams& p, long long t, long long at, int rows, const float (&m)[2][4],
                                            const float (&root)[2][4]) {
  const int lane = threadIdx.x % 32;
  const unsigned long long quad = (unsigned long long)at / 4;
  const uint4 coins = philox(make_uint4((unsigned)quad, (unsigned)(quad >> 32), (unsigned)t, (unsigned)(t >> 32)), p.keys);
  const unsigned m0 = __reduce_max_sync(0xFFFFFFFFu, largest4(m[0])), r0 = __reduce_max_sync(0xFFFFFFFFu, largest4(root[0]));
  const unsigned m1 = __reduce_max_sync(0xFFFFFFFFu, largest4(m[1])), r1 = __reduce_max_sync(0xFFFFFFFFu, largest4(root[1]));
  const float mine = __uint_as_float(max((lane & 2) == 0 ? ((lane & 1) == 0 ? m0 : r0) : ((lane & 1) == 0 ? m1 : r1), kLeastScale));
  const float inverse = __fdiv_rn(1.0f, mine);
  const unsigned odd = __ballot_sync(0xFFFFFFFFu, !finite(mine));
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    if (r >= rows) break;
    uint2 c = codes_of(m[r], root[r], __shfl_sync(0xFFFFFFFFu, inverse, 2 * r), __shfl_sync(0xFFFFFFFFu, inverse, 2 * r + 1),
                       r == 0 ? coins.x : coins.z, r == 0 ? coins.y : coins.w);
    if (odd != 0u) {                                           // a row that is not finite: code 0 times its scale is a NaN
      if (((odd >> (2 * r)) & 1u) != 0u) c.x = 0u;
      if (((odd >> (2 * r + 1)) & 1u) != 0u) c.y = 0u;
    }
    *reinterpret_cast<uint32_t*>(static_cast<unsigned char*>(p.m) + at + 128 * r) = c.x;
    *reinterpret_cast<uint32_t*>(static_cast<unsigned char*>(p.v) + at + 128 * r) = c.y;
  }
  if (lane < 2 * rows) ((lane & 1) == 0 ? p.m_scale : p.r_scale)[at / 128 + lane / 2] = mine;
  if (odd != 0u && lane == 0) atomicOr(p.status, QADAM_ST_NONFINITE);
}

// Two rows at the end of their tensor, or of a tensor that is not aligned.
__device__ __noinline__ void step_pair_apart(const AdamParams& p, const void* g, int t, int i0, float c) {
  const int lane = threadIdx.x % 32;
  const StepScalars now = scalars_of(p);
  const AdamTile T = p.tiles[t];
  const float keep = (float)(1.0 - now.lr * (double)T.decay);
  const bool gfits = aligned4(g, T.gtype), wfits = aligned4(T.w, T.wtype);
  const int rows = i0 + 128 >= T.left ? 1 : 2;
  float m[2][4] = {}, root[2][4] = {};
#pragma unroll 1
  for (int r = 0; r < rows; ++r) {
    const int i = i0 + 128 * r + 4 * lane;
    const long long at = T.at + i;
    float gx[4], x[4];
    to_floats(load_raw4(g, T.gtype, T.begin + i, T.begin + T.left, gfits && i + 4 <= T.left), T.gtype, gx);
    if (p.master != nullptr) to_floats(load_raw4(p.master + T.at, QADAM_F32, i, T.left, true), QADAM_F32, x);
    else to_floats(load_raw4(T.w, T.wtype, T.begin + i, T.begin + T.left, wfits && i + 4 <= T.left), T.wtype, x);
    mul4(gx, gx, c);
    step_row(p, now.a, now.b, keep, gx, x, *reinterpret_cast<const uint32_t*>(static_cast<const unsigned char*>(p.m) + at),
             *reinterpret_cast<const uint32_t*>(static_cast<const unsigned char*>(p.v) + at), p.m_scale[at / 128], p.r_scale[at / 128], m[r], root[r]);
    if (p.master != nullptr) *reinterpret_cast<float4*>(p.master + at) = make_float4(x[0], x[1], x[2], x[3]);
    store_raw4(T.w, T.wtype, T.begin + i, T.begin + T.left, wfits && i + 4 <= T.left, from_floats(x, T.wtype));
  }
  put_moments(p, now.t, T.at + i0 + 4 * lane, rows, m, root);
}

template <bool HALF>
__device__ __forceinline__ Raw4 load_whole4(const char* p) {
  if constexpr (HALF) {
    const uint2 q = *reinterpret_cast<const uint2*>(p);
    return {{q.x, q.y, 0u, 0u}};
  } else {
    const uint4 q = *reinterpret_cast<const uint4*>(p);
    return {{q.x, q.y, q.z, q.w}};
  }
}

template <bool W16, bool G16, bool MASTER, int CAP>
__global__ void __launch_bounds__(kAdamThreads, kEightCtas) adamw8_kernel(const __grid_constant__ AdamParams p,
                                                                         const __grid_constant__ Pointers<CAP> grads) {
  wait_for_previous_launch();
  constexpr bool X16 = W16 && !MASTER;                         // what the step reads
  constexpr int kGBytes = G16 ? 2 : 4, kWBytes = W16 ? 2 : 4;
  const int t = p.first + blockIdx.x;
  const AdamTile& T = p.tiles[t];
  const char* const g = static_cast<const char*>(grads.at[T.seg - p.tensor_base]);
  float c;
  if (!gradient_factor(p, c) || g == nullptr) return;
  const int lane = threadIdx.x % 32;
  const int left = T.left, gtype = T.gtype, wtype = T.wtype;
  const bool fits = ((reinterpret_cast<uintptr_t>(g) & (4 * kGBytes - 1)) | (reinterpret_cast<uintptr_t>(T.w) & (4 * kWBytes - 1))) == 0;
  const int mine = kPair * p.pairs, first = threadIdx.x / 32 * mine;       // the warp's elements in the tile
  const char* from = g + (T.begin + first + 4 * lane) * kGBytes;
  char* w = static_cast<char*>(T.w) + (T.begin + first + 4 * lane) * kWBytes;
  long long at = T.at + first + 4 * lane;
  const float a = scalars_of(p).a, b = scalars_of(p).b;
  const float keep = (float)(1.0 - scalars_of(p).lr * (double)T.decay);
#pragma unroll 1
  for (int i0 = first; i0 < first + mine && i0 < left; i0 += kPair) {
    if (!fits || i0 + kPair > left) {
      step_pair_apart(p, g, t, i0, c);
    } else {
      Raw4 rg[2], rx[2];
      uint32_t cm[2], cr[2];
      float sm[2], sr[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        rg[r] = load_whole4<G16>(from + 128 * kGBytes * r);
        rx[r] = load_whole4<X16>(MASTER ? reinterpret_cast<const char*>(p.master + at + 128 * r) : w + 128 * kWBytes * r);
        cm[r] = *reinterpret_cast<const uint32_t*>(static_cast<const unsigned char*>(p.m) + at + 128 * r);
        cr[r] = *reinterpret_cast<const uint32_t*>(static_cast<const unsigned char*>(p.v) + at + 128 * r);
        sm[r] = p.m_scale[at / 128 + r];
        sr[r] = p.r_scale[at / 128 + r];
      }
      float m[2][4], root[2][4];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float gx[4], x[4];
        to_floats(rg[r], G16 ? gtype : (int)QADAM_F32, gx);
        to_floats(rx[r], X16 ? wtype : (int)QADAM_F32, x);
        mul4(gx, gx, c);
        step_row(p, a, b, keep, gx, x, cm[r], cr[r], sm[r], sr[r], m[r], root[r]);
        if constexpr (MASTER) *reinterpret_cast<float4*>(p.master + at + 128 * r) = make_float4(x[0], x[1], x[2], x[3]);
        const Raw4 rw = from_floats(x, W16 ? wtype : (int)QADAM_F32);
        if constexpr (W16) *reinterpret_cast<uint2*>(w + 256 * r) = make_uint2(rw.w[0], rw.w[1]);
        else *reinterpret_cast<uint4*>(w + 512 * r) = make_uint4(rw.w[0], rw.w[1], rw.w[2], rw.w[3]);
      }
      put_moments(p, scalars_of(p).t, at, 2, m, root);
    }
    from += kPair * kGBytes;
    w += kPair * kWBytes;
    at += kPair;
  }
}

// The scalars of the next step, from the device's own count and step size.
__global__ void adamw_count_kernel(StepScalars* now, long long* count, const float* lr, float lr_default, float beta1,
                                   float beta2, const float* grad_scale) {
  wait_for_previous_launch();
  const long long t = *count + 1;
  if (grad_scale == nullptr || finite(*grad_scale)) *count = t;
  *now = step_scalars(lr != nullptr ? (double)*lr : (double)lr_default, beta1, beta2, t);
}

// 8-bit moments as the values they stand for, four elements to a thread.  Bound by its writes, 8 bytes of 10: 200 us for
// 109.5 x 10^6 elements, 5.5 TB/s, whether a thread has loads for 4, 8, 16 or 32 elements under way (199 to 214 us).
constexpr int kReadThreads = 256;
constexpr int kReadCtasPerSm = 16;

__global__ void __launch_bounds__(kReadThreads) adamw_moments_kernel(const uint32_t* m, const uint32_t* r, const float* m_scale,
                                                                     const float* r_scale, long long quads, float4* m32, float4* v32) {
  wait_for_previous_launch();
  for (long long q = (long long)blockIdx.x * kReadThreads + threadIdx.x; q < quads; q += (long long)gridDim.x * kReadThreads) {
    float x[4];
    if (m32 != nullptr) {
      const uint32_t a = m[q];
      const float s = m_scale[q / 32];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        x[k] = __uint_as_float(__float_as_uint(__fmul_rn(CodeM::value(a, k), s)) | ((a << (24 - 8 * k)) & 0x80000000u));
      m32[q] = make_float4(x[0], x[1], x[2], x[3]);
    }
    if (v32 != nullptr) {
      const uint32_t a = r[q];
      const float s = r_scale[q / 32];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float z = __fmul_rn(CodeR::value(a, k), s);
        x[k] = __fmul_rn(z, z);
      }
      v32[q] = make_float4(x[0], x[1], x[2], x[3]);
    }
  }
}

struct AdamGeometry {
  struct Run {                 // tiles of one launch
    int first, num, tensor_base, tensors, kind;
  };
  std::vector<AdamTile> tiles;
  std::vector<Run> runs;
  std::vector<int> wtype, gtype;                             // [S]
  std::vector<int64_t> off, len;
  int64_t D = 0;
  int pairs = 1;
  size_t off_now = 0, workspace_bytes = 0;
};

int adam_geometry(const qadam_adamw_config* c, AdamGeometry* g) {
  if (!c) return QADAM_ERR_NULL;
  if (c->num_tensors < 1 || c->num_tensors > (1 << 20) || c->reserved != 0) return QADAM_ERR_SIZE;
  if (!c->len) return QADAM_ERR_NULL;
  if (c->state_bits != 32 && c->state_bits != 8) return QADAM_ERR_TYPE;
  if (c->master != 0 && c->master != 1) return QADAM_ERR_SIZE;
  if (!(c->beta1 >= 0.0f && c->beta1 < 1.0f) || !(c->beta2 >= 0.0f && c->beta2 < 1.0f) || !(c->eps >= kLeastEps) ||
      !std::isfinite(c->eps) || !(c->lr >= 0.0f) || !std::isfinite(c->lr))
    return QADAM_ERR_HYPER;
  int64_t tiles = 0, off = 0;
  for (int s = 0; s < c->num_tensors; ++s) {
    if ((c->weight_type && !known_type(c->weight_type[s])) || (c->grad_type && !known_type(c->grad_type[s]))) return QADAM_ERR_TYPE;
    if (c->decay && (!(c->decay[s] >= 0.0f) || !std::isfinite(c->decay[s]))) return QADAM_ERR_HYPER;
    if (c->len[s] < 0 || c->len[s] > (int64_t)1 << 40) return QADAM_ERR_SIZE;
    tiles += (c->len[s] + kAdamTile - 1) / kAdamTile;
    if (tiles > (int64_t)1 << 30) return QADAM_ERR_SIZE;
  }
  const size_t S = (size_t)c->num_tensors;
  g->tiles.reserve((size_t)tiles);
  g->wtype.resize(S); g->gtype.resize(S); g->off.resize(S);
  g->len.assign(c->len, c->len + S);
  for (size_t s = 0; s < S; ++s) {
    g->wtype[s] = c->weight_type ? c->weight_type[s] : QADAM_F32;
    g->gtype[s] = c->grad_type ? c->grad_type[s] : QADAM_F32;
    g->off[s] = off;
    off += (c->len[s] + kAlign - 1) / kAlign * kAlign;
  }
  // a launch takes the tensors that it has pointers for; with 8-bit moments, those of one kind
  if (c->state_bits == 8)
    while (g->pairs < kEightPairs && off / (2 * g->pairs * kPair) >= kEightWave) g->pairs *= 2;
  const int64_t tile = (int64_t)kAdamTile * g->pairs;
  for (size_t base = 0; base < S; base += kManyPointers) {
    const size_t end = std::min(S, base + kManyPointers);
    for (int kind = 0; kind < (c->state_bits == 8 ? 4 : 1); ++kind) {
      const int first = (int)g->tiles.size();
      for (size_t s = base; s < end; ++s) {
        if (c->state_bits == 8 && kind != (g->wtype[s] == QADAM_F32 ? 0 : 2) + (g->gtype[s] == QADAM_F32 ? 0 : 1)) continue;
        for (int64_t o = 0; o < c->len[s]; o += tile)
          g->tiles.push_back(AdamTile{nullptr, (long long)o, (long long)(g->off[s] + o), (int)std::min<int64_t>(c->len[s] - o, 1 << 30),
                                      (int)s, c->decay ? c->decay[s] : 0.0f, (short)g->wtype[s], (short)g->gtype[s], {0, 0}});
      }
      const int num = (int)g->tiles.size() - first;
      if (num > 0) g->runs.push_back({first, num, (int)base, (int)(end - base), kind});
    }
  }
  g->D = off;
  size_t wo = round_up256(g->tiles.size() * sizeof(AdamTile));
  g->off_now = wo;
  wo += 256;
  g->workspace_bytes = wo;
  return QADAM_OK;
}

}  // namespace

struct qadam_adamw {
  qadam_adamw_config cfg;      // scalars only: the lists are the caller's
  qadam_adamw_buffers buf;
  AdamGeometry geo;
  std::vector<const void*> grads;
  bool bound = false;
  int device = 0, sm_count = 0;
  int64_t launches = 0;
};

namespace {

template <bool W16, bool G16, bool MASTER, int CAP>
bool launch_eight(const AdamParams& p, const Pointers<CAP>& grads, cudaStream_t st) {
  return launch(adamw8_kernel<W16, G16, MASTER, CAP>, p.num_tiles, kAdamThreads, 0, 0, st, p, grads);
}

template <int CAP>
bool launch_adam(qadam_adamw* c, const AdamParams& p, const AdamGeometry::Run& run, cudaStream_t st) {
  static_assert(sizeof(Pointers<CAP>) + sizeof(AdamParams) <= 32764, "kernel parameters");
  Pointers<CAP> grads;
  std::copy(c->grads.begin() + run.tensor_base, c->grads.begin() + run.tensor_base + run.tensors, grads.at);
  c->launches += 1;
  if (c->cfg.state_bits == 32) return launch(adamw_kernel<CAP>, p.num_tiles, kAdamThreads, 0, 0, st, p, grads);
  switch (run.kind + (p.master != nullptr ? 4 : 0)) {
    case 0: return launch_eight<false, false, false>(p, grads, st);
    case 1: return launch_eight<false, true, false>(p, grads, st);
    case 2: return launch_eight<true, false, false>(p, grads, st);
    case 3: return launch_eight<true, true, false>(p, grads, st);
    case 4: return launch_eight<false, false, true>(p, grads, st);
    case 5: return launch_eight<false, true, true>(p, grads, st);
    case 6: return launch_eight<true, false, true>(p, grads, st);
    default: return launch_eight<true, true, true>(p, grads, st);
  }
}

int enqueue_step(qadam_adamw* c, const StepScalars& now, const StepScalars* counted, const float* grad_scale, cudaStream_t st) {
  AdamParams p;
  unsigned char* ws = static_cast<unsigned char*>(c->buf.workspace);
  p.tiles = reinterpret_cast<const AdamTile*>(ws);
  p.beta1 = c->cfg.beta1; p.beta2 = c->cfg.beta2;
  p.c1 = 1.0f - c->cfg.beta1; p.c2 = 1.0f - c->cfg.beta2;
  p.eps = c->cfg.eps;
  p.now = now;
  p.counted = counted;
  p.pairs = c->geo.pairs;
  p.grad_scale = grad_scale;
  p.master = c->buf.master;
  p.m = c->buf.m; p.v = c->buf.v;
  p.m_scale = c->buf.m_scale; p.r_scale = c->buf.r_scale;
  for (unsigned i = 0; i < 10; ++i) {
    p.keys.k[2 * i] = (unsigned)c->cfg.seed + i * 0x9E3779B9u;
    p.keys.k[2 * i + 1] = (unsigned)(c->cfg.seed >> 32) + i * 0xBB67AE85u;
  }
  p.status = c->buf.status;
  for (const AdamGeometry::Run& run : c->geo.runs) {
    p.tensor_base = run.tensor_base;
    p.first = run.first;
    p.num_tiles = run.num;
    if (!(run.tensors <= kFewPointers ? launch_adam<kFewPointers>(c, p, run, st) : launch_adam<kManyPointers>(c, p, run, st)))
      return QADAM_ERR_CUDA;
  }
  return QADAM_OK;
}

}  // namespace

extern "C" {

int qadam_adamw_query_sizes(const qadam_adamw_config* cfg, int64_t* D, int64_t* off, size_t* workspace_bytes) try {
  AdamGeometry g;
  const int rc = adam_geometry(cfg, &g);
  if (rc != QADAM_OK) return rc;
  if (D) *D = g.D;
  if (off)
    std::copy(g.off.begin(), g.off.end(), off);
  if (workspace_bytes) *workspace_bytes = g.workspace_bytes;
  return QADAM_OK;
} catch (const std::bad_alloc&) {
  return QADAM_ERR_SIZE;
}

int qadam_adamw_create(const qadam_adamw_config* cfg, const qadam_adamw_buffers* b, qadam_adamw** out) try {
  if (!out) return QADAM_ERR_NULL;
  *out = nullptr;
  if (!cfg || !b) return QADAM_ERR_NULL;
  AdamGeometry g;
  const int rc = adam_geometry(cfg, &g);
  if (rc != QADAM_OK) return rc;
  const bool eight = cfg->state_bits == 8;
  if (!b->weights || !b->m || !b->v || !b->workspace || !b->status || !b->count || (cfg->master && !b->master) ||
      (eight && (!b->m_scale || !b->r_scale)))
    return QADAM_ERR_NULL;
  for (size_t s = 0; s < g.len.size(); ++s) {
    if (!b->weights[s] && g.len[s] > 0) return QADAM_ERR_NULL;
    if (!is_aligned(b->weights[s], type_bytes(g.wtype[s]))) return QADAM_ERR_ALIGN;
  }
  for (AdamTile& t : g.tiles) t.w = b->weights[t.seg];
  if (!is_aligned(b->m, 16) || !is_aligned(b->v, 16) || (cfg->master && !is_aligned(b->master, 16)) ||
      (eight && (!is_aligned(b->m_scale, 16) || !is_aligned(b->r_scale, 16))) || !is_aligned(b->count, 8) ||
      !is_aligned(b->status, 4) || !is_aligned(b->workspace, 256))
    return QADAM_ERR_ALIGN;
  if (b->workspace_bytes < g.workspace_bytes) return QADAM_ERR_WORKSPACE;
  int device = 0, sms = 0;
  if (!cuda_call(cudaGetDevice(&device)) ||
      !cuda_call(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device)))
    return QADAM_ERR_CUDA;
  unsigned char* ws = static_cast<unsigned char*>(b->workspace);
  if (!g.tiles.empty() &&
      !cuda_call(cudaMemcpy(ws, g.tiles.data(), g.tiles.size() * sizeof(AdamTile), cudaMemcpyHostToDevice)))
    return QADAM_ERR_CUDA;
  if (!cuda_call(cudaMemset(b->status, 0, sizeof(unsigned))) || !cuda_call(cudaStreamSynchronize(nullptr)))
    return QADAM_ERR_CUDA;
  qadam_adamw* c = new qadam_adamw;
  c->cfg = *cfg;
  c->cfg.len = nullptr; c->cfg.weight_type = nullptr; c->cfg.grad_type = nullptr; c->cfg.decay = nullptr;
  c->buf = *b;
  c->buf.weights = nullptr;
  if (!cfg->master) c->buf.master = nullptr;
  c->geo = std::move(g);
  c->device = device;
  c->sm_count = sms;
  *out = c;
  return QADAM_OK;
} catch (const std::bad_alloc&) {
  return QADAM_ERR_SIZE;
}

int qadam_adamw_bind(qadam_adamw* c, const void* const* grads) try {
  if (!c || !grads) return QADAM_ERR_NULL;
  for (size_t s = 0; s < c->geo.len.size(); ++s)
    if (!is_aligned(grads[s], type_bytes(c->geo.gtype[s]))) return QADAM_ERR_ALIGN;
  c->grads.assign(grads, grads + c->geo.len.size());
  c->bound = true;
  return QADAM_OK;
} catch (const std::bad_alloc&) {
  return QADAM_ERR_SIZE;
}

int qadam_adamw_step(qadam_adamw* c, int64_t step, float lr, const float* grad_scale, void* stream) {
  if (!c || !c->bound) return QADAM_ERR_NULL;
  if (step < 1) return QADAM_ERR_STEP;
  if (std::isnan(lr) || std::isinf(lr)) return QADAM_ERR_HYPER;
  if (!is_aligned(grad_scale, 4)) return QADAM_ERR_ALIGN;
  const OnDevice on(c->device);
  if (!on.ok()) return QADAM_ERR_CUDA;
  return enqueue_step(c, step_scalars(lr < 0.0f ? c->cfg.lr : lr, c->cfg.beta1, c->cfg.beta2, step), nullptr, grad_scale,
                      static_cast<cudaStream_t>(stream));
}

int qadam_adamw_step_counted(qadam_adamw* c, const float* lr, const float* grad_scale, void* stream) {
  if (!c || !c->bound) return QADAM_ERR_NULL;
  if (!is_aligned(grad_scale, 4) || !is_aligned(lr, 4)) return QADAM_ERR_ALIGN;
  const OnDevice on(c->device);
  if (!on.ok()) return QADAM_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  StepScalars* now = reinterpret_cast<StepScalars*>(static_cast<unsigned char*>(c->buf.workspace) + c->geo.off_now);
  if (!launch(adamw_count_kernel, 1, 1, 0, 0, st, now, reinterpret_cast<long long*>(c->buf.count), lr, c->cfg.lr, c->cfg.beta1,
              c->cfg.beta2, grad_scale))
    return QADAM_ERR_CUDA;
  c->launches += 1;
  return enqueue_step(c, StepScalars{}, now, grad_scale, st);
}

int qadam_adamw_moments(qadam_adamw* c, float* m32, float* v32, void* stream) {
  if (!c || (!m32 && !v32)) return QADAM_ERR_NULL;
  if (c->cfg.state_bits != 8) return QADAM_ERR_TYPE;
  if (!is_aligned(m32, 16) || !is_aligned(v32, 16)) return QADAM_ERR_ALIGN;
  const long long quads = c->geo.D / 4;
  if (quads == 0) return QADAM_OK;
  const OnDevice on(c->device);
  if (!on.ok()) return QADAM_ERR_CUDA;
  const long long grid = std::min<long long>((quads + kReadThreads - 1) / kReadThreads, (long long)c->sm_count * kReadCtasPerSm);
  if (!launch(adamw_moments_kernel, grid, kReadThreads, 0, 0, static_cast<cudaStream_t>(stream), static_cast<const uint32_t*>(c->buf.m),
              static_cast<const uint32_t*>(c->buf.v), static_cast<const float*>(c->buf.m_scale), static_cast<const float*>(c->buf.r_scale),
              quads, reinterpret_cast<float4*>(m32), reinterpret_cast<float4*>(v32)))
    return QADAM_ERR_CUDA;
  c->launches += 1;
  return QADAM_OK;
}

int qadam_adamw_poll_status(qadam_adamw* c, void* stream, uint32_t* host_status) {
  if (!c || !host_status) return QADAM_ERR_NULL;
  const OnDevice on(c->device);
  if (!on.ok()) return QADAM_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (!cuda_call(cudaMemcpyAsync(host_status, c->buf.status, sizeof(uint32_t), cudaMemcpyDeviceToHost, st)) ||
      !cuda_call(cudaStreamSynchronize(st)))
    return QADAM_ERR_CUDA;
  return QADAM_OK;
}

int64_t qadam_adamw_launch_count(const qadam_adamw* c) { return c ? c->launches : QADAM_ERR_NULL; }

int qadam_adamw_destroy(qadam_adamw* c) {
  if (!c) return QADAM_ERR_NULL;
  delete c;
  return QADAM_OK;
}

}  // extern "C"
