// Rows of eight elements at a time, and reductions over the threads that share a row: what the operators on token rows use.
#pragma once

#include "qadam_tensors.cuh"

namespace qadam {

// Eight consecutive elements as they lie in memory.
template <int TY>
struct Raw8 {
  uint32_t w[TY == QADAM_F32 ? 8 : 4];
};

template <int TY>
__device__ __forceinline__ Raw8<TY> load_raw8(const void* p) {          // 16-byte aligned
  Raw8<TY> r;
  const uint4 a = *static_cast<const uint4*>(p);
  r.w[0] = a.x; r.w[1] = a.y; r.w[2] = a.z; r.w[3] = a.w;
  if constexpr (TY == QADAM_F32) {
    const uint4 b = static_cast<const uint4*>(p)[1];
    r.w[4] = b.x; r.w[5] = b.y; r.w[6] = b.z; r.w[7] = b.w;
  }
  return r;
}

template <int TY>
__device__ __forceinline__ void store_raw8(void* p, const Raw8<TY>& r) {
  *static_cast<uint4*>(p) = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
  if constexpr (TY == QADAM_F32) static_cast<uint4*>(p)[1] = make_uint4(r.w[4], r.w[5], r.w[6], r.w[7]);
}

template <int TY>
__device__ __forceinline__ void raw8_to_floats(const Raw8<TY>& r, float (&x)[8]) {
  if constexpr (TY == QADAM_F32) {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = __uint_as_float(r.w[k]);
  } else if constexpr (TY == QADAM_BF16) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[2 * k] = __uint_as_float(r.w[k] << 16);
      x[2 * k + 1] = __uint_as_float(r.w[k] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[2 * k] = half_bits_to_float(r.w[k] & 0xFFFFu);
      x[2 * k + 1] = half_bits_to_float(r.w[k] >> 16);
    }
  }
}

template <int TY>
__device__ __forceinline__ Raw8<TY> floats_to_raw8(const float (&x)[8]) {
  Raw8<TY> r;
#pragma unroll
  for (int k = 0; k < 8; k += 2) {
    if constexpr (TY == QADAM_F32) {
      r.w[k] = __float_as_uint(x[k]);
      r.w[k + 1] = __float_as_uint(x[k + 1]);
    } else if constexpr (TY == QADAM_BF16) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[k], x[k + 1]);
      r.w[k / 2] = *reinterpret_cast<const uint32_t*>(&h);
    } else {
      const __half2 h = __floats2half2_rn(x[k], x[k + 1]);
      r.w[k / 2] = *reinterpret_cast<const uint32_t*>(&h);
    }
  }
  return r;
}

template <int TY>
__device__ __forceinline__ float load_one(const void* p, long long i) {
  if constexpr (TY == QADAM_F32) return static_cast<const float*>(p)[i];
  const uint32_t b = static_cast<const unsigned short*>(p)[i];
  return TY == QADAM_BF16 ? __uint_as_float(b << 16) : half_bits_to_float(b);
}

template <int TY>
__device__ __forceinline__ void store_one(void* p, long long i, float v) {
  if constexpr (TY == QADAM_F32) static_cast<float*>(p)[i] = v;
  else if constexpr (TY == QADAM_BF16) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
  else static_cast<__half*>(p)[i] = __float2half_rn(v);
}

// The value as the type holds it.
template <int TY>
__device__ __forceinline__ float rounded(float v) {
  if constexpr (TY == QADAM_F32) return v;
  else if constexpr (TY == QADAM_BF16) return __bfloat162float(__float2bfloat16_rn(v));
  else return __half2float(__float2half_rn(v));
}

__device__ __forceinline__ float load_one_of(const void* p, int type, long long i) {
  return type == QADAM_F32 ? load_one<QADAM_F32>(p, i) : type == QADAM_BF16 ? load_one<QADAM_BF16>(p, i) : load_one<QADAM_F16>(p, i);
}

__device__ __forceinline__ void store_one_of(void* p, int type, long long i, float v) {
  if (type == QADAM_F32) store_one<QADAM_F32>(p, i, v);
  else if (type == QADAM_BF16) store_one<QADAM_BF16>(p, i, v);
  else store_one<QADAM_F16>(p, i, v);
}

// Eight elements from i on; vec: they begin on 16 bytes.
__device__ __forceinline__ void load_eight_of(const void* p, int type, long long i, bool vec, float (&x)[8]) {
  if (!vec) {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = load_one_of(p, type, i + k);
  } else if (type == QADAM_F32) {
    raw8_to_floats<QADAM_F32>(load_raw8<QADAM_F32>(static_cast<const float*>(p) + i), x);
  } else if (type == QADAM_BF16) {
    raw8_to_floats<QADAM_BF16>(load_raw8<QADAM_BF16>(static_cast<const unsigned short*>(p) + i), x);
  } else {
    raw8_to_floats<QADAM_F16>(load_raw8<QADAM_F16>(static_cast<const unsigned short*>(p) + i), x);
  }
}

__device__ __forceinline__ float warp_add(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}

// Reductions over the threads of a row: a warp, or (CTA) a whole block of whole warps.  A block's reductions take turns with
// two buffers, so one barrier each is enough: a buffer is written again only behind the barrier of the reduction between.
struct RowShared {
  float f[2][32][2];
  uint32_t u[2][32];
};

template <bool CTA>
class RowGroup {
 public:
  __device__ explicit RowGroup(RowShared* s) : s_(s) {}

  __device__ __forceinline__ float add(float v) {
    v = warp_add(v);
    if constexpr (CTA) {
      if (threadIdx.x % 32 == 0) s_->f[turn_][threadIdx.x / 32][0] = v;
      __syncthreads();
      v = warp_add(lane_in_use() ? s_->f[turn_][threadIdx.x % 32][0] : 0.0f);
      turn_ ^= 1;
    }
    return v;
  }
  __device__ __forceinline__ void add2(float& a, float& b) {
    a = warp_add(a);
    b = warp_add(b);
    if constexpr (CTA) {
      if (threadIdx.x % 32 == 0) {
        s_->f[turn_][threadIdx.x / 32][0] = a;
        s_->f[turn_][threadIdx.x / 32][1] = b;
      }
      __syncthreads();
      a = warp_add(lane_in_use() ? s_->f[turn_][threadIdx.x % 32][0] : 0.0f);
      b = warp_add(lane_in_use() ? s_->f[turn_][threadIdx.x % 32][1] : 0.0f);
      turn_ ^= 1;
    }
  }
  __device__ __forceinline__ uint32_t max(uint32_t v) {
    v = __reduce_max_sync(0xFFFFFFFFu, v);
    if constexpr (CTA) {
      if (threadIdx.x % 32 == 0) s_->u[turn_][threadIdx.x / 32] = v;
      __syncthreads();
      v = __reduce_max_sync(0xFFFFFFFFu, lane_in_use() ? s_->u[turn_][threadIdx.x % 32] : 0u);
      turn_ ^= 1;
    }
    return v;
  }
  __device__ __forceinline__ int add(int v) {
    v = __reduce_add_sync(0xFFFFFFFFu, v);
    if constexpr (CTA) {
      if (threadIdx.x % 32 == 0) s_->u[turn_][threadIdx.x / 32] = (uint32_t)v;
      __syncthreads();
      v = __reduce_add_sync(0xFFFFFFFFu, lane_in_use() ? (int)s_->u[turn_][threadIdx.x % 32] : 0);
      turn_ ^= 1;
    }
    return v;
  }

 private:
  __device__ __forceinline__ bool lane_in_use() const { return threadIdx.x % 32 < blockDim.x / 32; }
  RowShared* s_;
  int turn_ = 0;
};

// Rows in 8 bits: a = max(largest |x|, 2^-100), q = rne(x fl(127 / a)), worth a / 127.  `largest`: the bits of the largest
// |x|, which a NaN exceeds.  A row with a value that is not finite is worth NaN.
struct ByteScale {
  float per, worth;
};
__device__ __forceinline__ ByteScale byte_scale(uint32_t largest) {
  if (largest >= 0x7F800000u) return {0.0f, __uint_as_float(0x7FC00000u)};
  const float a = fmaxf(__uint_as_float(largest), 7.888609052210118e-31f);
  return {__fdiv_rn(127.0f, a), __fdiv_rn(a, 127.0f)};
}
__device__ __forceinline__ int to_byte(float x, float per) { return __float2int_rn(__fmul_rn(x, per)); }      // (a NaN gives 0)
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t four_bytes(int a, int b, int c, int d) {
  return __byte_perm(__byte_perm((uint32_t)a, (uint32_t)b, 0x0040), __byte_perm((uint32_t)c, (uint32_t)d, 0x0040), 0x5410);
}

}  // namespace qadam
