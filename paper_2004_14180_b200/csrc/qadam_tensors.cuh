// Lists of tensors of mixed element types: what the operators that walk over a whole set of
// tensors in one launch (AdamW, gradient norm) and those at an embedding table share.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "qadam.h"
#include "qadam_device.cuh"
#include "qadam_host.h"

namespace qadam {

inline bool cuda_call(cudaError_t e) {
  if (e != cudaSuccess) {
    record_cuda_error((int)e);
    return false;
  }
  return true;
}

// The current device for the life of the object, put back at its end.
class OnDevice {
 public:
  explicit OnDevice(int device) {
    ok_ = cuda_call(cudaGetDevice(&before_));
    if (ok_ && before_ != device) {
      ok_ = cuda_call(cudaSetDevice(device));
      changed_ = ok_;
    }
  }
  ~OnDevice() {
    if (changed_) (void)cudaSetDevice(before_);
  }
  OnDevice(const OnDevice&) = delete;
  OnDevice& operator=(const OnDevice&) = delete;
  bool ok() const { return ok_; }

 private:
  int before_ = 0;
  bool ok_ = false, changed_ = false;
};

inline bool known_type(int t) { return t == QADAM_F32 || t == QADAM_BF16 || t == QADAM_F16; }
__host__ __device__ inline int type_bytes(int t) { return t == QADAM_F32 ? 4 : 2; }
inline bool is_aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
inline size_t round_up256(size_t v) { return (v + 255) / 256 * 256; }

// Launches `kernel` so that it may be brought up while what is before it in the stream ends (every kernel that is launched
// so begins with wait_for_previous_launch).  The kernels before it say nothing early, so what is gained is the launch
// alone: 2 us of 14 (norm of 11.7 x 10^6 elements), 11 us of 161 over the five launches of a long embedding gradient.
// Saying so early gained nothing more.  cluster > 0: CTAs of a cluster.
template <typename... P, typename... A>
inline bool launch(void (*kernel)(P...), long long grid, int block, size_t smem, int cluster, cudaStream_t st, const A&... args) {
  cudaLaunchConfig_t config = {};
  config.gridDim = dim3((unsigned)grid);
  config.blockDim = dim3((unsigned)block);
  config.dynamicSmemBytes = smem;
  config.stream = st;
  cudaLaunchAttribute attributes[2];
  attributes[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attributes[0].val.programmaticStreamSerializationAllowed = 1;
  config.attrs = attributes;
  config.numAttrs = 1;
  if (cluster > 0) {
    attributes[1].id = cudaLaunchAttributeClusterDimension;
    attributes[1].val.clusterDim.x = (unsigned)cluster;
    attributes[1].val.clusterDim.y = attributes[1].val.clusterDim.z = 1;
    config.numAttrs = 2;
  }
  return cuda_call(cudaLaunchKernelEx(&config, kernel, args...));
}

// The tensors that one launch reads through pointers that may change from call to call.  They
// travel as kernel parameters, so a call needs no copy to the device, two calls never share a table
// that one of them is still reading, and a captured launch keeps its own.  4 KB of parameters
// hold the small form; a list longer than the large one takes several launches.
template <int CAP>
struct Pointers {
  const void* at[CAP];
};
constexpr int kFewPointers = 448;
constexpr int kManyPointers = 3584;

// Four consecutive elements as they lie in memory: 16-bit types fill two words.
struct Raw4 {
  uint32_t w[4];
};

// Element index `i` (a multiple of 4) of a tensor whose elements from `len` on do not exist (they
// read as zero).  `whole`: all four are there and aligned for one access.
__device__ __forceinline__ Raw4 load_raw4(const void* p, int type, long long i, long long len, bool whole) {
  Raw4 r = {{0u, 0u, 0u, 0u}};
  if (type == QADAM_F32) {
    const uint32_t* q = static_cast<const uint32_t*>(p) + i;
    if (whole) {
      const uint4 v = *reinterpret_cast<const uint4*>(q);
      r = {{v.x, v.y, v.z, v.w}};
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (i + k < len) r.w[k] = q[k];
    }
  } else {
    const unsigned short* q = static_cast<const unsigned short*>(p) + i;
    if (whole) {
      const uint2 v = *reinterpret_cast<const uint2*>(q);
      r.w[0] = v.x;
      r.w[1] = v.y;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (i + k < len) r.w[k / 2] |= (uint32_t)q[k] << (16 * (k % 2));
    }
  }
  return r;
}

__device__ __forceinline__ float half_bits_to_float(uint32_t b) { return __half2float(__ushort_as_half((unsigned short)b)); }

__device__ __forceinline__ void to_floats(const Raw4& r, int type, float (&x)[4]) {
  if (type == QADAM_F32) {
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = __uint_as_float(r.w[k]);
  } else if (type == QADAM_BF16) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      x[2 * k] = __uint_as_float(r.w[k] << 16);
      x[2 * k + 1] = __uint_as_float(r.w[k] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      x[2 * k] = half_bits_to_float(r.w[k] & 0xFFFFu);
      x[2 * k + 1] = half_bits_to_float(r.w[k] >> 16);
    }
  }
}

// Rounded to nearest even; binary16 overflows to infinity, as a conversion does.
__device__ __forceinline__ Raw4 from_floats(const float (&x)[4], int type) {
  Raw4 r = {{0u, 0u, 0u, 0u}};
  if (type == QADAM_F32) {
#pragma unroll
    for (int k = 0; k < 4; ++k) r.w[k] = __float_as_uint(x[k]);
  } else if (type == QADAM_BF16) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * k], x[2 * k + 1]);
      r.w[k] = *reinterpret_cast<const uint32_t*>(&h);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const __half2 h = __floats2half2_rn(x[2 * k], x[2 * k + 1]);
      r.w[k] = *reinterpret_cast<const uint32_t*>(&h);
    }
  }
  return r;
}

__device__ __forceinline__ void store_raw4(void* p, int type, long long i, long long len, bool whole, const Raw4& r) {
  if (type == QADAM_F32) {
    uint32_t* q = static_cast<uint32_t*>(p) + i;
    if (whole) {
      *reinterpret_cast<uint4*>(q) = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (i + k < len) q[k] = r.w[k];
    }
  } else {
    unsigned short* q = static_cast<unsigned short*>(p) + i;
    if (whole) {
      *reinterpret_cast<uint2*>(q) = make_uint2(r.w[0], r.w[1]);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (i + k < len) q[k] = (unsigned short)(r.w[k / 2] >> (16 * (k % 2)));
    }
  }
}

// Whether accesses of four elements at multiples of 4 are aligned.
__device__ __forceinline__ bool aligned4(const void* p, int type) {
  return (reinterpret_cast<uintptr_t>(p) & (unsigned)(4 * type_bytes(type) - 1)) == 0;
}

}  // namespace qadam
