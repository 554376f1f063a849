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

__device__ __forceinline__ float warp_add(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}

// Sums over a row divided by its width, correctly rounded (but for quotients below 2^-126), without a division for each row: a quotient from the
// rounded reciprocal, and what it leaves over, which is exact (P. Markstein, Computation of elementary functions on the IBM RISC
// System/6000 processor, 1990).  The product with the reciprocal alone may be off by a unit in the last place: the mean of
// 1000 times 200 was 200.00002.  Divisions: 25.3 in place of 22.9 us for the norm of 65536 x 256 bf16.
struct RowWidth {
  float n, per;
  __host__ __device__ static RowWidth of(int width) { return {(float)width, 1.0f / (float)width}; }
  __device__ __forceinline__ float mean_of(float sum) const {
    const float q = sum * per;
    return fabsf(q) < __int_as_float(0x7F800000) ? fmaf(fmaf(-q, n, sum), per, q) : q;
  }
};

// Reductions over the threads that share a row: a warp, or (MANY) up to 32 warps of a CTA, that have a barrier of their own.  Reductions
// take turns with two buffers, so one barrier each is enough: a buffer is written again only behind the barrier of the reduction
// between.
struct GroupShared {
  float f[2][32][2];
};

template <bool MANY>
class RowGroup {
 public:
  // warps: of the group; number: of the group in its CTA, which is its barrier's too (from 1 on)
  __device__ RowGroup(GroupShared* s, int warps, int number) : s_(s), warps_(warps), barrier_(number + 1) {}

  __device__ __forceinline__ void sync() {
    if constexpr (MANY) asm volatile("bar.sync %0, %1;" ::"r"(barrier_), "r"(warps_ * 32) : "memory");
    else __syncwarp();
  }
  __device__ __forceinline__ float add(float v) {
    v = warp_add(v);
    if constexpr (MANY) {
      put(v, 0);
      sync();
      v = warp_add(got(0));
      turn_ ^= 1;
    }
    return v;
  }
  // The means of two sums at the price of one: the warp's lower half has a, its upper half b.
  __device__ __forceinline__ void mean2(float& a, float& b, const RowWidth& width) {
    const bool upper = threadIdx.x % 32 >= 16;
    float mine = upper ? b : a;
    mine += __shfl_xor_sync(0xFFFFFFFFu, upper ? a : b, 16);
    mine = half_add(mine);
    if constexpr (MANY) {
      const int lane = threadIdx.x % 16;
      if (lane == 0) s_->f[turn_][warp()][upper] = mine;
      sync();
      mine = lane < warps_ ? s_->f[turn_][lane][upper] : 0.0f;
      if (warps_ > 16) mine += lane + 16 < warps_ ? s_->f[turn_][lane + 16][upper] : 0.0f;
      mine = half_add(mine);
      turn_ ^= 1;
    }
    mine = width.mean_of(mine);
    const float other = __shfl_xor_sync(0xFFFFFFFFu, mine, 16);
    a = upper ? other : mine;
    b = upper ? mine : other;
  }
  __device__ __forceinline__ uint32_t max(uint32_t v) {
    v = __reduce_max_sync(0xFFFFFFFFu, v);
    if constexpr (MANY) {
      put(__uint_as_float(v), 0);
      sync();
      v = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(got(0)));
      turn_ ^= 1;
    }
    return v;
  }
  __device__ __forceinline__ int add(int v) {
    v = __reduce_add_sync(0xFFFFFFFFu, v);
    if constexpr (MANY) {
      put(__int_as_float(v), 0);
      sync();
      v = __reduce_add_sync(0xFFFFFFFFu, __float_as_int(got(0)));
      turn_ ^= 1;
    }
    return v;
  }

 private:
  __device__ static __forceinline__ float half_add(float v) {
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
  }
  __device__ __forceinline__ int warp() const { return (int)(threadIdx.x / 32) % warps_; }
  __device__ __forceinline__ void put(float v, int i) {
    if (threadIdx.x % 32 == 0) s_->f[turn_][warp()][i] = v;
  }
  __device__ __forceinline__ float got(int i) const { return (int)(threadIdx.x % 32) < warps_ ? s_->f[turn_][threadIdx.x % 32][i] : 0.0f; }
  GroupShared* s_;
  int warps_, barrier_, turn_ = 0;
};

// How a row's elements are dealt out, 8 NV to each of a group's threads, in pairs: a warp has 256 NV elements in a row, its lanes take
// turns with pieces of 16 bytes (VEC), or with elements.  So the distances between a thread's pieces are known when the kernel is
// compiled, and whether one is in the row is a comparison with a constant.  An element beyond the row reads as zero.
template <int TY, int NV, bool VEC>
struct RowPart {
  static constexpr int kBytes = TY == QADAM_F32 ? 4 : 2;
  static constexpr int kPiece = VEC ? 16 / kBytes : 1;     // consecutive elements
  static constexpr int kPieces = 8 * NV / kPiece;
  static constexpr int kPairs = 4 * NV;
  static constexpr int kStep = VEC ? 1 : 2;                // pieces that hold whole pairs
  static constexpr int kStepPairs = VEC ? kPiece / 2 : 1;
  using Row = float2[kPairs];

  int width, threads, t;
  int first, left;                                         // column of the first piece; from there to the row's end
  bool all;                                                // the warp's elements are all in the row
  __device__ __forceinline__ RowPart(int w, int n, int i) : width(w), threads(n), t(i) {
    first = i / 32 * (256 * NV) + i % 32 * kPiece;
    left = w - first;
    all = (i / 32 + 1) * (256 * NV) <= w;
  }
  __device__ __forceinline__ int column(int q) const { return first + q * 32 * kPiece; }             // a piece's first
  __device__ __forceinline__ bool has(int q) const { return q * 32 * kPiece < left; }
  __device__ __forceinline__ static constexpr int piece_of(int e) { return e / kPiece; }

  // from global or shared memory
  __device__ __forceinline__ void read(const void* row, Row& x) const {
    const char* from = static_cast<const char*>(row) + (long long)first * kBytes;
    if constexpr (VEC) {
      uint4 r[kPieces];
#pragma unroll
      for (int q = 0; q < kPieces; ++q) r[q] = has(q) ? *reinterpret_cast<const uint4*>(from + q * 512) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int q = 0; q < kPieces; ++q) unpack(r[q], &x[q * kPiece / 2]);
    } else {
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        x[i].x = has(2 * i) ? load_one<TY>(from, 64 * i) : 0.0f;
        x[i].y = has(2 * i + 1) ? load_one<TY>(from, 64 * i + 32) : 0.0f;
      }
    }
  }
  __device__ __forceinline__ void store(void* row, const Row& x) const {
    char* to = static_cast<char*>(row) + (long long)first * kBytes;
    if constexpr (VEC) {
#pragma unroll
      for (int q = 0; q < kPieces; ++q)
        if (has(q)) *reinterpret_cast<uint4*>(to + q * 512) = packed(&x[q * kPiece / 2]);
    } else {
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        if (has(2 * i)) store_one<TY>(to, 64 * i, x[i].x);
        if (has(2 * i + 1)) store_one<TY>(to, 64 * i + 32, x[i].y);
      }
    }
  }
  // Piece q of a row in shared memory (see slot_bytes; `row`: where it lies in global memory), and its counterpart in global memory.  (The
  // pair of elements of q and q + 1, where a piece is one element.)
  __device__ __forceinline__ void read_piece(const uint8_t* slot, const char* row, int q, float2* x) const {
    if constexpr (VEC) {
      unpack(*reinterpret_cast<const uint4*>(slot + first * kBytes + q * 512), x);
    } else {
      const uint8_t* from = slot + (reinterpret_cast<uintptr_t>(row) & 15u) + first * kBytes;
      x[0] = make_float2(load_one<TY>(from, 32 * q), load_one<TY>(from, 32 * q + 32));
    }
  }
  __device__ __forceinline__ void load_piece(const char* row, int q, float2* x) const {
    const char* from = row + (long long)first * kBytes;
    if constexpr (VEC) {
      unpack(has(q) ? *reinterpret_cast<const uint4*>(from + q * 512) : make_uint4(0u, 0u, 0u, 0u), x);
    } else {
      x[0] = make_float2(has(q) ? load_one<TY>(from, 32 * q) : 0.0f, has(q + 1) ? load_one<TY>(from, 32 * q + 32) : 0.0f);
    }
  }
  __device__ __forceinline__ void store_piece(char* row, int q, const float2* x) const {
    char* to = row + (long long)first * kBytes;
    if constexpr (VEC) {
      if (has(q)) *reinterpret_cast<uint4*>(to + q * 512) = packed(x);
    } else {
      if (has(q)) store_one<TY>(to, 32 * q, x[0].x);
      if (has(q + 1)) store_one<TY>(to, 32 * q + 32, x[0].y);
    }
  }
  // Clears what of piece q (and the next one, where a piece is one element) is beyond the row.
  __device__ __forceinline__ void clear_beyond(int q, float2* x) const {
#pragma unroll
    for (int k = 0; k < kStepPairs; ++k) {
      if (!has(q)) x[k].x = 0.0f;
      if (!has(VEC ? q : q + 1)) x[k].y = 0.0f;
    }
  }
  // x becomes what is stored.
  __device__ __forceinline__ void store_rounded(void* row, Row& x) const {
    store(row, x);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) x[i] = make_float2(rounded<TY>(x[i].x), rounded<TY>(x[i].y));
  }
  // Parameters of one type, beginning on 16 bytes if VEC, of piece q (and the next one, where a piece is one element).
  template <int PT>
  __device__ __forceinline__ void read_parameters(const void* p, int q, float2* x) const {
    const char* from = static_cast<const char*>(p) + (long long)column(q) * (PT == QADAM_F32 ? 4 : 2);
    if constexpr (VEC) {
      if (!has(q)) return;
#pragma unroll
      for (int k = 0; k < kPiece; k += 4) {
        if constexpr (PT == QADAM_F32) {
          const float4 v = *reinterpret_cast<const float4*>(from + 4 * k);
          x[k / 2] = make_float2(v.x, v.y);
          x[k / 2 + 1] = make_float2(v.z, v.w);
        } else {
          const uint2 v = *reinterpret_cast<const uint2*>(from + 2 * k);
          float y[4];
          to_floats(Raw4{{v.x, v.y, 0u, 0u}}, PT, y);
          x[k / 2] = make_float2(y[0], y[1]);
          x[k / 2 + 1] = make_float2(y[2], y[3]);
        }
      }
    } else {
      if (has(q)) x[0].x = load_one<PT>(from, 0);
      if (has(q + 1)) x[0].y = load_one<PT>(from, 32);
    }
  }
  // Parameters of any type, anywhere.
  __device__ __forceinline__ void read_any(const void* p, int type, int q, float2* x) const {
#pragma unroll
    for (int k = 0; k < kStep * kPiece; ++k) {
      const int at = VEC ? column(q) + k : column(q + k);
      if (has(VEC ? q : q + k)) (k % 2 ? x[k / 2].y : x[k / 2].x) = load_one_of(p, type, at);
    }
  }

  // ---- a row in shared memory: its bytes, as far from 16 as in memory, then zeros for all the group's threads (who clear the place
  // once; a copy clears what a row that lay further behind may have left)
  __host__ __device__ static constexpr int slot_bytes(int threads) { return threads * 8 * NV * kBytes + (VEC ? 0 : 32); }

  // Copies a row behind the threads' backs, in pieces of 16 bytes; before the first whole one words of 4, of which a copy reads as many bytes as
  // are in the row, and zeros up to where a row that lay here before may have ended.  (By loads and stores of the row's ends, which a group's
  // first warp waited for: 191 us in place of 146 for the gradient of 30011 x 2049 fp32.)  VEC: a thread copies what it will read.
  // `base`: nothing is read before it; of a word that begins before its row half is another row's, or what lies between.
  __device__ __forceinline__ void fetch(uint8_t* slot, const char* row, const char* base) const {
    const unsigned at = (unsigned)__cvta_generic_to_shared(slot);
    if constexpr (VEC) {
      const char* from = row + (long long)first * kBytes;
      const unsigned to = at + (unsigned)(first * kBytes);
#pragma unroll
      for (int q = 0; q < kPieces; ++q)
        if (has(q)) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + q * 512u), "l"(from + q * 512) : "memory");
    } else {
      const int bytes = width * kBytes, phase = (int)(reinterpret_cast<uintptr_t>(row) & 15u);
      const int start = phase ? 16 : 0, pieces = (((bytes + 30) & ~15) - start) >> 4;
      const unsigned to = at + (unsigned)(start + t * 16);
      const char* from = row + (start - phase) + t * 16;
      const int here = bytes - (start - phase) - t * 16;     // bytes of the row from there on
      constexpr int kEach = (8 * NV * kBytes + 15) / 16;
#pragma unroll
      for (int q = 0; q <= kEach; ++q)
        if (q * threads + t < pieces)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + (unsigned)(q * threads * 16)), "l"(from + q * threads * 16),
                       "r"(max(0, min(16, here - q * threads * 16)))
                       : "memory");
      if (t < 4 && phase / 4 + t < 4 && phase) {
        const int in = (phase & ~3) + 4 * t, whole = max(0, min(4, phase + bytes - in));
        const char* word = row + (in - phase);
        if (word >= base) {
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(at + (unsigned)in), "l"(word), "r"(whole) : "memory");
        } else {                                           // 16 bits, the first of all rows
          *reinterpret_cast<unsigned short*>(slot + phase) = *reinterpret_cast<const unsigned short*>(row);
        }
      }
    }
  }
  __device__ __forceinline__ void read_slot(const uint8_t* slot, const char* row, Row& x) const {
#pragma unroll
    for (int q = 0; q < kPieces; q += kStep) read_piece(slot, row, q, &x[q / kStep * kStepPairs]);
  }
  // Binary32 parameters in shared memory, one for each element that the group's threads have.
  __device__ __forceinline__ void read_shared(const float* p, int q, float2* x) const {
    if constexpr (VEC) {
#pragma unroll
      for (int k = 0; k < kPiece; k += 4) {
        const float4 v = *reinterpret_cast<const float4*>(p + column(q) + k);
        x[k / 2] = make_float2(v.x, v.y);
        x[k / 2 + 1] = make_float2(v.z, v.w);
      }
    } else {
      x[0] = make_float2(p[column(q)], p[column(q + 1)]);
    }
  }

 private:
  __device__ static __forceinline__ void unpack(const uint4& r, float2* x) {
    if constexpr (TY == QADAM_F32) {
      x[0] = make_float2(__uint_as_float(r.x), __uint_as_float(r.y));
      x[1] = make_float2(__uint_as_float(r.z), __uint_as_float(r.w));
    } else {
      const Raw8<TY> h = {{r.x, r.y, r.z, r.w}};
      float y[8];
      raw8_to_floats<TY>(h, y);
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = make_float2(y[2 * k], y[2 * k + 1]);
    }
  }
  __device__ static __forceinline__ uint4 packed(const float2* x) {
    if constexpr (TY == QADAM_F32) {
      return make_uint4(__float_as_uint(x[0].x), __float_as_uint(x[0].y), __float_as_uint(x[1].x), __float_as_uint(x[1].y));
    } else {
      const float y[8] = {x[0].x, x[0].y, x[1].x, x[1].y, x[2].x, x[2].y, x[3].x, x[3].y};
      const Raw8<TY> h = floats_to_raw8<TY>(y);
      return make_uint4(h.w[0], h.w[1], h.w[2], h.w[3]);
    }
  }
};
__device__ __forceinline__ void fetched() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All but the youngest `left` fetches (0 .. 2) are there.
__device__ __forceinline__ void wait_fetched(int left) {
  if (left == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else if (left == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// Clears n bytes (a multiple of 16) of shared memory with all of a CTA's threads.
__device__ __forceinline__ void clear_shared(uint8_t* p, int n) {
  for (int i = threadIdx.x * 16; i < n; i += blockDim.x * 16) *reinterpret_cast<uint4*>(p + i) = make_uint4(0u, 0u, 0u, 0u);
}
// A row of parameters as binary32, zeros from its width on up to n; `without`: what stands for parameters that there are none of.
__device__ __forceinline__ void fill_parameters(float* to, const void* p, int type, float without, int width, int n) {
  for (int i = threadIdx.x; i < n; i += blockDim.x) to[i] = i >= width ? 0.0f : p ? load_one_of(p, type, i) : without;
}

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
// The largest magnitude of three, NaN if one is.
__device__ __forceinline__ float largest_of(float m, float a, float b) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(m), "f"(a), "f"(b));
  return r;
}
// Four quotients as bytes: 1.5 x 2^23 added to a product of at most 2^22 leaves it rounded, ties to even, in the last bits.
// (The products one by one: a packed product and a packed sum were compiled into one operation with one rounding.)
__device__ __forceinline__ uint32_t to_bytes(float2 a, float2 b, float per) {
  const float2 magic = make_float2(12582912.0f, 12582912.0f);
  a = add2_rn(make_float2(__fmul_rn(a.x, per), __fmul_rn(a.y, per)), magic);
  b = add2_rn(make_float2(__fmul_rn(b.x, per), __fmul_rn(b.y, per)), magic);
  return __byte_perm(__byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0040), __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x0040), 0x5410);
}
__device__ __forceinline__ int to_byte(float x, float per) { return __float2int_rn(__fmul_rn(x, per)); }      // (a NaN gives 0)
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

}  // namespace qadam
