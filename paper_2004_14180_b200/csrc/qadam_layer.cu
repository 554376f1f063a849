// Layer norm and its gradients, rows and columns in 8 bits, packed weights as rows of 8 bits:
// qadam_layer_norm*, qadam_quantize_*, qadam_held_rows.
//
//   xhat = (h - mean) rstd,  y = xhat w + b                         mean, rstd: of the row
//   dx = rstd (g - mean(g) - xhat mean(g xhat)) + ds,  g = dy w      dw = sum over rows of dy xhat,  db = sum over rows of dy
//   q = rne(x (127 / a)),  a = max(max |x|, 2^-100)
//
// All of it is bound by HBM in principle: a row is read once and written once, a few operations an element.  In practice these kernels are bound by
// instructions (10 to 25 an element and thread) as soon as a row costs more than its elements: what is done for a row (places, reductions over
// its threads, reciprocals) is why a thread has 16 to 32 elements, and a row no more threads than that takes.  Arithmetic is binary32, in
// packed pairs; 16-bit results are rounded once, at the end.
#include "qadam.h"

#include <algorithm>
#include <atomic>
#include <cmath>

#include "qadam_rows.cuh"

using namespace qadam;

namespace {

constexpr int kWarpRowThreads = 128;                       // rows of at most 1024 elements: a warp each, four to a CTA
constexpr int kWarpRowWidth = 1024;
constexpr int kGroupRowWidth = 16384;                      // a group of warps for a row, in registers; beyond, a CTA reads the row again
constexpr int kGroupMostThreads = 768;                     // of an SM, that go from row to row
constexpr int kWideThreads = 1024;
constexpr int kSms = 148;
constexpr int kRingBytes = 220 * 1024;                     // of an SM's shared memory, for rows under way

struct RowParams {
  const char* x;
  long long x_stride;                                      // elements, as all strides here
  const char* r;
  long long r_stride;
  const void* w;
  int w_type;
  const void* b;
  int b_type;
  int alike;                                               // the type of w and b (of w, if there is no b), or -1, see kAnyType
  char* sum;
  long long sum_stride;
  char* out;
  long long out_stride;
  float* mean;
  float* rstd;
  signed char* q;
  long long q_stride;
  float* scale;
  int* sums;
  long long rows;
  int width;
  RowWidth by;
  int normed;                                              // 0: the rows are quantized as they are (times w, if given)
  float eps;
};

// ---------------------------------------------------------------- rows in registers

// h w + b; PT: the type of both, w's alone where there is no b, or kAnyType: w and b of types of their own, anywhere, each there or not.
constexpr int kAnyType = -1, kShared = 3;                  // kShared: binary32 of both in shared memory
template <int PT, int TY, int NV, bool VEC>
__device__ __forceinline__ void scale_and_shift(const RowParams& p, const RowPart<TY, NV, VEC>& part, const float* shared, float2 (&h)[4 * NV]) {
  using Part = RowPart<TY, NV, VEC>;
#pragma unroll
  for (int q = 0; q < Part::kPieces; q += Part::kStep) {
    float2 w[Part::kStepPairs], b[Part::kStepPairs];
#pragma unroll
    for (int k = 0; k < Part::kStepPairs; ++k) w[k] = b[k] = make_float2(0.0f, 0.0f);                 // (beyond the row: zero)
    if constexpr (PT == kShared) {
      part.read_shared(shared, q, w);
      part.read_shared(shared + part.threads * 8 * NV, q, b);
    } else if constexpr (PT != kAnyType) {
      part.template read_parameters<PT>(p.w, q, w);
      if (p.b) part.template read_parameters<PT>(p.b, q, b);
    } else {
      if (p.w) part.read_any(p.w, p.w_type, q, w);
      if (p.b) part.read_any(p.b, p.b_type, q, b);
    }
#pragma unroll
    for (int k = 0; k < Part::kStepPairs; ++k) {
      float2& y = h[q / Part::kStep * Part::kStepPairs + k];
      if (PT != kAnyType || p.w) y = fma2_rn(y, w[k], b[k]);
      else y = add2_rn(y, b[k]);
    }
  }
}

// 1 / sqrt(v) to 3 halves of a step: CUDA's, which is off by up to four, and a step of Newton's method, which squares what it is off by and adds a
// rounding of its own.  (No number if the first is 0 or infinite, and so is what it is the root of.)  65536 x 256 bf16: 23.8 us, with a
// correctly rounded one 24.5.
__device__ __forceinline__ float reciprocal_root(float v) {
  const float y = rsqrtf(v), off = fmaf(-v * y, y, 1.0f);
  return off == off ? fmaf(0.5f * y, off, y) : y;
}

// What becomes of a row h, dealt out to a group's threads: normed, scaled, written, in 8 bits.
template <int TY, int NV, bool VEC, bool MANY>
__device__ __forceinline__ void finish_row(const RowParams& p, const RowPart<TY, NV, VEC>& part, RowGroup<MANY>& group, long long row,
                                           const float* shared, float2 (&h)[4 * NV]) {
  using Part = RowPart<TY, NV, VEC>;
  if (p.normed) {
    float2 s = h[0];
#pragma unroll
    for (int i = 1; i < Part::kPairs; ++i) s = add2_rn(s, h[i]);
    const float mean = p.by.mean_of(group.add(s.x + s.y));
    const float2 less = make_float2(-mean, -mean);
#pragma unroll
    for (int i = 0; i < Part::kPairs; ++i) h[i] = add2_rn(h[i], less);
    if (!part.all) {
#pragma unroll
      for (int i = 0; i < Part::kPairs; ++i) {
        if (!part.has(Part::piece_of(2 * i))) h[i].x = 0.0f;
        if (!part.has(Part::piece_of(2 * i + 1))) h[i].y = 0.0f;
      }
    }
    s = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < Part::kPairs; ++i) s = fma2_rn(h[i], h[i], s);
    const float rstd = reciprocal_root(p.by.mean_of(group.add(s.x + s.y)) + p.eps);
    if (part.t == 0) {
      if (p.mean) p.mean[row] = mean;
      if (p.rstd) p.rstd[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < Part::kPairs; ++i) h[i] = mul2_rn(h[i], make_float2(rstd, rstd));
  }
  if (p.w || p.b) {
    if (shared) {
      scale_and_shift<kShared>(p, part, shared, h);
    } else {
      switch (p.alike) {                                   // (told apart once, not for each element)
        case QADAM_F32: scale_and_shift<QADAM_F32>(p, part, nullptr, h); break;
        case QADAM_BF16: scale_and_shift<QADAM_BF16>(p, part, nullptr, h); break;
        case QADAM_F16: scale_and_shift<QADAM_F16>(p, part, nullptr, h); break;
        default: scale_and_shift<kAnyType>(p, part, nullptr, h);
      }
    }
  }
  if (p.out) part.store(p.out + row * p.out_stride * Part::kBytes, h);
  if (p.q) {
    float largest = 0.0f;
#pragma unroll
    for (int i = 0; i < Part::kPairs; ++i) largest = largest_of(largest, h[i].x, h[i].y);
    const ByteScale s = byte_scale(group.max(abs_bits(largest)));
    signed char* q = p.q + row * p.q_stride;
    const uint32_t finite = s.per > 0.0f ? 0xFFFFFFFFu : 0u;
    int sum = 0;
    signed char* to = q + part.first;
    uint32_t c[Part::kPairs / 2];
#pragma unroll
    for (int i = 0; i < Part::kPairs; i += 2) {
      c[i / 2] = to_bytes(h[i], h[i + 1], s.per) & finite;
      sum = __dp4a((int)c[i / 2], 0x01010101, sum);        // (beyond the row: zeros)
    }
    if constexpr (VEC) {
#pragma unroll
      for (int n = 0; n < Part::kPieces; ++n) {
        if (part.has(n)) {
          if constexpr (Part::kPiece == 8) *reinterpret_cast<uint2*>(to + n * 256) = make_uint2(c[2 * n], c[2 * n + 1]);
          else *reinterpret_cast<uint32_t*>(to + n * 128) = c[n];
        }
      }
    } else {
#pragma unroll
      for (int n = 0; n < Part::kPieces; ++n)
        if (part.has(n)) to[n * 32] = (signed char)(c[n / 4] >> (8 * (n % 4)));
    }
    if (p.sums) sum = group.add(sum);
    if (part.t == 0) {
      p.scale[row] = s.worth;
      if (p.sums) p.sums[row] = sum;
    }
  }
}

// One pass: a row is read once, held in registers for mean, sum of squares around it and largest value, and written once.
// There is a warp for each row: enough of them are on an SM to keep its share of the loads under way.  8192 x 768 bf16, the sum with a residual
// and its norm: 8.6 us (50 MB; 7.8 at the copy rate); 16 rows: 2.1 us in a row of such launches.
template <int TY, int NV, bool VEC>
__global__ void __launch_bounds__(kWarpRowThreads) warp_row_kernel(const __grid_constant__ RowParams p) {
  wait_for_previous_launch();
  let_next_launch_start();                                 // (a product behind it is then brought up beside it: one token's 9.5 -> 8.0 us)
  using Part = RowPart<TY, NV, VEC>;
  RowGroup<false> group(nullptr, 1, 0);
  const Part part(p.width, 32, threadIdx.x % 32);
  const long long row = (long long)blockIdx.x * (kWarpRowThreads / 32) + threadIdx.x / 32;
  if (row >= p.rows) return;
  typename Part::Row h;
  part.read(p.x + row * p.x_stride * Part::kBytes, h);
  if (p.r) {
    typename Part::Row r;
    part.read(p.r + row * p.r_stride * Part::kBytes, r);
#pragma unroll
    for (int i = 0; i < Part::kPairs; ++i) h[i] = add2_rn(h[i], r[i]);
    part.store_rounded(p.sum + row * p.sum_stride * Part::kBytes, h);
  }
  finish_row(p, part, group, row, nullptr, h);
}

// Wider rows, and many: a group of warps (a warp) goes from row to row, with the next ones under way in shared memory, where the parameters are
// too.  65536 x 768 bf16: norm 44 us (201 MB, 4.6 TB/s: instructions), norm into 8 bits 46, rows as they are into 8 bits 25 (151 MB,
// 6.0 TB/s); 16384 x 8192 bf16 into 8 bits 76 to 88 us (403 MB, 62 at the copy rate; 117 with a CTA for each row); norm of 30011 x 2049 fp32, which
// begin anywhere, 120 us (492 MB, 76).
constexpr int kGroupWarps = 8;                             // of a CTA, in groups, or one group of up to 16
template <int TY, int NV, bool VEC, bool MANY, int MOST>
__global__ void __launch_bounds__(MOST, MOST == 256 ? 3 : 1) group_row_kernel(const __grid_constant__ RowParams p, int warps, int stages, int with_parameters) {
  extern __shared__ __align__(16) uint8_t slots[];         // [groups][stages][1 or 2][a row]; with_parameters: then w, b
  __shared__ GroupShared shared[kGroupWarps];
  wait_for_previous_launch();
  let_next_launch_start();
  using Part = RowPart<TY, NV, VEC>;
  const int threads = MANY ? warps * 32 : 32, number = (int)threadIdx.x / threads;
  const int groups = blockDim.x / threads;
  const Part part(p.width, threads, (int)threadIdx.x % threads);
  RowGroup<MANY> group(&shared[number], warps, number);
  const int each = Part::slot_bytes(threads), both = p.r ? 2 * each : each;
  uint8_t* ring = slots + number * stages * both;
  float* parameters = with_parameters ? reinterpret_cast<float*>(slots + groups * stages * both) : nullptr;
  clear_shared(slots, groups * stages * both);
  if (parameters) {
    fill_parameters(parameters, p.w, p.w_type, 1.0f, p.width, threads * 8 * NV);
    fill_parameters(parameters + threads * 8 * NV, p.b, p.b_type, 0.0f, p.width, threads * 8 * NV);
  }
  __syncthreads();
  const long long first = (long long)blockIdx.x * groups + number, step = (long long)gridDim.x * groups;
  const auto fetch = [&](long long row, int stage) {
    if (row < p.rows) {
      part.fetch(ring + stage * both, p.x + row * p.x_stride * Part::kBytes, p.x);
      if (p.r) part.fetch(ring + stage * both + each, p.r + row * p.r_stride * Part::kBytes, p.r);
    }
    fetched();
  };
  for (int i = 0; i + 1 < stages; ++i) fetch(first + i * step, i);
  int stage = 0;
  for (long long row = first; row < p.rows; row += step) {
    wait_fetched(stages - 2);
    if constexpr (!VEC) group.sync();                      // (what others have copied; what the row before has left)
    fetch(row + (stages - 1) * step, stage == 0 ? stages - 1 : stage - 1);
    typename Part::Row h;
    part.read_slot(ring + stage * both, p.x + row * p.x_stride * Part::kBytes, h);
    if (p.r) {
      typename Part::Row r;
      part.read_slot(ring + stage * both + each, p.r + row * p.r_stride * Part::kBytes, r);
#pragma unroll
      for (int i = 0; i < Part::kPairs; ++i) h[i] = add2_rn(h[i], r[i]);
      part.store_rounded(p.sum + row * p.sum_stride * Part::kBytes, h);
    }
    finish_row(p, part, group, row, parameters, h);
    stage = stage + 1 == stages ? 0 : stage + 1;
  }
}

// Rows too wide for a CTA's registers: read again for each thing that is known only at the row's end.  2000 x 20001 fp32: 130 us (320 MB, 50 at the
// copy rate), 2000 x 32768 bf16 182 (262 MB, 41): an element to an access.
template <int TY>
__global__ void __launch_bounds__(kWideThreads) wide_row_kernel(const __grid_constant__ RowParams p) {
  __shared__ GroupShared shared;
  wait_for_previous_launch();
  constexpr int kBytes = TY == QADAM_F32 ? 4 : 2;
  RowGroup<true> group(&shared, kWideThreads / 32, 0);
  const long long row = blockIdx.x;
  const char* x = p.x + row * p.x_stride * kBytes;
  const char* r = p.r ? p.r + row * p.r_stride * kBytes : nullptr;
  const auto element = [&](int col) {
    const float v = load_one<TY>(x, col);
    return r ? rounded<TY>(v + load_one<TY>(r, col)) : v;
  };
  float mean = 0.0f, rstd = 1.0f;
  if (p.normed) {
    float s = 0.0f;
    for (int col = threadIdx.x; col < p.width; col += kWideThreads) s += element(col);
    mean = group.add(s) / (float)p.width;
    s = 0.0f;
    for (int col = threadIdx.x; col < p.width; col += kWideThreads) {
      const float d = element(col) - mean;
      s = fmaf(d, d, s);
    }
    rstd = 1.0f / sqrtf(group.add(s) / (float)p.width + p.eps);
    if (threadIdx.x == 0) {
      if (p.mean) p.mean[row] = mean;
      if (p.rstd) p.rstd[row] = rstd;
    }
  }
  const auto result = [&](int col, float h) {
    return fmaf((h - mean) * rstd, p.w ? load_one_of(p.w, p.w_type, col) : 1.0f, p.b ? load_one_of(p.b, p.b_type, col) : 0.0f);
  };
  uint32_t largest = 0u;
  for (int col = threadIdx.x; col < p.width; col += kWideThreads) {
    const float h = element(col), y = result(col, h);
    if (r) store_one<TY>(p.sum + row * p.sum_stride * kBytes, col, h);
    if (p.out) store_one<TY>(p.out + row * p.out_stride * kBytes, col, y);
    largest = max(largest, abs_bits(y));
  }
  if (p.q) {
    const ByteScale s = byte_scale(group.max(largest));
    int sum = 0;
    for (int col = threadIdx.x; col < p.width; col += kWideThreads) {
      const int c = to_byte(result(col, element(col)), s.per);
      sum += c;
      p.q[row * p.q_stride + col] = (signed char)c;
    }
    sum = group.add(sum);
    if (threadIdx.x == 0) {
      p.scale[row] = s.worth;
      if (p.sums) p.sums[row] = sum;
    }
  }
}

// CTAs of `threads` threads that an SM has at a time (of most_threads), and stages of `bytes`, with `besides` of their own, that each of
// them has then: 2 or 3, or none if two do not fit.
struct Residents {
  int per_sm, stages;
};
Residents residents(int threads, int most_threads, int bytes, int besides) {
  const int per_sm = std::max(1, std::min(most_threads / threads, kRingBytes / (2 * bytes + besides + 2048)));
  const int stages = std::min(3, (kRingBytes / per_sm - 2048 - besides) / bytes);
  return {per_sm, stages < 2 ? 0 : stages};
}

// The limit of dynamic shared memory belongs to the kernel and the device: it is raised once, to the same for every launch.
template <auto KERNEL>
bool allow_ring(size_t bytes) {
  if (bytes <= 40 * 1024) return true;
  static std::atomic<uint64_t> raised{0};
  int device = 0;
  if (!cuda_call(cudaGetDevice(&device))) return false;
  const uint64_t bit = (uint64_t)1 << (device % 64);
  if (raised.load() & bit) return true;
  if (!cuda_call(cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes))) return false;
  raised.fetch_or(bit);
  return true;
}

template <int TY, int NV, bool VEC, bool MANY>
bool launch_group_rows(const RowParams& p, cudaStream_t st) {
  const int warps = (p.width + 256 * NV - 1) / (256 * NV), groups = std::max(1, kGroupWarps / warps);
  const int threads = warps * groups * 32, bytes = RowPart<TY, NV, VEC>::slot_bytes(warps * 32) * (p.r ? 2 : 1) * groups;
  // w and b in shared memory, if they take no more than a quarter of it
  const int parameters = p.w || p.b ? 2 * warps * 32 * 8 * NV * (int)sizeof(float) : 0;
  const int kept = parameters * 4 <= kRingBytes / std::max(1, kGroupMostThreads / threads) ? parameters : 0;
  const Residents r = residents(threads, kGroupMostThreads, bytes, kept);
  if (r.stages == 0) return launch(wide_row_kernel<TY>, p.rows, kWideThreads, 0, 0, st, p);
  const size_t smem = (size_t)r.stages * bytes + kept;
  const long long grid = std::min<long long>((p.rows + groups - 1) / groups, (long long)kSms * r.per_sm);
  if (threads <= 256)
    return allow_ring<group_row_kernel<TY, NV, VEC, MANY, 256>>(smem) &&
           launch(group_row_kernel<TY, NV, VEC, MANY, 256>, grid, threads, smem, 0, st, p, warps, r.stages, kept ? 1 : 0);
  if constexpr (MANY)
    return allow_ring<group_row_kernel<TY, NV, VEC, true, 512>>(smem) &&
           launch(group_row_kernel<TY, NV, VEC, true, 512>, grid, threads, smem, 0, st, p, warps, r.stages, kept ? 1 : 0);
  return false;                                            // (one warp to a row: eight to a CTA)
}
template <int TY, int NV>
bool launch_group_rows(const RowParams& p, bool vec, cudaStream_t st) {
  return vec ? launch_group_rows<TY, NV, true, true>(p, st) : launch_group_rows<TY, NV, false, true>(p, st);
}

// Rows of a warp: each its own, until there are so many that an SM's warps would do several one after the other: then they go from row
// to row (65536 x 768 bf16: a warp for each 46 us).
constexpr long long kManyRows = 4 * kSms * (kGroupMostThreads / 32);
template <int TY, int NV>
bool launch_warp_rows(const RowParams& p, bool vec, cudaStream_t st) {
  if (p.rows >= kManyRows) return vec ? launch_group_rows<TY, NV, true, false>(p, st) : launch_group_rows<TY, NV, false, false>(p, st);
  const long long grid = (p.rows + kWarpRowThreads / 32 - 1) / (kWarpRowThreads / 32);
  return vec ? launch(warp_row_kernel<TY, NV, true>, grid, kWarpRowThreads, 0, 0, st, p) : launch(warp_row_kernel<TY, NV, false>, grid, kWarpRowThreads, 0, 0, st, p);
}

template <int TY>
bool enqueue_rows_of(const RowParams& p, bool vec, cudaStream_t st) {
  if (p.width <= 256) return launch_warp_rows<TY, 1>(p, vec, st);
  if (p.width <= 512) return launch_warp_rows<TY, 2>(p, vec, st);
  if (p.width <= 768) return launch_warp_rows<TY, 3>(p, vec, st);
  if (p.width <= kWarpRowWidth) return launch_warp_rows<TY, 4>(p, vec, st);
  if (p.width > kGroupRowWidth) return launch(wide_row_kernel<TY>, p.rows, kWideThreads, 0, 0, st, p);
  // 24 or 32 elements to a thread, whichever leaves fewer threads without
  const int three = (p.width + 767) / 768 * 768, four = (p.width + 1023) / 1024 * 1024;
  return three < four && three <= 16 * 768 ? launch_group_rows<TY, 3>(p, vec, st) : launch_group_rows<TY, 4>(p, vec, st);
}

int enqueue_rows(const RowParams& p, int type, bool vec, cudaStream_t st) {
  const bool ok = type == QADAM_F32 ? enqueue_rows_of<QADAM_F32>(p, vec, st)
                  : type == QADAM_BF16 ? enqueue_rows_of<QADAM_BF16>(p, vec, st) : enqueue_rows_of<QADAM_F16>(p, vec, st);
  return ok ? QADAM_OK : QADAM_ERR_CUDA;
}

// ---------------------------------------------------------------- gradients

constexpr int kGradWarps = 6;                              // of a CTA, in groups, two CTAs to an SM; or one group of up to 11 in a CTA of its own
constexpr int kGradMoreWarps = 8, kGradMostWarps = 12;          // (8: registers for two such CTAs, 16384 x 4096 fp32 and fp16 too)
constexpr int kGradGroupWidth = 8192;                      // beyond, rows are read again, and the columns' sums are a pass of their own

struct GradParams {
  const char* dy;
  long long dy_stride;
  const char* x;
  long long x_stride;
  const char* ds;
  long long ds_stride;
  int ds_ahead;                                            // ds is fetched ahead as the others are (there is room for it)
  char* dx;
  long long dx_stride;
  const float* mean;
  const float* rstd;
  const void* w;
  int w_type;
  float* partial;                                          // [gridDim.x][2][width], or NULL
  long long rows;
  int width;
};

// Warps of an SM that there are registers for.
__host__ __device__ constexpr int grad_warps_of_sm(int nv, bool many) { return many && nv == 2 ? 18 : 12; }

// A warp (rows of up to 768 elements), or a group of them, goes from row to row, with the next ones under way, and adds up its rows' part of the
// weight's and bias's gradients in registers; the CTA's sums go to the workspace.  65536 x 768 bf16 with ds: 70 us (403 MB, 62 at the copy
// rate); 8192 x 768: 9.1 us, and 6.0 more for the sums' end and the launch that joins them; 30012 x 2048 fp32: 119 us (114); 30011 x 2049: 144.
// (Clusters of four CTAs that join their sums first: fewer CTAs find room, 30 us in place of 17 for 8192 x 768.)
// Where an SM gets 12 warps, registers hold a row between its sums and its result (2 to 4 % less time); where it gets 18, the row is read from
// shared memory again.  (Eight elements to a thread, and more warps to a row: 375 instructions for 256 elements, most of them for the
// row, not for elements.)
template <int TY, int NV, bool VEC, bool MANY, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, grad_warps_of_sm(NV, MANY) / WARPS) row_grad_kernel(const __grid_constant__ GradParams p, int warps, int stages) {
  extern __shared__ __align__(16) uint8_t slots[];         // [groups][stages][2 or 3][a row], w; at the end the groups' sums [groups][2][width]
  __shared__ GroupShared shared[MANY ? kGradWarps : 1];
  wait_for_previous_launch();
  using Part = RowPart<TY, NV, VEC>;
  constexpr int kBytes = Part::kBytes;
  constexpr bool kHold = grad_warps_of_sm(NV, MANY) == 12;
  const int threads = MANY ? warps * 32 : 32, number = (int)threadIdx.x / threads;
  const int groups = blockDim.x / threads;
  const Part part(p.width, threads, (int)threadIdx.x % threads);
  RowGroup<MANY> group(&shared[MANY ? number : 0], warps, number);
  const int each = Part::slot_bytes(threads), all_of = p.ds_ahead ? 3 * each : 2 * each;
  uint8_t* ring = slots + number * stages * all_of;
  const float* w = reinterpret_cast<const float*>(slots + groups * stages * all_of);
  clear_shared(slots, groups * stages * all_of);
  fill_parameters(reinterpret_cast<float*>(slots + groups * stages * all_of), p.w, p.w_type, 1.0f, p.width, threads * 8 * NV);
  __syncthreads();
  const RowWidth width = RowWidth::of(p.width);
  const long long first = (long long)blockIdx.x * groups + number, step = (long long)gridDim.x * groups;
  // rows to come: where they lie
  const char *next_x = p.x + first * p.x_stride * kBytes, *next_dy = p.dy + first * p.dy_stride * kBytes, *next_ds = p.ds + first * p.ds_stride * kBytes;
  const long long x_step = step * p.x_stride * kBytes, dy_step = step * p.dy_stride * kBytes, ds_step = step * p.ds_stride * kBytes;
  const auto fetch = [&](long long row, int stage) {
    if (row < p.rows) {
      uint8_t* to = ring + stage * all_of;
      part.fetch(to, next_x, p.x);
      part.fetch(to + each, next_dy, p.dy);
      if (p.ds_ahead) part.fetch(to + 2 * each, next_ds, p.ds);
    }
    next_x += x_step;
    next_dy += dy_step;
    next_ds += ds_step;
    fetched();
  };
  for (int i = 0; i + 1 < stages; ++i) fetch(first + i * step, i);
  typename Part::Row dw, db;
#pragma unroll
  for (int i = 0; i < Part::kPairs; ++i) dw[i] = db[i] = make_float2(0.0f, 0.0f);
  int stage = 0;
  for (long long row = first; row < p.rows; row += step) {
    const float mean = p.mean[row], rstd = p.rstd[row];
    wait_fetched(stages - 2);
    if constexpr (!VEC) group.sync();                      // (what others have copied; what the row before has left)
    fetch(row + (stages - 1) * step, stage == 0 ? stages - 1 : stage - 1);
    const uint8_t* from = ring + stage * all_of;
    // (of these rows' addresses only the last four bits count, and those only where pieces do not begin on 16 bytes)
    const char *x = p.x + row * p.x_stride * kBytes, *dy = p.dy + row * p.dy_stride * kBytes, *ds = p.ds + row * p.ds_stride * kBytes;
    const float2 less = make_float2(-mean, -mean), times = make_float2(rstd, rstd);
    float2 along2 = make_float2(0.0f, 0.0f), all2 = along2;
    typename Part::Row held_h, held_g;
    const auto add_up = [&](bool clears) __attribute__((always_inline)) {
#pragma unroll
      for (int q = 0; q < Part::kPieces; q += Part::kStep) {
        float2 h[Part::kStepPairs], g[Part::kStepPairs], by[Part::kStepPairs];
        part.read_piece(from, x, q, h);
        part.read_piece(from + each, dy, q, g);
        part.read_shared(w, q, by);
#pragma unroll
        for (int k = 0; k < Part::kStepPairs; ++k) h[k] = mul2_rn(add2_rn(h[k], less), times);
        if (clears) part.clear_beyond(q, h);
#pragma unroll
        for (int k = 0; k < Part::kStepPairs; ++k) {
          const int i = q / Part::kStep * Part::kStepPairs + k;
          dw[i] = fma2_rn(g[k], h[k], dw[i]);
          db[i] = add2_rn(db[i], g[k]);
          g[k] = mul2_rn(g[k], by[k]);
          along2 = fma2_rn(g[k], h[k], along2);
          all2 = add2_rn(all2, g[k]);
          if constexpr (kHold) {
            held_h[i] = h[k];
            held_g[i] = g[k];
          }
        }
      }
    };
    // Beyond the row g is zero, and so is g h unless 0 - mean times rstd is infinite.  (Where three CTAs share an SM, one loop for both takes 131
    // us in place of 119 for 30012 x 2048 fp32; elsewhere two loops cost more: 200 in place of 192 for 16384 x 4096 fp32.)
    if constexpr (MANY && NV == 2 && WARPS == kGradWarps) {
      if (part.all || fabsf(mean * rstd) < __int_as_float(0x7F800000)) add_up(false);
      else add_up(true);
    } else {
      add_up(!part.all);
    }
    float along = along2.x + along2.y, all = all2.x + all2.y;
    group.mean2(along, all, width);
    const float2 minus_along = make_float2(-along, -along), minus_all = make_float2(-all, -all);
    if constexpr (!kHold) asm volatile("" ::: "memory");  // the row is read again
    char* dx = p.dx + row * p.dx_stride * kBytes;
#pragma unroll
    for (int q = 0; q < Part::kPieces; q += Part::kStep) {
      float2 h[Part::kStepPairs], g[Part::kStepPairs], by[Part::kStepPairs], s[Part::kStepPairs];
      if constexpr (!kHold) {
        part.read_piece(from, x, q, h);
        part.read_piece(from + each, dy, q, g);
      }
#pragma unroll
      for (int k = 0; k < Part::kStepPairs; ++k) s[k] = make_float2(0.0f, 0.0f);
      if (p.ds_ahead) part.read_piece(from + 2 * each, ds, q, s);
      else if (p.ds) part.load_piece(ds, q, s);
      if constexpr (!kHold) part.read_shared(w, q, by);
#pragma unroll
      for (int k = 0; k < Part::kStepPairs; ++k) {
        if constexpr (kHold) {
          h[k] = held_h[q / Part::kStep * Part::kStepPairs + k];
          g[k] = held_g[q / Part::kStep * Part::kStepPairs + k];
        } else {
          h[k] = mul2_rn(add2_rn(h[k], less), times);
          g[k] = mul2_rn(g[k], by[k]);
        }
        s[k] = fma2_rn(times, fma2_rn(h[k], minus_along, add2_rn(g[k], minus_all)), s[k]);
      }
      part.store_piece(dx, q, s);
    }
    stage = stage + 1 == stages ? 0 : stage + 1;
  }
  if (!p.partial) return;
  float* sums = p.partial + (size_t)blockIdx.x * 2 * p.width;
  float* to = groups == 1 ? sums : reinterpret_cast<float*>(slots) + (size_t)number * 2 * p.width;
  if (groups > 1) {
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
  }
#pragma unroll
  for (int q = 0; q < Part::kPieces; ++q) {
    if (part.has(q)) {
      if constexpr (VEC) {                                 // (16 bytes at a time: one by one, eight lanes would meet in a bank)
#pragma unroll
        for (int k = 0; k < Part::kPiece; k += 4) {
          const int i = (q * Part::kPiece + k) / 2, col = part.column(q) + k;
          *reinterpret_cast<float4*>(to + col) = make_float4(dw[i].x, dw[i].y, dw[i + 1].x, dw[i + 1].y);
          *reinterpret_cast<float4*>(to + p.width + col) = make_float4(db[i].x, db[i].y, db[i + 1].x, db[i + 1].y);
        }
      } else {
        to[part.column(q)] = q % 2 ? dw[q / 2].y : dw[q / 2].x;
        to[p.width + part.column(q)] = q % 2 ? db[q / 2].y : db[q / 2].x;
      }
    }
  }
  if (groups > 1) {
    __syncthreads();
    const float* each_of = reinterpret_cast<const float*>(slots);
    for (int i = threadIdx.x; i < 2 * p.width; i += blockDim.x) {
      float s = each_of[i];
      for (int n = 1; n < groups; ++n) s += each_of[n * 2 * p.width + i];
      sums[i] = s;
    }
  }
}

// Rows too wide for registers: the rows' gradient by reading twice, the columns' sums by another pass.  2000 x 20001 fp32: 280 us (480 MB, 74 at the
// copy rate).
template <int TY>
__global__ void __launch_bounds__(kWideThreads) wide_row_grad_kernel(const __grid_constant__ GradParams p) {
  __shared__ GroupShared shared;
  wait_for_previous_launch();
  constexpr int kBytes = TY == QADAM_F32 ? 4 : 2;
  RowGroup<true> group(&shared, kWideThreads / 32, 0);
  const long long row = blockIdx.x;
  const char* x = p.x + row * p.x_stride * kBytes;
  const char* dy = p.dy + row * p.dy_stride * kBytes;
  const float mean = p.mean[row], rstd = p.rstd[row];
  float along = 0.0f, all = 0.0f;
  for (int col = threadIdx.x; col < p.width; col += kWideThreads) {
    const float h = (load_one<TY>(x, col) - mean) * rstd;
    const float g = load_one<TY>(dy, col) * (p.w ? load_one_of(p.w, p.w_type, col) : 1.0f);
    along = fmaf(g, h, along);
    all += g;
  }
  group.mean2(along, all, RowWidth::of(p.width));
  for (int col = threadIdx.x; col < p.width; col += kWideThreads) {
    const float h = (load_one<TY>(x, col) - mean) * rstd;
    const float g = load_one<TY>(dy, col) * (p.w ? load_one_of(p.w, p.w_type, col) : 1.0f);
    store_one<TY>(p.dx + row * p.dx_stride * kBytes, col,
                  fmaf(rstd, (g - all) - h * along, p.ds ? load_one<TY>(p.ds + row * p.ds_stride * kBytes, col) : 0.0f));
  }
}

template <int TY>
__global__ void __launch_bounds__(256) wide_column_grad_kernel(const __grid_constant__ GradParams p, int chunks) {
  wait_for_previous_launch();
  constexpr int kBytes = TY == QADAM_F32 ? 4 : 2;
  const long long col = (long long)blockIdx.x / chunks * 256 + threadIdx.x;
  const int chunk = (int)(blockIdx.x % chunks);
  if (col >= p.width) return;
  const long long from = p.rows * chunk / chunks, to = p.rows * (chunk + 1) / chunks;
  float dw = 0.0f, db = 0.0f;
  for (long long row = from; row < to; ++row) {
    const float dy = load_one<TY>(p.dy + row * p.dy_stride * kBytes, col);
    dw = fmaf(dy, (load_one<TY>(p.x + row * p.x_stride * kBytes, col) - p.mean[row]) * p.rstd[row], dw);
    db += dy;
  }
  float* part = p.partial + (size_t)chunk * 2 * p.width;
  part[col] = dw;
  part[p.width + col] = db;
}

// The CTAs' sums joined, in an order that their number fixes: 32 columns of either sum to a CTA, the parts dealt out to its warps, who
// ask for ten at a time.
constexpr int kJoinWarps = 16;
__global__ void __launch_bounds__(kJoinWarps * 32) join_grad_kernel(const float* partial, int parts, int width, void* dw, void* db, int type,
                                                                   int accumulate) {
  __shared__ float sum[kJoinWarps][32];
  wait_for_previous_launch();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int tiles = (width + 31) / 32, which = (int)blockIdx.x / tiles;
  const int col = ((int)blockIdx.x - which * tiles) * 32 + lane;
  void* to = which == 0 ? dw : db;
  if (!to) return;
  float a = 0.0f;
  if (col < width) {
    const float* part = partial + ((size_t)warp * 2 + which) * width + col;
#pragma unroll 10
    for (int i = warp; i < parts; i += kJoinWarps, part += (size_t)kJoinWarps * 2 * width) a += *part;
  }
  sum[warp][lane] = a;
  __syncthreads();
  if (warp > 0 || col >= width) return;
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < kJoinWarps; ++i) s += sum[i][lane];
  store_one_of(to, type, col, accumulate ? load_one_of(to, type, col) + s : s);
}

// CTAs of the gradient, and so partial sums: as many as are on the device's SMs at a time, at most one to the rows of its groups.  (Shared memory may
// have room for fewer: then there are fewer, see launch_grad.)
struct GradShape {
  int pieces;                                              // NV of the kernel: 8 elements each
  int warps, groups, threads, per_sm;
};
GradShape grad_shape(int width, bool vec) {
  GradShape g;
  // Rows of a warp: 8, 16 or 24 elements to a thread.  Wider ones: 16, and so more warps on an SM (30012 x 2048 fp32: 119 us, with 24 147),
  // but 24 where elements are taken one by one and a row's ends cost more (30011 x 2049 fp32, when a row's ends were not yet fetched ahead: 194 us, with 16 222), and beyond 6144.
  g.pieces = width <= 768 ? (width + 255) / 256 : vec && width <= kGradMostWarps * 512 ? 2 : 3;
  g.warps = (width + 256 * g.pieces - 1) / (256 * g.pieces);
  g.groups = std::max(1, kGradWarps / g.warps);
  g.threads = g.warps * g.groups * 32;
  g.per_sm = std::max(1, grad_warps_of_sm(g.pieces, g.warps > 1) * 32 / g.threads);
  return g;
}
int grad_parts(long long rows, int width, bool vec) {
  if (width > kGradGroupWidth) return (int)std::min<long long>(rows, std::max(1, 4 * kSms * 256 / width));
  const GradShape g = grad_shape(width, vec);
  return (int)std::min<long long>((rows + g.groups - 1) / g.groups, g.per_sm * kSms);
}

template <int TY, int NV, bool VEC, bool MANY, int WARPS>
bool launch_grad(GradParams p, const GradShape& g, int& parts, cudaStream_t st) {
  const int slot = RowPart<TY, NV, VEC>::slot_bytes(g.warps * 32) * g.groups, weights = g.warps * 32 * 8 * NV * (int)sizeof(float);
  p.ds_ahead = p.ds && residents(g.threads, g.threads, 3 * slot, weights).stages > 0;               // (not for fp32 rows beyond 6144)
  const int bytes = (p.ds_ahead ? 3 : 2) * slot;
  const Residents r = residents(g.threads, g.per_sm * g.threads, bytes, weights);
  // (More CTAs than there is room for would come in a second wave: 30012 x 2048 fp32 with ds 191 us in place of 151.  With ds not fetched ahead, so
  // that there is room for all: 218.)
  parts = std::min(parts, r.per_sm * kSms);
  static_assert(kRingBytes - 2048 >= 4 * (kGradMostWarps * 768 * 4 + 32) + kGradMostWarps * 768 * 4, "two stages of two rows");
  const size_t smem = std::max((size_t)r.stages * bytes + weights, g.groups == 1 ? 0 : (size_t)g.groups * 2 * p.width * sizeof(float));
  return allow_ring<row_grad_kernel<TY, NV, VEC, MANY, WARPS>>(smem) && launch(row_grad_kernel<TY, NV, VEC, MANY, WARPS>, parts, g.threads, smem, 0, st, p, g.warps, r.stages);
}
template <int TY, bool VEC>
bool launch_grad(const GradParams& p, int& parts, cudaStream_t st) {
  const GradShape g = grad_shape(p.width, VEC);
  if (g.warps == 1) {
    return g.pieces == 1 ? launch_grad<TY, 1, VEC, false, kGradWarps>(p, g, parts, st)
           : g.pieces == 2 ? launch_grad<TY, 2, VEC, false, kGradWarps>(p, g, parts, st) : launch_grad<TY, 3, VEC, false, kGradWarps>(p, g, parts, st);
  }
  if constexpr (VEC) {
    if (g.warps <= kGradWarps) return launch_grad<TY, 2, VEC, true, kGradWarps>(p, g, parts, st);
    if (g.pieces == 2 && g.warps <= kGradMoreWarps) return launch_grad<TY, 2, VEC, true, kGradMoreWarps>(p, g, parts, st);
    return g.pieces == 2 ? launch_grad<TY, 2, VEC, true, kGradMostWarps>(p, g, parts, st) : launch_grad<TY, 3, VEC, true, kGradMostWarps>(p, g, parts, st);
  } else {
    return g.warps <= kGradWarps ? launch_grad<TY, 3, VEC, true, kGradWarps>(p, g, parts, st) : launch_grad<TY, 3, VEC, true, kGradMostWarps>(p, g, parts, st);
  }
}

template <int TY>
bool enqueue_grad_of(const GradParams& p, int& parts, bool vec, cudaStream_t st) {
  if (p.width <= kGradGroupWidth) return vec ? launch_grad<TY, true>(p, parts, st) : launch_grad<TY, false>(p, parts, st);
  if (!launch(wide_row_grad_kernel<TY>, p.rows, kWideThreads, 0, 0, st, p)) return false;
  return !p.partial || launch(wide_column_grad_kernel<TY>, (long long)(p.width + 255) / 256 * parts, 256, 0, 0, st, p, parts);
}

// ---------------------------------------------------------------- columns in 8 bits

// The largest values of 256 columns over a chunk of rows, then the transposed bytes: the second pass finds in L2 what the
// first has read, as long as it is not larger than that.  8192 x 2304 bf16: 13 us (57 MB, 8.8 at the copy rate; the second pass is bound by its
// instructions, 10 an element); 16384 x 4096, read twice from HBM: 65 us (335 MB, 52).
constexpr int kColThreads = 256;
constexpr int kColMaxChunks = 64;
constexpr int kTileRows = 128, kTileCols = 64, kTilesEach = 4;       // kTilesEach: tiles below each other that a CTA takes

struct ColumnParams {
  const char* x;
  long long stride;
  long long rows;
  int width, chunks;
  uint32_t* largest;                                       // [chunks][width], bits
  signed char* q;
  long long q_stride;
  float* scale;
};

template <int TY, bool VEC>
__global__ void __launch_bounds__(kColThreads) column_max_kernel(const __grid_constant__ ColumnParams p) {
  __shared__ uint32_t best[kColThreads / 32][256];
  wait_for_previous_launch();
  constexpr int kBytes = TY == QADAM_F32 ? 4 : 2;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const long long first = (long long)(blockIdx.x / p.chunks) * 256;
  const int chunk = (int)(blockIdx.x % p.chunks);
  const long long from = p.rows * chunk / p.chunks, to = p.rows * (chunk + 1) / p.chunks;
  uint32_t m[8] = {};
#pragma unroll 16
  for (long long row = from + warp; row < to; row += kColThreads / 32) {
    const char* x = p.x + row * p.stride * kBytes;
    if constexpr (VEC) {
      const long long col = first + lane * 8;
      if (col < p.width) {
        float v[8];
        raw8_to_floats<TY>(load_raw8<TY>(x + col * kBytes), v);
#pragma unroll
        for (int k = 0; k < 8; ++k) m[k] = max(m[k], abs_bits(v[k]));
      }
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const long long col = first + k * 32 + lane;
        if (col < p.width) m[k] = max(m[k], abs_bits(load_one<TY>(x, col)));
      }
    }
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) best[warp][VEC ? lane * 8 + k : k * 32 + lane] = m[k];
  __syncthreads();
  uint32_t v = 0u;
#pragma unroll
  for (int w = 0; w < kColThreads / 32; ++w) v = max(v, best[w][threadIdx.x]);
  if (first + threadIdx.x < p.width) p.largest[(size_t)chunk * p.width + first + threadIdx.x] = v;
}

template <int TY, bool VEC>
__global__ void __launch_bounds__(kColThreads) column_bytes_kernel(const __grid_constant__ ColumnParams p, int row_blocks) {
  __shared__ uint32_t most[kColThreads / kTileCols][kTileCols];
  __shared__ float per[kTileCols];
  // a column's bytes; the words of columns that a warp writes at a time are swapped so that they fall into different banks
  __shared__ __align__(16) uint32_t tile[kTileCols][kTileRows / 4];
  const auto swap = [](int c) { return (VEC ? c >> 3 : c) & 7; };
  wait_for_previous_launch();
  constexpr int kBytes = TY == QADAM_F32 ? 4 : 2;
  const long long first = (long long)(blockIdx.x / row_blocks) * kTileCols;
  const long long from = (long long)(blockIdx.x % row_blocks) * (kTilesEach * kTileRows);
  // a warp has 4 rows at a time in each of 4 groups of eight lanes; a lane 8 columns
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int quad = warp * 4 + lane / 8;                                      // 32 groups of 4 rows
  const int c0 = VEC ? lane % 8 * 8 : lane % 8;
  const int columns_left = (int)min((long long)kTileCols, p.width - first) - c0;
  const char* x = p.x + ((from + quad * 4) * p.stride + first + c0) * kBytes;
  const long long row_bytes = p.stride * kBytes;
  // four rows of the tile that begins at `top`, as they lie in memory
  struct Four {
    Raw8<VEC ? TY : QADAM_F32> row[4];
  };
  const auto load = [&](long long top, const char* at) {
    Four f = {};
    const int rows_left = (int)max(0ll, min((long long)4, p.rows - top - quad * 4));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (VEC) {
        if (i < rows_left && columns_left > 0) f.row[i] = load_raw8<TY>(at + i * row_bytes);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) f.row[i].w[k] = i < rows_left && 8 * k < columns_left ? __float_as_uint(load_one<TY>(at + i * row_bytes, 8 * k)) : 0u;
      }
    }
    return f;
  };
  Four now = load(from, x);
  const int mine = threadIdx.x % kTileCols;
  if (first + mine < p.width) {
    constexpr int kShare = kColThreads / kTileCols;
    uint32_t m = 0u;
    const uint32_t* from = p.largest + (size_t)(threadIdx.x / kTileCols) * p.width + first + mine;
#pragma unroll 8
    for (int chunk = threadIdx.x / kTileCols; chunk < p.chunks; chunk += kShare, from += (size_t)kShare * p.width) m = max(m, *from);
    most[threadIdx.x / kTileCols][mine] = m;
  }
  __syncthreads();
  if (threadIdx.x < kTileCols && first + threadIdx.x < p.width) {
    const ByteScale s = byte_scale(max(max(most[0][threadIdx.x], most[1][threadIdx.x]), max(most[2][threadIdx.x], most[3][threadIdx.x])));
    per[threadIdx.x] = s.per;
    if (from == 0) p.scale[first + threadIdx.x] = s.worth;
  }
  __syncthreads();
  float f[8];
  constexpr int kNext = VEC ? 1 : 8;
#pragma unroll
  for (int k = 0; k < 8; ++k) f[k] = k * kNext < columns_left ? per[c0 + k * kNext] : 0.0f;
  uint32_t* to = &tile[c0][quad ^ swap(c0) << 2];            // (the same swap for all columns of a thread)
#pragma unroll 1
  for (int n = 0; n < kTilesEach; ++n) {
    const long long top = from + n * kTileRows;
    if (top >= p.rows) return;
    x += kTileRows * row_bytes;
    const Four next = n + 1 < kTilesEach ? load(top + kTileRows, x) : now;
    float v[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) raw8_to_floats<VEC ? TY : QADAM_F32>(now.row[i], v[i]);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t bytes = to_bytes(make_float2(v[0][k], v[1][k]), make_float2(v[2][k], v[3][k]), f[k]);
      if (k * kNext < columns_left) to[k * kNext * (kTileRows / 4)] = f[k] > 0.0f ? bytes : 0u;
    }
    __syncthreads();
    // 16 rows' bytes of a column at a time; columns of the result have room up to a multiple of 16
    for (int i = threadIdx.x; i < kTileCols * (kTileRows / 16); i += kColThreads) {
      const int c = i / (kTileRows / 16), part = i % (kTileRows / 16);
      const long long row = top + part * 16;
      if (first + c < p.width && row < p.rows)
        *reinterpret_cast<uint4*>(p.q + (first + c) * p.q_stride + row) = *reinterpret_cast<const uint4*>(&tile[c][(part ^ swap(c)) * 4]);
    }
    __syncthreads();
    now = next;
  }
}

int column_chunks(long long rows, long long width) {
  const long long strips = (width + 255) / 256;
  return (int)std::max<long long>(1, std::min<long long>({(long long)kColMaxChunks, rows / 32, (6 * kSms + strips - 1) / strips}));
}

template <int TY, bool VEC>
bool launch_columns(const ColumnParams& p, cudaStream_t st) {
  const long long strips = (p.width + 255) / 256, tiles = (p.width + kTileCols - 1) / kTileCols;
  const int row_blocks = (int)((p.rows + kTilesEach * kTileRows - 1) / (kTilesEach * kTileRows));
  return launch(column_max_kernel<TY, VEC>, strips * p.chunks, kColThreads, 0, 0, st, p) &&
         launch(column_bytes_kernel<TY, VEC>, tiles * row_blocks, kColThreads, 0, 0, st, p, row_blocks);
}

// ---------------------------------------------------------------- packed weights as rows of 8 bits

struct HeldParams {
  const uint32_t* codes;
  long long words;
  long long first;
  long long rows;
  int width, pieces;                                       // pieces of 16 elements in a row
  signed char* q;
  long long q_stride;
  float* scale;
};

// A thread decodes 16 consecutive codes: (16 BITS + 31) / 32 + 1 words at most, one store of 16 bytes.  1537 x 1001 codes of 4 bits: 1.7 us; 8192 x 8192
// of 8 bits 24.5 (134 MB, 21 at the copy rate), of 4 bits 23.5 (16).
template <int BITS>
__global__ void __launch_bounds__(256) held_rows_kernel(const __grid_constant__ HeldParams p) {
  wait_for_previous_launch();
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  const long long row = i / p.pieces;
  const int col = (int)(i % p.pieces) * 16;
  if (row >= p.rows) return;
  const long long bit = (p.first + row * p.width + col) * BITS;
  const long long at = bit >> 5;
  const int shift = (int)(bit & 31);
  constexpr int kWords = (16 * BITS + 31 + 31) / 32;
  uint32_t w[kWords + 1];
#pragma unroll
  for (int k = 0; k < kWords; ++k) w[k] = p.codes[min(at + k, p.words - 1)];    // (a row may end before the piece does)
  w[kWords] = 0u;
  uint32_t packed[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int k = 0; k < kWords; ++k) w[k] = __funnelshift_r(w[k], w[k + 1], shift);
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const int from = k * BITS, j = from / 32, b = from % 32;
    uint32_t code = w[j] >> b;
    if (b + BITS > 32) code |= w[j + 1] << (32 - b);
    const int level = (int)(code & ((1u << BITS) - 1u)) - (1 << (BITS - 2));
    packed[k / 4] |= (uint32_t)(level & 255) << (8 * (k % 4));
  }
  *reinterpret_cast<uint4*>(p.q + row * p.q_stride + col) = make_uint4(packed[0], packed[1], packed[2], packed[3]);
  if (p.scale && col == 0) p.scale[row] = 1.0f / (float)(1 << (BITS - 1));
}

// ---------------------------------------------------------------- arguments

constexpr int64_t kMostRows = (int64_t)1 << 31, kMostWidth = (int64_t)1 << 24;

bool bad_rows(int64_t rows, int64_t width) { return rows < 0 || rows >= kMostRows || width < 1 || width > kMostWidth; }
bool bad_stride(int64_t stride, int64_t width) { return stride < width || stride > (int64_t)1 << 40; }
bool whole(int64_t width, int type) { return width * type_bytes(type) % 16 == 0; }               // pieces of 16 bytes
// What a row's parameters may be read as (see RowParams): vec: they have to begin on 16 bytes for it.
int alike_type(const void* w, int w_type, const void* b, int b_type, bool vec) {
  if (!w || (b && b_type != w_type) || (vec && (!is_aligned(w, 16) || !is_aligned(b, 16)))) return kAnyType;
  return w_type;
}
bool on16(const void* p, int64_t stride, int type) { return is_aligned(p, 16) && stride * type_bytes(type) % 16 == 0; }

}  // namespace

extern "C" {

int qadam_layer_norm(const qadam_layer_norm_args* args, void* stream) {
  if (!args) return QADAM_ERR_NULL;
  const auto [x, x_stride, residual, residual_stride, weight, bias, rows, width, sum, sum_stride, out, out_stride, mean, rstd, q, q_stride, scale, sums, type,
              weight_type, bias_type, eps] = *args;
  if (bad_rows(rows, width)) return QADAM_ERR_SIZE;
  if (!known_type(type) || (weight && !known_type(weight_type)) || (bias && !known_type(bias_type))) return QADAM_ERR_TYPE;
  if (!(eps >= 0.0f) || !std::isfinite(eps)) return QADAM_ERR_HYPER;
  if ((rows > 0 && !x) || (residual != nullptr) != (sum != nullptr) || (!out && !q && !mean && !rstd) || (q && !scale)) return QADAM_ERR_NULL;
  if (bad_stride(x_stride, width) || (residual && (bad_stride(residual_stride, width) || bad_stride(sum_stride, width))) ||
      (out && bad_stride(out_stride, width)) || (q && bad_stride(q_stride, width)))
    return QADAM_ERR_SIZE;
  const size_t e = type_bytes(type);
  if (!is_aligned(x, e) || !is_aligned(residual, e) || !is_aligned(sum, e) || !is_aligned(out, e) ||
      (weight && !is_aligned(weight, type_bytes(weight_type))) || (bias && !is_aligned(bias, type_bytes(bias_type))) || !is_aligned(mean, 4) ||
      !is_aligned(rstd, 4) || !is_aligned(scale, 4) || !is_aligned(sums, 4) || (q && (!is_aligned(q, 16) || q_stride % 16 != 0)))
    return QADAM_ERR_ALIGN;
  if (rows == 0) return QADAM_OK;
  RowParams p = {};
  p.x = static_cast<const char*>(x); p.x_stride = x_stride;
  p.r = static_cast<const char*>(residual); p.r_stride = residual_stride;
  p.w = weight; p.w_type = weight_type;
  p.b = bias; p.b_type = bias_type;
  p.sum = static_cast<char*>(sum); p.sum_stride = sum_stride;
  p.out = static_cast<char*>(out); p.out_stride = out_stride;
  p.mean = mean; p.rstd = rstd;
  p.q = reinterpret_cast<signed char*>(q); p.q_stride = q_stride; p.scale = scale; p.sums = sums;
  p.rows = rows; p.width = (int)width; p.by = RowWidth::of(p.width); p.normed = 1; p.eps = eps;
  const bool vec = whole(width, type) && on16(x, x_stride, type) && (!residual || (on16(residual, residual_stride, type) && on16(sum, sum_stride, type))) &&
                   (!out || on16(out, out_stride, type));
  p.alike = alike_type(weight, weight_type, bias, bias_type, vec);
  return enqueue_rows(p, type, vec, static_cast<cudaStream_t>(stream));
}

int qadam_quantize_rows(const void* x, int32_t type, int64_t x_stride, const float* columns, int64_t rows, int64_t width, int8_t* q,
                        int64_t q_stride, float* scale, int32_t* sums, void* stream) {
  if (bad_rows(rows, width) || bad_stride(x_stride, width) || bad_stride(q_stride, width)) return QADAM_ERR_SIZE;
  if (!known_type(type)) return QADAM_ERR_TYPE;
  if (rows > 0 && (!x || !q || !scale)) return QADAM_ERR_NULL;
  if (!is_aligned(x, type_bytes(type)) || !is_aligned(columns, 4) || !is_aligned(q, 16) || q_stride % 16 != 0 || !is_aligned(scale, 4) ||
      !is_aligned(sums, 4))
    return QADAM_ERR_ALIGN;
  if (rows == 0) return QADAM_OK;
  RowParams p = {};
  p.x = static_cast<const char*>(x); p.x_stride = x_stride;
  p.w = columns; p.w_type = QADAM_F32;
  p.q = reinterpret_cast<signed char*>(q); p.q_stride = q_stride; p.scale = scale; p.sums = sums;
  p.rows = rows; p.width = (int)width;
  const bool vec = whole(width, type) && on16(x, x_stride, type);
  p.alike = alike_type(columns, QADAM_F32, nullptr, 0, vec);
  return enqueue_rows(p, type, vec, static_cast<cudaStream_t>(stream));
}

int qadam_layer_norm_grad_query_sizes(int64_t rows, int64_t width, size_t* workspace_bytes) {
  if (bad_rows(rows, width)) return QADAM_ERR_SIZE;
  const int parts = std::max(grad_parts(rows, (int)width, true), grad_parts(rows, (int)width, false));   // (the call may meet either)
  if (workspace_bytes) *workspace_bytes = round_up256((size_t)parts * 2 * (size_t)width * sizeof(float));
  return QADAM_OK;
}

int qadam_layer_norm_grad(const qadam_layer_norm_grad_args* args, void* stream) {
  if (!args) return QADAM_ERR_NULL;
  const auto [dy, dy_stride, x, x_stride, mean, rstd, weight, dsum, dsum_stride, rows, width, dx, dx_stride, dweight, dbias, workspace, workspace_bytes, type,
              weight_type, grad_type, accumulate] = *args;
  if (bad_rows(rows, width)) return QADAM_ERR_SIZE;
  const bool sums = dweight || dbias;
  if (!known_type(type) || (weight && !known_type(weight_type)) || (sums && !known_type(grad_type))) return QADAM_ERR_TYPE;
  const bool vec = whole(width, type) && on16(dy, dy_stride, type) && on16(x, x_stride, type) && on16(dx, dx_stride, type) &&
                   (!dsum || on16(dsum, dsum_stride, type));
  int parts = grad_parts(rows, (int)width, vec);
  if ((rows > 0 && (!dy || !x || !mean || !rstd || !dx)) || (sums && parts > 0 && !workspace)) return QADAM_ERR_NULL;
  if (bad_stride(dy_stride, width) || bad_stride(x_stride, width) || bad_stride(dx_stride, width) || (dsum && bad_stride(dsum_stride, width)))
    return QADAM_ERR_SIZE;
  if (accumulate != 0 && accumulate != 1) return QADAM_ERR_SIZE;
  const size_t e = type_bytes(type);
  if (!is_aligned(dy, e) || !is_aligned(x, e) || !is_aligned(dsum, e) || !is_aligned(dx, e) || !is_aligned(mean, 4) || !is_aligned(rstd, 4) ||
      (weight && !is_aligned(weight, type_bytes(weight_type))) ||
      (sums && (!is_aligned(dweight, type_bytes(grad_type)) || !is_aligned(dbias, type_bytes(grad_type)) || !is_aligned(workspace, 256))))
    return QADAM_ERR_ALIGN;
  if (sums && workspace_bytes < parts * 2 * width * (int64_t)sizeof(float)) return QADAM_ERR_WORKSPACE;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (rows > 0) {
    GradParams p = {};
    p.dy = static_cast<const char*>(dy); p.dy_stride = dy_stride;
    p.x = static_cast<const char*>(x); p.x_stride = x_stride;
    p.ds = static_cast<const char*>(dsum); p.ds_stride = dsum_stride;
    p.dx = static_cast<char*>(dx); p.dx_stride = dx_stride;
    p.mean = mean; p.rstd = rstd;
    p.w = weight; p.w_type = weight_type;
    p.partial = sums ? static_cast<float*>(workspace) : nullptr;
    p.rows = rows; p.width = (int)width;
    const bool ok = type == QADAM_F32 ? enqueue_grad_of<QADAM_F32>(p, parts, vec, st)
                    : type == QADAM_BF16 ? enqueue_grad_of<QADAM_BF16>(p, parts, vec, st) : enqueue_grad_of<QADAM_F16>(p, parts, vec, st);
    if (!ok) return QADAM_ERR_CUDA;
  }
  if (sums && (rows > 0 || !accumulate)) {
    if (!launch(join_grad_kernel, 2 * ((width + 31) / 32), kJoinWarps * 32, 0, 0, st, static_cast<const float*>(workspace), parts, (int)width, dweight, dbias,
                (int)grad_type, (int)accumulate))
      return QADAM_ERR_CUDA;
  }
  return QADAM_OK;
}

int qadam_quantize_columns_query_sizes(int64_t rows, int64_t width, size_t* workspace_bytes) {
  if (bad_rows(rows, width)) return QADAM_ERR_SIZE;
  if (workspace_bytes) *workspace_bytes = round_up256((size_t)column_chunks(rows, width) * (size_t)width * sizeof(uint32_t));
  return QADAM_OK;
}

int qadam_quantize_columns(const void* x, int32_t type, int64_t x_stride, int64_t rows, int64_t width, int8_t* q, int64_t q_stride, float* scale,
                           void* workspace, size_t workspace_bytes, void* stream) {
  if (bad_rows(rows, width) || rows < 1 || bad_stride(x_stride, width) || bad_stride(q_stride, (rows + 15) / 16 * 16)) return QADAM_ERR_SIZE;
  if (!known_type(type)) return QADAM_ERR_TYPE;
  if (!x || !q || !scale || !workspace) return QADAM_ERR_NULL;
  if (!is_aligned(x, type_bytes(type)) || !is_aligned(q, 16) || q_stride % 16 != 0 || !is_aligned(scale, 4) || !is_aligned(workspace, 256))
    return QADAM_ERR_ALIGN;
  ColumnParams p = {};
  p.x = static_cast<const char*>(x); p.stride = x_stride; p.rows = rows; p.width = (int)width;
  p.chunks = column_chunks(rows, width);
  if (workspace_bytes < (size_t)p.chunks * (size_t)width * sizeof(uint32_t)) return QADAM_ERR_WORKSPACE;
  p.largest = static_cast<uint32_t*>(workspace);
  p.q = reinterpret_cast<signed char*>(q); p.q_stride = q_stride; p.scale = scale;
  if ((width + kTileCols - 1) / kTileCols * ((rows + kTileRows - 1) / kTileRows) >= kMostRows) return QADAM_ERR_SIZE;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool vec = width % 8 == 0 && on16(x, x_stride, type);
  const bool ok = type == QADAM_F32    ? (vec ? launch_columns<QADAM_F32, true>(p, st) : launch_columns<QADAM_F32, false>(p, st))
                  : type == QADAM_BF16 ? (vec ? launch_columns<QADAM_BF16, true>(p, st) : launch_columns<QADAM_BF16, false>(p, st))
                                       : (vec ? launch_columns<QADAM_F16, true>(p, st) : launch_columns<QADAM_F16, false>(p, st));
  return ok ? QADAM_OK : QADAM_ERR_CUDA;
}

int qadam_held_rows(const void* wcodes, size_t wcode_bytes, int32_t kx, int64_t first, int64_t rows, int64_t width, int8_t* q,
                    int64_t q_stride, float* scale, void* stream) {
  if (bad_rows(rows, width) || bad_stride(q_stride, (width + 15) / 16 * 16)) return QADAM_ERR_SIZE;
  if (kx < 0 || kx > 6) return QADAM_ERR_LEVEL;
  if (!wcodes || (rows > 0 && !q)) return QADAM_ERR_NULL;
  if (!is_aligned(wcodes, 16) || !is_aligned(q, 16) || q_stride % 16 != 0 || !is_aligned(scale, 4)) return QADAM_ERR_ALIGN;
  if (first < 0 || first > (int64_t)1 << 44 || wcode_bytes % 16 != 0 || wcode_bytes / 2 > (size_t)1 << 44) return QADAM_ERR_SIZE;
  const int64_t held = (int64_t)(wcode_bytes * 8 / (size_t)(kx + 2));
  if (first > held || rows > (held - first) / width) return QADAM_ERR_SIZE;
  if (rows == 0) return QADAM_OK;
  HeldParams p = {};
  p.codes = static_cast<const uint32_t*>(wcodes); p.words = (long long)(wcode_bytes / 4); p.first = first;
  p.rows = rows; p.width = (int)width; p.pieces = (int)((width + 15) / 16);
  p.q = reinterpret_cast<signed char*>(q); p.q_stride = q_stride; p.scale = scale;
  const long long grid = (rows * p.pieces + 255) / 256;
  if (grid >= kMostRows) return QADAM_ERR_SIZE;
  using Kernel = void (*)(HeldParams);
  static constexpr Kernel kernels[] = {held_rows_kernel<2>, held_rows_kernel<3>, held_rows_kernel<4>, held_rows_kernel<5>,
                                       held_rows_kernel<6>, held_rows_kernel<7>, held_rows_kernel<8>};
  return launch(kernels[kx], grid, 256, 0, 0, static_cast<cudaStream_t>(stream), p) ? QADAM_OK : QADAM_ERR_CUDA;
}

}  // extern "C"
