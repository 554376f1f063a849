// Layer norm and its gradients, rows and columns in 8 bits, packed weights as rows of 8 bits:
// qadam_layer_norm*, qadam_quantize_*, qadam_held_rows.
#include "qadam.h"

#include <algorithm>
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
  int w_type, w_vec;
  const void* b;
  int b_type, b_vec;
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
  int normed;                                              // 0: the rows are quantized as they are (times w, if given)
  float eps;
};

// ---------------------------------------------------------------- rows in registers

// What becomes of a row h, dealt out to a group's threads: normed, scaled, written, in 8 bits.
template <int TY, int NV, bool VEC, bool MANY>
__device__ __forceinline__ void finish_row(const RowParams& p, const RowPart<TY, NV, VEC>& part, RowGroup<MANY>& group, long long row, float2 (&h)[4 * NV]) {
  using Part = RowPart<TY, NV, VEC>;
  if (p.normed) {
    float2 s = h[0];
#pragma unroll
    for (int i = 1; i < Part::kPairs; ++i) s = add2_rn(s, h[i]);
    const float mean = group.add(s.x + s.y) / (float)p.width;
    const float2 less = make_float2(-mean, -mean);
    s = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < Part::kPairs; ++i) {
      h[i] = add2_rn(h[i], less);
      if constexpr (VEC) {
        if (!part.has(Part::piece_of(2 * i))) h[i] = make_float2(0.0f, 0.0f);
      } else {
        if (!part.has(2 * i)) h[i].x = 0.0f;
        if (!part.has(2 * i + 1)) h[i].y = 0.0f;
      }
      s = fma2_rn(h[i], h[i], s);
    }
    const float rstd = 1.0f / sqrtf(group.add(s.x + s.y) / (float)p.width + p.eps);
    if (part.t == 0) {
      if (p.mean) p.mean[row] = mean;
      if (p.rstd) p.rstd[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < Part::kPairs; ++i) h[i] = mul2_rn(h[i], make_float2(rstd, rstd));
  }
  if (p.w || p.b) {
#pragma unroll
    for (int q = 0; q < Part::kPieces; q += Part::kStep) {
      float2 w[Part::kStepPairs], b[Part::kStepPairs];
#pragma unroll
      for (int k = 0; k < Part::kStepPairs; ++k) w[k] = b[k] = make_float2(0.0f, 0.0f);               // (beyond the row: zero)
      if (p.w) part.read_parameters(p.w, p.w_type, p.w_vec, q, w);
      if (p.b) part.read_parameters(p.b, p.b_type, p.b_vec, q, b);
#pragma unroll
      for (int k = 0; k < Part::kStepPairs; ++k) {
        float2& y = h[q / Part::kStep * Part::kStepPairs + k];
        y = p.w ? p.b ? fma2_rn(y, w[k], b[k]) : mul2_rn(y, w[k]) : add2_rn(y, b[k]);
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
#pragma unroll
    for (int i = 0; i < Part::kPairs; i += 2) {
      const uint32_t c = to_bytes(h[i], h[i + 1], s.per) & finite;
      sum = __dp4a((int)c, 0x01010101, sum);               // (beyond the row: zeros)
      if constexpr (VEC) {
        constexpr int kWords = Part::kPiece / 4;           // of a piece
        if (part.has(i / (2 * kWords))) *reinterpret_cast<uint32_t*>(q + part.column(i / (2 * kWords)) + i / 2 % kWords * 4) = c;
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (part.has(2 * i + k)) q[part.column(2 * i + k)] = (signed char)(c >> (8 * k));
      }
    }
    if (p.sums) sum = group.add(sum);
    if (part.t == 0) {
      p.scale[row] = s.worth;
      if (p.sums) p.sums[row] = sum;
    }
  }
}

// One pass: a row is read once, held in registers for mean, sum of squares around it and largest value, and written once.
// Bound by HBM.  There is a warp for each row: enough of them are on an SM to keep its share of the loads under way.
template <int TY, int NV, bool VEC>
__global__ void __launch_bounds__(kWarpRowThreads) warp_row_kernel(const __grid_constant__ RowParams p) {
  wait_for_previous_launch();
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
  finish_row(p, part, group, row, h);
}

// Wider rows: a group of warps goes from row to row, with the next ones under way.
constexpr int kGroupWarps = 8;                             // of a CTA, in groups, or one group of up to 16
template <int TY, int NV, bool VEC, int MOST>
__global__ void __launch_bounds__(MOST, MOST == 256 ? 3 : 1) group_row_kernel(const __grid_constant__ RowParams p, int warps, int stages) {
  extern __shared__ __align__(16) uint8_t slots[];         // [groups][stages][1 or 2][a row]
  __shared__ GroupShared shared[kGroupWarps];
  wait_for_previous_launch();
  using Part = RowPart<TY, NV, VEC>;
  const int threads = warps * 32, number = (int)threadIdx.x / threads;
  const int groups = blockDim.x / threads;
  const Part part(p.width, threads, (int)threadIdx.x % threads);
  RowGroup<true> group(&shared[number], warps, number);
  const int each = Part::slot_bytes(p.width), both = p.r ? 2 * each : each;
  uint8_t* ring = slots + number * stages * both;
  const long long first = (long long)blockIdx.x * groups + number, step = (long long)gridDim.x * groups;
  const auto fetch = [&](long long row, int stage) {
    if (row < p.rows) {
      part.fetch(ring + stage * both, p.x + row * p.x_stride * Part::kBytes);
      if (p.r) part.fetch(ring + stage * both + each, p.r + row * p.r_stride * Part::kBytes);
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
    finish_row(p, part, group, row, h);
    stage = stage + 1 == stages ? 0 : stage + 1;
  }
}

// Rows too wide for a CTA's registers: read again for each thing that is known only at the row's end.
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

template <int TY, int NV>
bool launch_warp_rows(const RowParams& p, bool vec, cudaStream_t st) {
  const long long grid = (p.rows + kWarpRowThreads / 32 - 1) / (kWarpRowThreads / 32);
  return vec ? launch(warp_row_kernel<TY, NV, true>, grid, kWarpRowThreads, 0, 0, st, p) : launch(warp_row_kernel<TY, NV, false>, grid, kWarpRowThreads, 0, 0, st, p);
}

// CTAs of `threads` threads that an SM has at a time (of most_threads), and stages of `bytes` that each of them has then: 2 or 3,
// or none if two do not fit.
struct Residents {
  int per_sm, stages;
};
Residents residents(int threads, int most_threads, int bytes) {
  const int per_sm = std::max(1, std::min(most_threads / threads, kRingBytes / (2 * bytes + 2048)));
  const int stages = std::min(3, (kRingBytes / per_sm - 2048) / bytes);
  return {per_sm, stages < 2 ? 0 : stages};
}

// The limit of dynamic shared memory belongs to the kernel: it is raised to the same for every launch that needs it.
template <typename K>
bool allow_ring(K kernel, size_t bytes) {
  return bytes <= 40 * 1024 || cuda_call(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes));
}

template <int TY, int NV, bool VEC>
bool launch_group_rows(const RowParams& p, cudaStream_t st) {
  const int warps = (p.width + 256 * NV - 1) / (256 * NV), groups = std::max(1, kGroupWarps / warps);
  const int threads = warps * groups * 32, bytes = RowPart<TY, NV, VEC>::slot_bytes(p.width) * (p.r ? 2 : 1) * groups;
  const Residents r = residents(threads, kGroupMostThreads, bytes);
  if (r.stages == 0) return launch(wide_row_kernel<TY>, p.rows, kWideThreads, 0, 0, st, p);
  const auto kernel = threads <= 256 ? group_row_kernel<TY, NV, VEC, 256> : group_row_kernel<TY, NV, VEC, 512>;
  return allow_ring(kernel, (size_t)r.stages * bytes) &&
         launch(kernel, std::min<long long>((p.rows + groups - 1) / groups, (long long)kSms * r.per_sm), threads, (size_t)r.stages * bytes, 0, st, p, warps,
                r.stages);
}
template <int TY, int NV>
bool launch_group_rows(const RowParams& p, bool vec, cudaStream_t st) {
  return vec ? launch_group_rows<TY, NV, true>(p, st) : launch_group_rows<TY, NV, false>(p, st);
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

constexpr int kGradWarps = 12;                             // of a CTA, in groups, or one group of up to 32
constexpr int kGradGroupWidth = 8192;                      // beyond, rows are read again, and the columns' sums are a pass of their own

struct GradParams {
  const char* dy;
  long long dy_stride;
  const char* x;
  long long x_stride;
  const char* ds;
  long long ds_stride;
  char* dx;
  long long dx_stride;
  const float* mean;
  const float* rstd;
  const void* w;
  int w_type, w_vec;
  float* partial;                                          // [gridDim.x][2][width], or NULL
  long long rows;
  int width;
};

// A group of warps, eight elements to a thread, goes from row to row, with the next ones under way, and adds up its rows' part of the
// weight's and bias's gradients in registers; the CTA's sums go to the workspace.  One read, one write: bound by HBM.
template <int TY, bool VEC, int MOST>
__global__ void __launch_bounds__(MOST, MOST <= kGradWarps * 32 ? 2 : 1) row_grad_kernel(const __grid_constant__ GradParams p, int warps, int stages) {
  extern __shared__ __align__(16) uint8_t slots[];         // [groups][stages][2 or 3][a row]; at the end the groups' sums [groups][2][width]
  __shared__ GroupShared shared[kGradWarps];
  wait_for_previous_launch();
  using Part = RowPart<TY, 1, VEC>;
  constexpr int kBytes = Part::kBytes;
  const int threads = warps * 32, number = (int)threadIdx.x / threads;
  const int groups = blockDim.x / threads;
  const Part part(p.width, threads, (int)threadIdx.x % threads);
  RowGroup<true> group(&shared[number], warps, number);
  const int each = Part::slot_bytes(p.width), all_of = p.ds ? 3 * each : 2 * each;
  uint8_t* ring = slots + number * stages * all_of;
  const float per = 1.0f / (float)p.width;
  const long long first = (long long)blockIdx.x * groups + number, step = (long long)gridDim.x * groups;
  const auto fetch = [&](long long row, int stage) {
    if (row < p.rows) {
      uint8_t* to = ring + stage * all_of;
      part.fetch(to, p.x + row * p.x_stride * kBytes);
      part.fetch(to + each, p.dy + row * p.dy_stride * kBytes);
      if (p.ds) part.fetch(to + 2 * each, p.ds + row * p.ds_stride * kBytes);
    }
    fetched();
  };
  for (int i = 0; i + 1 < stages; ++i) fetch(first + i * step, i);
  typename Part::Row dw, db, w;
#pragma unroll
  for (int i = 0; i < Part::kPairs; ++i) {
    dw[i] = db[i] = make_float2(0.0f, 0.0f);
    w[i] = make_float2(1.0f, 1.0f);
  }
  if (p.w) {
#pragma unroll
    for (int q = 0; q < Part::kPieces; q += Part::kStep) part.read_parameters(p.w, p.w_type, p.w_vec, q, &w[q / Part::kStep * Part::kStepPairs]);
  }
  int stage = 0;
  for (long long row = first; row < p.rows; row += step) {
    const float mean = p.mean[row], rstd = p.rstd[row];
    wait_fetched(stages - 2);
    if constexpr (!VEC) group.sync();                      // (what others have copied; what the row before has left)
    fetch(row + (stages - 1) * step, stage == 0 ? stages - 1 : stage - 1);
    const uint8_t* from = ring + stage * all_of;
    const float2 less = make_float2(-mean, -mean), times = make_float2(rstd, rstd);
    typename Part::Row h, g;
    part.read_slot(from, p.x + row * p.x_stride * kBytes, h);
    part.read_slot(from + each, p.dy + row * p.dy_stride * kBytes, g);
    float2 along2 = make_float2(0.0f, 0.0f), all2 = along2;
#pragma unroll
    for (int i = 0; i < Part::kPairs; ++i) {               // (beyond the row g is zero)
      h[i] = mul2_rn(add2_rn(h[i], less), times);
      dw[i] = fma2_rn(g[i], h[i], dw[i]);
      db[i] = add2_rn(db[i], g[i]);
      g[i] = mul2_rn(g[i], w[i]);
      along2 = fma2_rn(g[i], h[i], along2);
      all2 = add2_rn(all2, g[i]);
    }
    float along = along2.x + along2.y, all = all2.x + all2.y;
    group.add2(along, all);
    along *= -per;
    all *= -per;
    typename Part::Row s;
    if (p.ds) {
      part.read_slot(from + 2 * each, p.ds + row * p.ds_stride * kBytes, s);
    } else {
#pragma unroll
      for (int i = 0; i < Part::kPairs; ++i) s[i] = make_float2(0.0f, 0.0f);
    }
#pragma unroll
    for (int i = 0; i < Part::kPairs; ++i)
      s[i] = fma2_rn(times, fma2_rn(h[i], make_float2(along, along), add2_rn(g[i], make_float2(all, all))), s[i]);
    part.store(p.dx + row * p.dx_stride * kBytes, s);
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
  for (int e = 0; e < 8; ++e) {
    if (part.has(Part::piece_of(e))) {
      const int col = part.column(Part::piece_of(e)) + e % Part::kPiece;
      to[col] = e % 2 ? dw[e / 2].y : dw[e / 2].x;
      to[p.width + col] = e % 2 ? db[e / 2].y : db[e / 2].x;
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

// Rows too wide for registers: the rows' gradient by reading twice, the columns' sums by another pass.
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
  group.add2(along, all);
  along /= (float)p.width;
  all /= (float)p.width;
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

// The CTAs' sums joined, in an order that the sizes fix: 32 columns to a CTA, the partial sums dealt out to its warps.
constexpr int kJoinWarps = 32;
__global__ void __launch_bounds__(kJoinWarps * 32) join_grad_kernel(const float* partial, int parts, int width, void* dw, void* db, int type,
                                                                   int accumulate) {
  __shared__ float sum[kJoinWarps][2][32];
  wait_for_previous_launch();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int col = blockIdx.x * 32 + lane;
  float a = 0.0f, b = 0.0f;
  if (col < width) {
#pragma unroll 4
    for (int i = warp; i < parts; i += kJoinWarps) {
      const float* part = partial + (size_t)i * 2 * width;
      a += part[col];
      b += part[width + col];
    }
  }
  sum[warp][0][lane] = a;
  sum[warp][1][lane] = b;
  __syncthreads();
  if (warp >= 2 || col >= width) return;
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < kJoinWarps; ++i) s += sum[i][warp][lane];
  void* to = warp == 0 ? dw : db;
  if (!to) return;
  store_one_of(to, type, col, accumulate ? load_one_of(to, type, col) + s : s);
}

// CTAs of the gradient, and so partial sums: as many as are on the device's SMs at a time, at most one to the rows of its groups.
struct GradShape {
  int warps, groups, threads, most, per_sm;                // most: threads of an SM that there are registers for
};
GradShape grad_shape(int width) {
  GradShape g;
  g.warps = (width + 255) / 256;
  g.groups = std::max(1, kGradWarps / g.warps);
  g.threads = g.warps * g.groups * 32;
  g.most = g.warps <= kGradWarps ? 2 * kGradWarps * 32 : 1024;
  g.per_sm = g.most / g.threads;
  return g;
}
int grad_parts(long long rows, int width) {
  if (width > kGradGroupWidth) return (int)std::min<long long>(rows, std::max(1, 4 * kSms * 256 / width));
  const GradShape g = grad_shape(width);
  return (int)std::min<long long>((rows + g.groups - 1) / g.groups, g.per_sm * kSms);
}

template <int TY, bool VEC>
bool launch_grad(const GradParams& p, int parts, cudaStream_t st) {
  const GradShape g = grad_shape(p.width);
  const int bytes = RowPart<TY, 1, VEC>::slot_bytes(p.width) * (p.ds ? 3 : 2) * g.groups;
  const Residents r = residents(g.threads, g.most, bytes);       // (at least two stages: 3 x 32 KB at the most)
  const size_t smem = std::max((size_t)r.stages * bytes, g.groups == 1 ? 0 : (size_t)g.groups * 2 * p.width * sizeof(float));
  const auto kernel = g.warps <= kGradWarps ? row_grad_kernel<TY, VEC, kGradWarps * 32> : row_grad_kernel<TY, VEC, 1024>;
  return allow_ring(kernel, smem) && launch(kernel, parts, g.threads, smem, 0, st, p, g.warps, r.stages);
}

template <int TY>
bool enqueue_grad_of(const GradParams& p, int parts, bool vec, cudaStream_t st) {
  if (p.width <= kGradGroupWidth) return vec ? launch_grad<TY, true>(p, parts, st) : launch_grad<TY, false>(p, parts, st);
  if (!launch(wide_row_grad_kernel<TY>, p.rows, kWideThreads, 0, 0, st, p)) return false;
  return !p.partial || launch(wide_column_grad_kernel<TY>, (long long)(p.width + 255) / 256 * parts, 256, 0, 0, st, p, parts);
}

// ---------------------------------------------------------------- columns in 8 bits

// The largest values of 256 columns over a chunk of rows, then the transposed bytes: the second pass finds in L2 what the
// first has read, as long as it is not larger than that.
constexpr int kColThreads = 256;
constexpr int kColMaxChunks = 64;
constexpr int kTileRows = 128, kTileCols = 64;

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
#pragma unroll 4
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
__global__ void __launch_bounds__(kColThreads) column_bytes_kernel(const __grid_constant__ ColumnParams p, int row_tiles) {
  __shared__ float per[kTileCols];
  __shared__ __align__(16) uint32_t tile[kTileCols][kTileRows / 4 + 4];     // a column's bytes, rows 16 apart in banks
  wait_for_previous_launch();
  constexpr int kBytes = TY == QADAM_F32 ? 4 : 2;
  const long long first = (long long)(blockIdx.x / row_tiles) * kTileCols;
  const long long top = (long long)(blockIdx.x % row_tiles) * kTileRows;
  // a warp has 4 rows at a time in each of 4 groups of eight lanes; a lane 8 columns
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int quad = warp * 4 + lane / 8;                                      // 32 groups of 4 rows
  const int c0 = VEC ? lane % 8 * 8 : lane % 8;
  float v[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const long long row = top + quad * 4 + i;
    const char* x = p.x + row * p.stride * kBytes;
    if constexpr (VEC) {
      Raw8<TY> raw = {};
      if (row < p.rows && first + c0 < p.width) raw = load_raw8<TY>(x + (first + c0) * kBytes);
      raw8_to_floats<TY>(raw, v[i]);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[i][k] = row < p.rows && first + c0 + 8 * k < p.width ? load_one<TY>(x, first + c0 + 8 * k) : 0.0f;
    }
  }
  if (threadIdx.x < kTileCols && first + threadIdx.x < p.width) {
    uint32_t m = 0u;
    for (int i = 0; i < p.chunks; ++i) m = max(m, p.largest[(size_t)i * p.width + first + threadIdx.x]);
    const ByteScale s = byte_scale(m);
    per[threadIdx.x] = s.per;
    if (top == 0) p.scale[first + threadIdx.x] = s.worth;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int c = VEC ? c0 + k : c0 + 8 * k;
    if (first + c < p.width) {
      const float f = per[c];
      tile[c][quad] = four_bytes(to_byte(v[0][k], f), to_byte(v[1][k], f), to_byte(v[2][k], f), to_byte(v[3][k], f));
    }
  }
  __syncthreads();
  // 16 rows' bytes of a column at a time; columns of the result have room up to a multiple of 16
  for (int i = threadIdx.x; i < kTileCols * (kTileRows / 16); i += kColThreads) {
    const int c = i / (kTileRows / 16), part = i % (kTileRows / 16);
    const long long row = top + part * 16;
    if (first + c < p.width && row < p.rows)
      *reinterpret_cast<uint4*>(p.q + (first + c) * p.q_stride + row) = *reinterpret_cast<const uint4*>(&tile[c][part * 4]);
  }
}

int column_chunks(long long rows, long long width) {
  const long long strips = (width + 255) / 256;
  return (int)std::max<long long>(1, std::min<long long>({(long long)kColMaxChunks, rows / 32, 4 * kSms / strips}));
}

template <int TY, bool VEC>
bool launch_columns(const ColumnParams& p, cudaStream_t st) {
  const long long strips = (p.width + 255) / 256, tiles = (p.width + kTileCols - 1) / kTileCols;
  const int row_tiles = (int)((p.rows + kTileRows - 1) / kTileRows);
  return launch(column_max_kernel<TY, VEC>, strips * p.chunks, kColThreads, 0, 0, st, p) &&
         launch(column_bytes_kernel<TY, VEC>, tiles * row_tiles, kColThreads, 0, 0, st, p, row_tiles);
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

// A thread decodes 16 consecutive codes: (16 BITS + 31) / 32 + 1 words at most, one store of 16 bytes.
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
bool on16(const void* p, int64_t stride, int type) { return is_aligned(p, 16) && stride * type_bytes(type) % 16 == 0; }

}  // namespace

extern "C" {

int qadam_layer_norm(const void* x, int32_t type, int64_t x_stride, const void* residual, int64_t residual_stride, const void* weight,
                     int32_t weight_type, const void* bias, int32_t bias_type, int64_t rows, int64_t width, float eps, void* sum,
                     int64_t sum_stride, void* out, int64_t out_stride, float* mean, float* rstd, int8_t* q, int64_t q_stride,
                     float* scale, int32_t* sums, void* stream) {
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
  p.w = weight; p.w_type = weight_type; p.w_vec = is_aligned(weight, 16);
  p.b = bias; p.b_type = bias_type; p.b_vec = is_aligned(bias, 16);
  p.sum = static_cast<char*>(sum); p.sum_stride = sum_stride;
  p.out = static_cast<char*>(out); p.out_stride = out_stride;
  p.mean = mean; p.rstd = rstd;
  p.q = reinterpret_cast<signed char*>(q); p.q_stride = q_stride; p.scale = scale; p.sums = sums;
  p.rows = rows; p.width = (int)width; p.normed = 1; p.eps = eps;
  const bool vec = whole(width, type) && on16(x, x_stride, type) && (!residual || (on16(residual, residual_stride, type) && on16(sum, sum_stride, type))) &&
                   (!out || on16(out, out_stride, type));
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
  p.w = columns; p.w_type = QADAM_F32; p.w_vec = is_aligned(columns, 16);
  p.q = reinterpret_cast<signed char*>(q); p.q_stride = q_stride; p.scale = scale; p.sums = sums;
  p.rows = rows; p.width = (int)width;
  return enqueue_rows(p, type, whole(width, type) && on16(x, x_stride, type), static_cast<cudaStream_t>(stream));
}

int qadam_layer_norm_grad_query_sizes(int64_t rows, int64_t width, size_t* workspace_bytes) {
  if (bad_rows(rows, width)) return QADAM_ERR_SIZE;
  if (workspace_bytes) *workspace_bytes = round_up256((size_t)grad_parts(rows, (int)width) * 2 * (size_t)width * sizeof(float));
  return QADAM_OK;
}

int qadam_layer_norm_grad(const void* dy, int32_t type, int64_t dy_stride, const void* x, int64_t x_stride, const float* mean,
                          const float* rstd, const void* weight, int32_t weight_type, const void* dsum, int64_t dsum_stride,
                          int64_t rows, int64_t width, void* dx, int64_t dx_stride, void* dweight, void* dbias, int32_t grad_type,
                          int32_t accumulate, void* workspace, size_t workspace_bytes, void* stream) {
  if (bad_rows(rows, width)) return QADAM_ERR_SIZE;
  const bool sums = dweight || dbias;
  if (!known_type(type) || (weight && !known_type(weight_type)) || (sums && !known_type(grad_type))) return QADAM_ERR_TYPE;
  const int parts = grad_parts(rows, (int)width);
  if ((rows > 0 && (!dy || !x || !mean || !rstd || !dx)) || (sums && parts > 0 && !workspace)) return QADAM_ERR_NULL;
  if (bad_stride(dy_stride, width) || bad_stride(x_stride, width) || bad_stride(dx_stride, width) || (dsum && bad_stride(dsum_stride, width)))
    return QADAM_ERR_SIZE;
  if (accumulate != 0 && accumulate != 1) return QADAM_ERR_SIZE;
  const size_t e = type_bytes(type);
  if (!is_aligned(dy, e) || !is_aligned(x, e) || !is_aligned(dsum, e) || !is_aligned(dx, e) || !is_aligned(mean, 4) || !is_aligned(rstd, 4) ||
      (weight && !is_aligned(weight, type_bytes(weight_type))) ||
      (sums && (!is_aligned(dweight, type_bytes(grad_type)) || !is_aligned(dbias, type_bytes(grad_type)) || !is_aligned(workspace, 256))))
    return QADAM_ERR_ALIGN;
  if (sums && workspace_bytes < (size_t)parts * 2 * (size_t)width * sizeof(float)) return QADAM_ERR_WORKSPACE;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (rows > 0) {
    GradParams p = {};
    p.dy = static_cast<const char*>(dy); p.dy_stride = dy_stride;
    p.x = static_cast<const char*>(x); p.x_stride = x_stride;
    p.ds = static_cast<const char*>(dsum); p.ds_stride = dsum_stride;
    p.dx = static_cast<char*>(dx); p.dx_stride = dx_stride;
    p.mean = mean; p.rstd = rstd;
    p.w = weight; p.w_type = weight_type; p.w_vec = is_aligned(weight, 16);
    p.partial = sums ? static_cast<float*>(workspace) : nullptr;
    p.rows = rows; p.width = (int)width;
    const bool vec = whole(width, type) && on16(dy, dy_stride, type) && on16(x, x_stride, type) && on16(dx, dx_stride, type) &&
                     (!dsum || on16(dsum, dsum_stride, type));
    const bool ok = type == QADAM_F32 ? enqueue_grad_of<QADAM_F32>(p, parts, vec, st)
                    : type == QADAM_BF16 ? enqueue_grad_of<QADAM_BF16>(p, parts, vec, st) : enqueue_grad_of<QADAM_F16>(p, parts, vec, st);
    if (!ok) return QADAM_ERR_CUDA;
  }
  if (sums && (rows > 0 || !accumulate)) {
    if (!launch(join_grad_kernel, (width + 31) / 32, kJoinWarps * 32, 0, 0, st, static_cast<const float*>(workspace), parts, (int)width, dweight, dbias,
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
