// The norm of many tensors and the factor that clips it: qadam_norm_*.
//
//   norm = sqrt(sum x^2),   factor = min(1, max_norm / norm)
//
// One read of the tensors: bound by HBM, as long as an element costs few instructions.  The squares of what a thread has
// in 16 bytes are added in binary32 (4 products and sums, or 8 exact products of 16-bit numbers: the sum of squares
// is off by at most 7 x 2^-24, the norm by half of that), everything else in binary64: with squares in binary64 this
// kernel takes 53 us in place of 37 for 109.5 x 10^6 bf16 (5.9 TB/s) and 33.8 in place of 32.7 for 47 x 10^6 fp32.  Squares that
// binary32 does not hold, of numbers below 1e-12 or above 1e19, are seen by their sum, and formed in binary64.  A short list
// is bound by what does not depend on its length: 1000 elements take 3.6 us, 10^6 5.1, 11.7 x 10^6 12.0, and every further 10^6
// 0.59 (6.8 TB/s).
#include "qadam.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "qadam_tensors.cuh"

using namespace qadam;

namespace {

constexpr int kNormThreads = 256;
constexpr int kNormLoads = 4;              // of 16 bytes, that a thread has under way
constexpr int kNormCtasPerSm = 4;
constexpr int kNormMaxCtas = 2048;         // partial sums there is room for

inline int norm_tile(int type) { return kNormThreads * kNormLoads * (16 / type_bytes(type)); }     // elements a CTA takes at a time

struct __align__(16) NormTile {
  long long begin;             // inside the tensor
  int left;                    // elements of the tensor from there on, no more than a tile
  int seg;
  int type;
  int reserved[3];
};

struct NormParams {
  const NormTile* tiles;
  int first, last;             // tiles of this launch
  int tensor_base;             // tensor of the first pointer
  double* partial;             // [kNormMaxCtas]
  unsigned* arrived;           // CTAs that have stored their partial; 0 between launches
  int slot;                    // first slot of this launch's partials
  int total;                   // partials of all launches of this run, or 0: this launch is not the last
  float max_norm;
  float* out;
};

// 16 bytes of a tensor, as they lie in memory; elements behind the last are zero.
__device__ __forceinline__ uint4 load16(const char* p, int type, int i, int left, bool aligned) {
  const int n = type == QADAM_F32 ? 4 : 8;
  if (aligned && i + n <= left) return *reinterpret_cast<const uint4*>(p + (size_t)i * (16 / n));
  uint32_t w[4] = {0u, 0u, 0u, 0u};
  if (type == QADAM_F32) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k < left) w[k] = reinterpret_cast<const uint32_t*>(p)[i + k];
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (i + k < left) w[k / 2] |= (uint32_t) reinterpret_cast<const unsigned short*>(p)[i + k] << (16 * (k % 2));
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int N>
__device__ __forceinline__ void add_squares(const float (&x)[N], double& sum) {
  float s = __fmul_rn(x[0], x[0]);
#pragma unroll
  for (int k = 1; k < N; ++k) s = fmaf(x[k], x[k], s);
  if (s >= 8.271806125530277e-25f && s <= 8.507059173023462e37f) {        // 2^-80, 2^126
    sum += (double)s;
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (x[k] != 0.0f) sum = fma((double)x[k], (double)x[k], sum);       // (a NaN is not 0 either)
  }
}

__device__ __forceinline__ void add_squares16(const uint4& r, int type, double& sum) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
  if (type == QADAM_F32) {
    const float x[4] = {__uint_as_float(w[0]), __uint_as_float(w[1]), __uint_as_float(w[2]), __uint_as_float(w[3])};
    add_squares<4>(x, sum);
    return;
  }
  float x[8];
  if (type == QADAM_BF16) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[2 * k] = __uint_as_float(w[k] << 16);
      x[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
    }
    add_squares<8>(x, sum);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[2 * k] = half_bits_to_float(w[k] & 0xFFFFu);
      x[2 * k + 1] = half_bits_to_float(w[k] >> 16);
    }
    add_squares<8>(x, sum);
  }
}

__device__ __forceinline__ double warp_sum(double s) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  return s;
}

// Sum over the CTA, in thread 0.
__device__ __forceinline__ double block_sum(double s, double* shared) {
  s = warp_sum(s);
  if (threadIdx.x % 32 == 0) shared[threadIdx.x / 32] = s;
  __syncthreads();
  s = 0.0;
  if (threadIdx.x < 32) {
    s = threadIdx.x < kNormThreads / 32 ? shared[threadIdx.x] : 0.0;
    s = warp_sum(s);
  }
  return s;
}

template <int CAP>
__global__ void __launch_bounds__(kNormThreads, kNormCtasPerSm) norm_kernel(const __grid_constant__ NormParams p,
                                                                            const __grid_constant__ Pointers<CAP> ptrs) {
  wait_for_previous_launch();
  __shared__ double shared[kNormThreads / 32];
  __shared__ bool last;
  double sum = 0.0;
  // the next tile's loads are under way while this one's squares are formed
  uint4 raw[2][kNormLoads];
  auto ask = [&](const NormTile& tile, uint4 (&to)[kNormLoads]) {
    const char* src = static_cast<const char*>(ptrs.at[tile.seg - p.tensor_base]);
    const int left = src != nullptr ? tile.left : 0, n = 16 / type_bytes(tile.type);
    src += tile.begin * type_bytes(tile.type);
    const bool aligned = (reinterpret_cast<uintptr_t>(src) & 15u) == 0;
#pragma unroll
    for (int k = 0; k < kNormLoads; ++k) {
      const int i = n * (threadIdx.x + k * kNormThreads);
      to[k] = make_uint4(0u, 0u, 0u, 0u);
      if (i < left) to[k] = load16(src, tile.type, i, left, aligned);
    }
  };
  const int step = gridDim.x;
  int t = p.first + blockIdx.x;
  int type[2];
  NormTile tile = p.tiles[t];
  type[0] = tile.type;
  ask(tile, raw[0]);
  if (t + step < p.last) tile = p.tiles[t + step];
  for (; t < p.last; t += 2 * step) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int now = t + h * step;
      if (now >= p.last) break;
      if (now + step < p.last) {
        type[h ^ 1] = tile.type;
        ask(tile, raw[h ^ 1]);
        if (now + 2 * step < p.last) tile = p.tiles[now + 2 * step];
      }
      if (type[h] == QADAM_F32) {
#pragma unroll
        for (int k = 0; k < kNormLoads; ++k) add_squares16(raw[h][k], QADAM_F32, sum);
      } else if (type[h] == QADAM_BF16) {
#pragma unroll
        for (int k = 0; k < kNormLoads; ++k) add_squares16(raw[h][k], QADAM_BF16, sum);
      } else {
#pragma unroll
        for (int k = 0; k < kNormLoads; ++k) add_squares16(raw[h][k], QADAM_F16, sum);
      }
    }
  }
  sum = block_sum(sum, shared);
  if (threadIdx.x == 0) {
    p.partial[p.slot + blockIdx.x] = sum;
    __threadfence();
    // counts up to the last CTA of the launch and begins again at 0
    last = atomicInc(p.arrived, gridDim.x - 1) == gridDim.x - 1 && p.total > 0;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  sum = 0.0;
  for (int i = threadIdx.x; i < p.total; i += kNormThreads) sum += __ldcg(p.partial + i);
  sum = block_sum(sum, shared);
  if (threadIdx.x == 0) {
    const float norm = (float)sqrt(sum);
    float factor = norm > p.max_norm ? __fdiv_rn(p.max_norm, norm) : 1.0f;
    if (!(norm <= 3.402823466e38f)) factor = __int_as_float(0x7FC00000);
    p.out[0] = norm;
    p.out[1] = factor;
  }
}

__global__ void norm_of_nothing_kernel(float* out) {
  wait_for_previous_launch();
  out[0] = 0.0f;
  out[1] = 1.0f;
}

struct NormGeometry {
  std::vector<NormTile> tiles;
  std::vector<int> first_tile, type;         // [num_tensors]
  size_t off_partial = 0, off_arrived = 0, workspace_bytes = 0;
};

int norm_geometry(const qadam_tensor_list* l, NormGeometry* g) {
  if (!l) return QADAM_ERR_NULL;
  if (l->num_tensors < 1 || l->num_tensors > (1 << 20) || l->reserved != 0) return QADAM_ERR_SIZE;
  if (!l->len) return QADAM_ERR_NULL;
  int64_t tiles = 0;
  for (int s = 0; s < l->num_tensors; ++s) {
    if (l->type && !known_type(l->type[s])) return QADAM_ERR_TYPE;
    if (l->len[s] < 0 || l->len[s] > (int64_t)1 << 40) return QADAM_ERR_SIZE;
    const int64_t tile = norm_tile(l->type ? l->type[s] : QADAM_F32);
    tiles += (l->len[s] + tile - 1) / tile;
    if (tiles > (int64_t)1 << 30) return QADAM_ERR_SIZE;
  }
  g->first_tile.resize(l->num_tensors);
  g->type.resize(l->num_tensors);
  g->tiles.reserve((size_t)tiles);
  for (int s = 0; s < l->num_tensors; ++s) {
    g->type[s] = l->type ? l->type[s] : QADAM_F32;
    g->first_tile[s] = (int)g->tiles.size();
    const int64_t tile = norm_tile(g->type[s]);
    for (int64_t o = 0; o < l->len[s]; o += tile)
      g->tiles.push_back(NormTile{(long long)o, (int)std::min<int64_t>(tile, l->len[s] - o), s, g->type[s], {0, 0, 0}});
  }
  size_t wo = round_up256(g->tiles.size() * sizeof(NormTile));
  g->off_partial = wo;
  wo += round_up256(kNormMaxCtas * sizeof(double));
  g->off_arrived = wo;
  wo += 256;
  g->workspace_bytes = wo;
  return QADAM_OK;
}

}  // namespace

struct qadam_norm {
  NormGeometry geo;
  std::vector<const void*> ptrs;
  unsigned char* workspace = nullptr;
  int device = 0, sm_count = 0;
  bool bound = false;
  int64_t launches = 0;
};

namespace {

template <int CAP>
int launch_norm(qadam_norm* c, NormParams p, int grid, int tensors, cudaStream_t st) {
  static_assert(sizeof(Pointers<CAP>) + sizeof(NormParams) <= 32764, "kernel parameters");
  Pointers<CAP> ptrs;
  std::copy(c->ptrs.begin() + p.tensor_base, c->ptrs.begin() + p.tensor_base + tensors, ptrs.at);
  if (!launch(norm_kernel<CAP>, grid, kNormThreads, 0, 0, st, p, ptrs)) return QADAM_ERR_CUDA;
  c->launches += 1;
  return QADAM_OK;
}

}  // namespace

extern "C" {

int qadam_norm_query_sizes(const qadam_tensor_list* list, size_t* workspace_bytes) try {
  NormGeometry g;
  const int rc = norm_geometry(list, &g);
  if (rc == QADAM_OK && workspace_bytes) *workspace_bytes = g.workspace_bytes;
  return rc;
} catch (const std::bad_alloc&) {
  return QADAM_ERR_SIZE;
}

int qadam_norm_create(const qadam_tensor_list* list, void* workspace, size_t workspace_bytes, qadam_norm** out) try {
  if (!out) return QADAM_ERR_NULL;
  *out = nullptr;
  NormGeometry g;
  const int rc = norm_geometry(list, &g);
  if (rc != QADAM_OK) return rc;
  if (!workspace) return QADAM_ERR_NULL;
  if (!is_aligned(workspace, 256)) return QADAM_ERR_ALIGN;
  if (workspace_bytes < g.workspace_bytes) return QADAM_ERR_WORKSPACE;
  int device = 0, sms = 0;
  if (!cuda_call(cudaGetDevice(&device)) ||
      !cuda_call(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device)))
    return QADAM_ERR_CUDA;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  if (!g.tiles.empty() &&
      !cuda_call(cudaMemcpy(ws, g.tiles.data(), g.tiles.size() * sizeof(NormTile), cudaMemcpyHostToDevice)))
    return QADAM_ERR_CUDA;
  if (!cuda_call(cudaMemset(ws + g.off_arrived, 0, sizeof(unsigned))) || !cuda_call(cudaStreamSynchronize(nullptr)))
    return QADAM_ERR_CUDA;
  qadam_norm* c = new qadam_norm;
  c->geo = std::move(g);
  c->workspace = ws;
  c->device = device;
  c->sm_count = sms;
  *out = c;
  return QADAM_OK;
} catch (const std::bad_alloc&) {
  return QADAM_ERR_SIZE;
}

int qadam_norm_bind(qadam_norm* c, const void* const* tensors) try {
  if (!c || !tensors) return QADAM_ERR_NULL;
  for (size_t s = 0; s < c->geo.type.size(); ++s)
    if (!is_aligned(tensors[s], type_bytes(c->geo.type[s]))) return QADAM_ERR_ALIGN;
  c->ptrs.assign(tensors, tensors + c->geo.type.size());
  c->bound = true;
  return QADAM_OK;
} catch (const std::bad_alloc&) {
  return QADAM_ERR_SIZE;
}

int qadam_norm_run(qadam_norm* c, float max_norm, float* out, void* stream) {
  if (!c || !out || !c->bound) return QADAM_ERR_NULL;
  if (!(max_norm > 0.0f)) return QADAM_ERR_HYPER;
  if (!is_aligned(out, 8)) return QADAM_ERR_ALIGN;
  const OnDevice on(c->device);
  if (!on.ok()) return QADAM_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int tensors = (int)c->geo.type.size(), tiles = (int)c->geo.tiles.size();
  if (tiles == 0) {
    if (!launch(norm_of_nothing_kernel, 1, 1, 0, 0, st, out)) return QADAM_ERR_CUDA;
    c->launches += 1;
    return QADAM_OK;
  }
  // Lists of more tensors than one launch has pointers for: every launch leaves its partial sums in slots
  // of its own and the last one adds all of them up.
  const int runs = (tensors + kManyPointers - 1) / kManyPointers;
  const int most = std::max(1, std::min(c->sm_count * kNormCtasPerSm, kNormMaxCtas / runs));
  NormParams p;
  p.tiles = reinterpret_cast<const NormTile*>(c->workspace);
  p.partial = reinterpret_cast<double*>(c->workspace + c->geo.off_partial);
  p.arrived = reinterpret_cast<unsigned*>(c->workspace + c->geo.off_arrived);
  p.max_norm = max_norm;
  p.out = out;
  p.slot = 0;
  for (int s = 0; s < tensors; s += kManyPointers) {
    const int count = std::min(kManyPointers, tensors - s);
    p.tensor_base = s;
    p.first = c->geo.first_tile[s];
    p.last = s + count < tensors ? c->geo.first_tile[s + count] : tiles;
    const bool last = p.last == tiles;            // (what follows, if anything, is empty tensors)
    if (p.first == p.last) continue;
    const int grid = std::min(most, p.last - p.first);
    p.total = last ? p.slot + grid : 0;
    const int rc = count <= kFewPointers ? launch_norm<kFewPointers>(c, p, grid, count, st)
                                         : launch_norm<kManyPointers>(c, p, grid, count, st);
    if (rc != QADAM_OK) return rc;
    p.slot += grid;
    if (last) break;
  }
  return QADAM_OK;
}

int64_t qadam_norm_launch_count(const qadam_norm* c) { return c ? c->launches : QADAM_ERR_NULL; }

int qadam_norm_destroy(qadam_norm* c) {
  if (!c) return QADAM_ERR_NULL;
  delete c;
  return QADAM_OK;
}

}  // extern "C"
