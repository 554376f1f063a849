// The norm of many tensors and the factor that clips it: qadam_norm_*.
//
//   norm = sqrt(sum x^2),   factor = min(1, max_norm / norm)
//
// One read of the tensors: bound by HBM.  Squares and sums are binary64: 2^26 binary32 squares summed
// in binary32 are off in the third digit, and a square of a binary32 number below 1e-19 or above
// 1e19 does not exist in binary32.
#include "qadam.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "qadam_tensors.cuh"

using namespace qadam;

namespace {

constexpr int kNormThreads = 256;
constexpr int kNormTile = 8192;            // elements a CTA takes at a time
constexpr int kNormCtasPerSm = 8;
constexpr int kNormMaxCtas = 2048;         // partial sums there is room for

struct NormTensor {
  long long len;
  int type;
  int first_tile;
};

struct NormParams {
  const Tile* tiles;              // runs of at most kNormTile elements: offset inside the tensor, count, tensor
  int first, last;                // tiles of this launch
  const NormTensor* tensors;
  int tensor_base;                // tensor of the first pointer
  double* partial;                // [kNormMaxCtas]
  unsigned* arrived;              // CTAs that have stored their partial; 0 between launches
  int slot;                       // first slot of this launch's partials
  int total;                      // partials of all launches of this run, or 0: this launch is not the last
  float max_norm;
  float* out;
};

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
__global__ void __launch_bounds__(kNormThreads) norm_kernel(const __grid_constant__ NormParams p,
                                                            const __grid_constant__ Pointers<CAP> ptrs) {
  __shared__ double shared[kNormThreads / 32];
  __shared__ bool last;
  double sum = 0.0;
  for (int t = p.first + blockIdx.x; t < p.last; t += gridDim.x) {
    const Tile tile = p.tiles[t];
    const void* src = ptrs.at[tile.seg - p.tensor_base];
    if (src == nullptr) continue;
    const NormTensor info = p.tensors[tile.seg];
    const bool fits = aligned4(src, info.type);
    constexpr int kQuads = kNormTile / (4 * kNormThreads);
    Raw4 raw[kQuads];
#pragma unroll
    for (int k = 0; k < kQuads; ++k) {
      const long long i = tile.off + 4 * (threadIdx.x + k * kNormThreads);
      if (i < info.len) raw[k] = load_raw4(src, info.type, i, info.len, fits && i + 4 <= info.len);
      else raw[k] = {{0u, 0u, 0u, 0u}};
    }
#pragma unroll
    for (int k = 0; k < kQuads; ++k) {
      float x[4];
      to_floats(raw[k], info.type, x);
#pragma unroll
      for (int j = 0; j < 4; ++j) sum = fma((double)x[j], (double)x[j], sum);
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
  out[0] = 0.0f;
  out[1] = 1.0f;
}

struct NormGeometry {
  std::vector<NormTensor> tensors;
  std::vector<Tile> tiles;
  size_t off_tensors = 0, off_partial = 0, off_arrived = 0, workspace_bytes = 0;
};

int norm_geometry(const qadam_tensor_list* l, NormGeometry* g) {
  if (!l) return QADAM_ERR_NULL;
  if (l->num_tensors < 1 || l->num_tensors > (1 << 20) || l->reserved != 0) return QADAM_ERR_SIZE;
  if (!l->len) return QADAM_ERR_NULL;
  int64_t tiles = 0;
  for (int s = 0; s < l->num_tensors; ++s) {
    if (l->type && !known_type(l->type[s])) return QADAM_ERR_TYPE;
    if (l->len[s] < 0 || l->len[s] > (int64_t)1 << 40) return QADAM_ERR_SIZE;
    tiles += (l->len[s] + kNormTile - 1) / kNormTile;
    if (tiles > (int64_t)1 << 30) return QADAM_ERR_SIZE;
  }
  g->tensors.resize(l->num_tensors);
  g->tiles.reserve((size_t)tiles);
  for (int s = 0; s < l->num_tensors; ++s) {
    g->tensors[s] = NormTensor{(long long)l->len[s], l->type ? l->type[s] : QADAM_F32, (int)g->tiles.size()};
    for (int64_t o = 0; o < l->len[s]; o += kNormTile)
      g->tiles.push_back(Tile{(long long)o, (int)std::min<int64_t>(kNormTile, l->len[s] - o), s});
  }
  size_t wo = round_up256(g->tiles.size() * sizeof(Tile));
  g->off_tensors = wo;
  wo += round_up256(g->tensors.size() * sizeof(NormTensor));
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
  norm_kernel<CAP><<<grid, kNormThreads, 0, st>>>(p, ptrs);
  if (!cuda_call(cudaGetLastError())) return QADAM_ERR_CUDA;
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
      !cuda_call(cudaMemcpy(ws, g.tiles.data(), g.tiles.size() * sizeof(Tile), cudaMemcpyHostToDevice)))
    return QADAM_ERR_CUDA;
  if (!cuda_call(cudaMemcpy(ws + g.off_tensors, g.tensors.data(), g.tensors.size() * sizeof(NormTensor), cudaMemcpyHostToDevice)) ||
      !cuda_call(cudaMemset(ws + g.off_arrived, 0, sizeof(unsigned))) || !cuda_call(cudaStreamSynchronize(nullptr)))
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
  for (size_t s = 0; s < c->geo.tensors.size(); ++s)
    if (!is_aligned(tensors[s], type_bytes(c->geo.tensors[s].type))) return QADAM_ERR_ALIGN;
  c->ptrs.assign(tensors, tensors + c->geo.tensors.size());
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
  const int tensors = (int)c->geo.tensors.size(), tiles = (int)c->geo.tiles.size();
  if (tiles == 0) {
    norm_of_nothing_kernel<<<1, 1, 0, st>>>(out);
    if (!cuda_call(cudaGetLastError())) return QADAM_ERR_CUDA;
    c->launches += 1;
    return QADAM_OK;
  }
  // Lists of more tensors than one launch has pointers for: every launch leaves its partial sums in slots
  // of its own and the last one adds all of them up.
  const int runs = (tensors + kManyPointers - 1) / kManyPointers;
  const int most = std::max(1, std::min(c->sm_count * kNormCtasPerSm, kNormMaxCtas / runs));
  NormParams p;
  p.tiles = reinterpret_cast<const Tile*>(c->workspace);
  p.tensors = reinterpret_cast<const NormTensor*>(c->workspace + c->geo.off_tensors);
  p.partial = reinterpret_cast<double*>(c->workspace + c->geo.off_partial);
  p.arrived = reinterpret_cast<unsigned*>(c->workspace + c->geo.off_arrived);
  p.max_norm = max_norm;
  p.out = out;
  p.slot = 0;
  for (int s = 0; s < tensors; s += kManyPointers) {
    const int count = std::min(kManyPointers, tensors - s);
    p.tensor_base = s;
    p.first = c->geo.tensors[s].first_tile;
    p.last = s + count < tensors ? c->geo.tensors[s + count].first_tile : tiles;
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
