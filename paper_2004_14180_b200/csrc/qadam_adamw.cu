// AdamW over many tensors at once, moments in 32 or in 8 bits: qadam_adamw_*.
//
//   m = b1 m + c1 g',  v = b2 v + c2 g'^2,  x = x k - a (m / (sqrt(v) b + eps))
//
// One read of gradient, weight and moments, one write of weight and moments, 15 operations an
// element: bound by HBM with 32-bit moments.  One launch for all tensors of all types.
#include "qadam.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "qadam_tensors.cuh"

using namespace qadam;

namespace {

constexpr int kAdamThreads = 256;
constexpr int kAdamCtas = 4;                                   // at least so many per SM
constexpr int kPair = 256;                                     // elements of two rows: what a warp takes at a time
constexpr int kAdamTile = kAdamThreads / 32 * kPair;           // 2048 elements per CTA
constexpr unsigned kLeastScale = 0x00800000u;                  // 2^-126

struct AdamTensor {
  void* w;
  long long off, len;          // padded layout
  float decay;
  int wtype, gtype;
  int first_tile;
};

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
  const Tile* tiles;           // runs of at most kAdamTile elements: offset inside the tensor, count, tensor
  const AdamTensor* tensors;
  int first;                   // tile of the first CTA
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
  __device__ __forceinline__ static unsigned of(float y, unsigned add, int least, int k) {
    const int c = max((int)(__float_as_uint(y) + add - kBase), least);
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

template <bool EIGHT, int CAP>
__global__ void __launch_bounds__(kAdamThreads, kAdamCtas) adamw_kernel(const __grid_constant__ AdamParams p,
                                                             const __grid_constant__ Pointers<CAP> grads) {
  const Tile tile = p.tiles[p.first + blockIdx.x];
  const void* g = grads.at[tile.seg - p.tensor_base];
  if (g == nullptr) return;
  float c = 1.0f;
  if (p.grad_scale != nullptr) {
    c = *p.grad_scale;
    if (!finite(c)) {
      if (threadIdx.x == 0) atomicOr(p.status, QADAM_ST_NONFINITE);
      return;
    }
  }
  const AdamTensor T = p.tensors[tile.seg];
  const int lane = threadIdx.x % 32;
  const long long begin = tile.off + threadIdx.x / 32 * kPair;          // of the warp's two rows, inside the tensor
  const long long i0 = begin + 4 * lane;
  const int rows = begin >= T.len ? 0 : begin + 128 >= T.len ? 1 : 2;
  if (rows == 0) return;
  const bool gfits = aligned4(g, T.gtype), wfits = aligned4(T.w, T.wtype);

  Raw4 rg[2], rx[2];
  float m[2][4], v[2][4];
  uint32_t cm[2], cr[2];
  float sm[2], sr[2];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    if (r >= rows) break;
    const long long i = i0 + 128 * r, at = T.off + i;
    rg[r] = load_raw4(g, T.gtype, i, T.len, gfits && i + 4 <= T.len);
    if (p.master != nullptr) rx[r] = load_raw4(p.master + T.off, QADAM_F32, i, T.len, true);
    else rx[r] = load_raw4(T.w, T.wtype, i, T.len, wfits && i + 4 <= T.len);
    if constexpr (EIGHT) {
      cm[r] = *reinterpret_cast<const uint32_t*>(static_cast<const unsigned char*>(p.m) + at);
      cr[r] = *reinterpret_cast<const uint32_t*>(static_cast<const unsigned char*>(p.v) + at);
      sm[r] = p.m_scale[at / 128];
      sr[r] = p.r_scale[at / 128];
    } else {
      const float4 a = *reinterpret_cast<const float4*>(static_cast<const float*>(p.m) + at);
      const float4 b = *reinterpret_cast<const float4*>(static_cast<const float*>(p.v) + at);
      m[r][0] = a.x; m[r][1] = a.y; m[r][2] = a.z; m[r][3] = a.w;
      v[r][0] = b.x; v[r][1] = b.y; v[r][2] = b.z; v[r][3] = b.w;
    }
  }
  const StepScalars now = p.counted != nullptr ? *p.counted : p.now;
  const float keep = (float)(1.0 - now.lr * (double)T.decay);
  uint4 coins = make_uint4(0u, 0u, 0u, 0u);
  if constexpr (EIGHT) {
    const unsigned long long quad = (unsigned long long)((T.off + begin) / 4 + lane);
    coins = philox(make_uint4((unsigned)quad, (unsigned)(quad >> 32), (unsigned)now.t, (unsigned)(now.t >> 32)), p.keys);
  }
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    if (r >= rows) break;
    const long long i = i0 + 128 * r, at = T.off + i;
    float gx[4], x[4], root[4];
    to_floats(rg[r], T.gtype, gx);
    to_floats(rx[r], p.master != nullptr ? (int)QADAM_F32 : T.wtype, x);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (EIGHT) {
        const float y = __fmul_rn(CodeM::value(cm[r], k), sm[r]);
        m[r][k] = __uint_as_float(__float_as_uint(y) | ((cm[r] << (24 - 8 * k)) & 0x80000000u));
        const float z = __fmul_rn(CodeR::value(cr[r], k), sr[r]);
        v[r][k] = __fmul_rn(z, z);
      }
      const float gc = __fmul_rn(gx[k], c);
      m[r][k] = __fadd_rn(__fmul_rn(p.beta1, m[r][k]), __fmul_rn(p.c1, gc));
      v[r][k] = __fadd_rn(__fmul_rn(p.beta2, v[r][k]), __fmul_rn(p.c2, __fmul_rn(gc, gc)));
      root[k] = __fsqrt_rn(v[r][k]);
      const float d = __fadd_rn(__fmul_rn(root[k], now.b), p.eps);
      x[k] = __fsub_rn(__fmul_rn(x[k], keep), __fmul_rn(now.a, __fdiv_rn(m[r][k], d)));
    }
    if (p.master != nullptr)
      *reinterpret_cast<float4*>(p.master + at) = make_float4(x[0], x[1], x[2], x[3]);
    store_raw4(T.w, T.wtype, i, T.len, wfits && i + 4 <= T.len, from_floats(x, T.wtype));
    if constexpr (EIGHT) {
      // the row's two scales, and one division for both: even lanes take m's, odd lanes r's
      const unsigned tm = __reduce_max_sync(0xFFFFFFFFu, largest4(m[r])), tr = __reduce_max_sync(0xFFFFFFFFu, largest4(root));
      const float mine = __uint_as_float(max((lane & 1) == 0 ? tm : tr, kLeastScale));
      const float inverse = __fdiv_rn(1.0f, mine);
      const float im = __shfl_sync(0xFFFFFFFFu, inverse, 0), ir = __shfl_sync(0xFFFFFFFFu, inverse, 1);
      uint32_t om = 0u, orr = 0u;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        // h: low half of a word for k = 0, 2, high half for 1, 3
        const unsigned word = r == 0 ? (k < 2 ? coins.x : coins.y) : (k < 2 ? coins.z : coins.w);
        const unsigned add_m = ((k % 2 == 0 ? word << 14 : word >> 2) & (63u << 14)) | (1u << 13);
        const unsigned add_r = ((k % 2 == 0 ? word << 3 : word >> 13) & (1023u << 9)) | (1u << 8);
        const unsigned sign = CodeM::shifted(__float_as_uint(m[r][k]), 8 * k - 24) & (128u << (8 * k));
        om |= CodeM::of(__fmul_rn(fabsf(m[r][k]), im), add_m, 0, k) | sign;
        orr |= CodeR::of(__fmul_rn(root[k], ir), add_r, root[k] > 0.0f ? 1 << CodeR::kDrop : 0, k);
      }
      // a row that is not finite: code 0 times its scale is a NaN
      if (!finite(__uint_as_float(tm))) om = 0u;
      if (!finite(__uint_as_float(tr))) orr = 0u;
      *reinterpret_cast<uint32_t*>(static_cast<unsigned char*>(p.m) + at) = om;
      *reinterpret_cast<uint32_t*>(static_cast<unsigned char*>(p.v) + at) = orr;
      if (lane < 2) {
        (lane == 0 ? p.m_scale : p.r_scale)[at / 128] = mine;
        if (!finite(mine)) atomicOr(p.status, QADAM_ST_NONFINITE);
      }
    } else {
      *reinterpret_cast<float4*>(static_cast<float*>(p.m) + at) = make_float4(m[r][0], m[r][1], m[r][2], m[r][3]);
      *reinterpret_cast<float4*>(static_cast<float*>(p.v) + at) = make_float4(v[r][0], v[r][1], v[r][2], v[r][3]);
    }
  }
}

// The scalars of the next step, from the device's own count and step size.
__global__ void adamw_count_kernel(StepScalars* now, long long* count, const float* lr, float lr_default, float beta1,
                                   float beta2, const float* grad_scale) {
  const long long t = *count + 1;
  if (grad_scale == nullptr || finite(*grad_scale)) *count = t;
  *now = step_scalars(lr != nullptr ? (double)*lr : (double)lr_default, beta1, beta2, t);
}

// 8-bit moments as the values they stand for, four elements to a thread.
__global__ void __launch_bounds__(kAdamThreads) adamw_moments_kernel(const uint32_t* m, const uint32_t* r, const float* m_scale,
                                                                     const float* r_scale, long long quads, float4* m32,
                                                                     float4* v32) {
  for (long long q = (long long)blockIdx.x * kAdamThreads + threadIdx.x; q < quads; q += (long long)gridDim.x * kAdamThreads) {
    float x[4];
    if (m32 != nullptr) {
      const uint32_t a = m[q];
      const float s = m_scale[q / 32];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float y = __fmul_rn(CodeM::value(a, k), s);
        x[k] = ((a >> (8 * k)) & 128u) != 0u ? -y : y;
      }
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
  std::vector<AdamTensor> tensors;
  std::vector<Tile> tiles;
  int64_t D = 0;
  size_t off_tensors = 0, off_now = 0, workspace_bytes = 0;
};

int adam_geometry(const qadam_adamw_config* c, AdamGeometry* g) {
  if (!c) return QADAM_ERR_NULL;
  if (c->num_tensors < 1 || c->num_tensors > (1 << 20) || c->reserved != 0) return QADAM_ERR_SIZE;
  if (!c->len) return QADAM_ERR_NULL;
  if (c->state_bits != 32 && c->state_bits != 8) return QADAM_ERR_TYPE;
  if (c->master != 0 && c->master != 1) return QADAM_ERR_SIZE;
  if (!(c->beta1 >= 0.0f && c->beta1 < 1.0f) || !(c->beta2 >= 0.0f && c->beta2 < 1.0f) || !(c->eps > 0.0f) ||
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
  g->tensors.resize(c->num_tensors);
  g->tiles.reserve((size_t)tiles);
  for (int s = 0; s < c->num_tensors; ++s) {
    AdamTensor& t = g->tensors[s];
    t.w = nullptr;
    t.off = off;
    t.len = c->len[s];
    t.decay = c->decay ? c->decay[s] : 0.0f;
    t.wtype = c->weight_type ? c->weight_type[s] : QADAM_F32;
    t.gtype = c->grad_type ? c->grad_type[s] : QADAM_F32;
    t.first_tile = (int)g->tiles.size();
    for (int64_t o = 0; o < c->len[s]; o += kAdamTile)
      g->tiles.push_back(Tile{(long long)o, (int)std::min<int64_t>(kAdamTile, c->len[s] - o), s});
    off += (c->len[s] + kAlign - 1) / kAlign * kAlign;
  }
  g->D = off;
  size_t wo = round_up256(g->tiles.size() * sizeof(Tile));
  g->off_tensors = wo;
  wo += round_up256(g->tensors.size() * sizeof(AdamTensor));
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

template <bool EIGHT, int CAP>
int launch_adam(qadam_adamw* c, const AdamParams& p, int grid, int tensors, cudaStream_t st) {
  static_assert(sizeof(Pointers<CAP>) + sizeof(AdamParams) <= 32764, "kernel parameters");
  Pointers<CAP> grads;
  std::copy(c->grads.begin() + p.tensor_base, c->grads.begin() + p.tensor_base + tensors, grads.at);
  adamw_kernel<EIGHT, CAP><<<grid, kAdamThreads, 0, st>>>(p, grads);
  if (!cuda_call(cudaGetLastError())) return QADAM_ERR_CUDA;
  c->launches += 1;
  return QADAM_OK;
}

int enqueue_step(qadam_adamw* c, const StepScalars& now, const StepScalars* counted, const float* grad_scale, cudaStream_t st) {
  AdamParams p;
  unsigned char* ws = static_cast<unsigned char*>(c->buf.workspace);
  p.tiles = reinterpret_cast<const Tile*>(ws);
  p.tensors = reinterpret_cast<const AdamTensor*>(ws + c->geo.off_tensors);
  p.beta1 = c->cfg.beta1; p.beta2 = c->cfg.beta2;
  p.c1 = 1.0f - c->cfg.beta1; p.c2 = 1.0f - c->cfg.beta2;
  p.eps = c->cfg.eps;
  p.now = now;
  p.counted = counted;
  p.grad_scale = grad_scale;
  p.master = c->buf.master;
  p.m = c->buf.m; p.v = c->buf.v;
  p.m_scale = c->buf.m_scale; p.r_scale = c->buf.r_scale;
  for (unsigned i = 0; i < 10; ++i) {
    p.keys.k[2 * i] = (unsigned)c->cfg.seed + i * 0x9E3779B9u;
    p.keys.k[2 * i + 1] = (unsigned)(c->cfg.seed >> 32) + i * 0xBB67AE85u;
  }
  p.status = c->buf.status;
  const int tensors = (int)c->geo.tensors.size(), tiles = (int)c->geo.tiles.size();
  for (int s = 0; s < tensors; s += kManyPointers) {
    const int count = std::min(kManyPointers, tensors - s);
    p.tensor_base = s;
    p.first = c->geo.tensors[s].first_tile;
    const int grid = (s + count < tensors ? c->geo.tensors[s + count].first_tile : tiles) - p.first;
    if (grid == 0) continue;
    const bool few = count <= kFewPointers;
    const int rc = c->cfg.state_bits == 8
                       ? (few ? launch_adam<true, kFewPointers>(c, p, grid, count, st) : launch_adam<true, kManyPointers>(c, p, grid, count, st))
                       : (few ? launch_adam<false, kFewPointers>(c, p, grid, count, st) : launch_adam<false, kManyPointers>(c, p, grid, count, st));
    if (rc != QADAM_OK) return rc;
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
    for (size_t s = 0; s < g.tensors.size(); ++s) off[s] = g.tensors[s].off;
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
  for (size_t s = 0; s < g.tensors.size(); ++s) {
    if (!b->weights[s] && g.tensors[s].len > 0) return QADAM_ERR_NULL;
    if (!is_aligned(b->weights[s], type_bytes(g.tensors[s].wtype))) return QADAM_ERR_ALIGN;
    g.tensors[s].w = b->weights[s];
  }
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
      !cuda_call(cudaMemcpy(ws, g.tiles.data(), g.tiles.size() * sizeof(Tile), cudaMemcpyHostToDevice)))
    return QADAM_ERR_CUDA;
  if (!cuda_call(cudaMemcpy(ws + g.off_tensors, g.tensors.data(), g.tensors.size() * sizeof(AdamTensor), cudaMemcpyHostToDevice)) ||
      !cuda_call(cudaMemset(b->status, 0, sizeof(unsigned))) || !cuda_call(cudaStreamSynchronize(nullptr)))
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
  for (size_t s = 0; s < c->geo.tensors.size(); ++s)
    if (!is_aligned(grads[s], type_bytes(c->geo.tensors[s].gtype))) return QADAM_ERR_ALIGN;
  c->grads.assign(grads, grads + c->geo.tensors.size());
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
  adamw_count_kernel<<<1, 1, 0, st>>>(now, reinterpret_cast<long long*>(c->buf.count), lr, c->cfg.lr, c->cfg.beta1,
                                      c->cfg.beta2, grad_scale);
  if (!cuda_call(cudaGetLastError())) return QADAM_ERR_CUDA;
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
  const long long grid = std::min<long long>((quads + kAdamThreads - 1) / kAdamThreads, (long long)c->sm_count * 16);
  adamw_moments_kernel<<<(int)grid, kAdamThreads, 0, static_cast<cudaStream_t>(stream)>>>(
      static_cast<const uint32_t*>(c->buf.m), static_cast<const uint32_t*>(c->buf.v), c->buf.m_scale, c->buf.r_scale, quads,
      reinterpret_cast<float4*>(m32), reinterpret_cast<float4*>(v32));
  if (!cuda_call(cudaGetLastError())) return QADAM_ERR_CUDA;
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
