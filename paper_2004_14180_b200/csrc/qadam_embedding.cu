// Rows of an embedding table and the table's gradient: qadam_embedding_*, qadam_held_lookup.
#include "qadam.h"

#include <algorithm>
#include <cmath>

#include "qadam_tensors.cuh"

using namespace qadam;

namespace {

__device__ __forceinline__ long long load_id(const void* ids, int id_bits, long long t) {
  return id_bits == 64 ? static_cast<const long long*>(ids)[t] : (long long)static_cast<const int*>(ids)[t];
}

// ---------------------------------------------------------------- lookup

constexpr int kLookThreads = 256;
constexpr int kLookQuads = 1024;            // quads of four columns a CTA covers

struct LookupParams {
  const void* table;           // rows, or packed codes
  int type;
  long long rows, stride;
  int width, quads;            // quads: of a row
  const void* ids;
  int id_bits;
  long long count;
  int per_cta;                 // tokens
  float scale;
  void* out;
  int out_type;
  long long out_stride;
  unsigned* status;
  // packed codes
  int kx;
  long long first, words;
};

// Four elements from element e on of the packed weights: code q + 2^kx stands for q 2^-(kx + 1).
__device__ __forceinline__ void held4(const LookupParams& p, long long e, float (&x)[4]) {
  const uint32_t* w = static_cast<const uint32_t*>(p.table);
  const int b = p.kx + 2;
  const long long bit = e * b;
  const long long at = bit >> 5;
  const int shift = (int)(bit & 31);
  const uint32_t w0 = w[at], w1 = w[min(at + 1, p.words - 1)], w2 = w[min(at + 2, p.words - 1)];
  const unsigned long long low = (unsigned long long)w0 | ((unsigned long long)w1 << 32);
  const unsigned long long bits = shift == 0 ? low : (low >> shift) | ((unsigned long long)w2 << (64 - shift));
  const float step = exp2i(-(p.kx + 1));
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = __fmul_rn((float)((int)((bits >> (k * b)) & ((1u << b) - 1u)) - (1 << p.kx)), step);
}

template <bool HELD>
__global__ void __launch_bounds__(kLookThreads) lookup_kernel(const __grid_constant__ LookupParams p) {
  const long long first = (long long)blockIdx.x * p.per_cta;
  const int tokens = (int)min((long long)p.per_cta, p.count - first);
  const int column0 = blockIdx.y * kLookQuads;
  const int quads = min(kLookQuads, p.quads - column0);
  const bool out_fits = aligned4(p.out, p.out_type) && p.out_stride % 4 == 0;
  const bool in_fits = !HELD && aligned4(p.table, p.type) && p.stride % 4 == 0;
  for (int q = threadIdx.x; q < tokens * quads; q += kLookThreads) {
    const long long t = first + q / quads;
    const int col = 4 * (column0 + q % quads);
    const long long id = load_id(p.ids, p.id_bits, t);
    float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (id >= 0 && id < p.rows) {
      if constexpr (HELD) {
        held4(p, p.first + id * p.width + col, x);
      } else {
        const char* row = static_cast<const char*>(p.table) + id * p.stride * type_bytes(p.type);
        to_floats(load_raw4(row, p.type, col, p.width, in_fits && col + 4 <= p.width), p.type, x);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = __fmul_rn(p.scale, x[k]);
    } else if (id >= p.rows && p.status != nullptr && col == 0) {
      atomicOr(p.status, QADAM_ST_INDEX);
    }
    char* row = static_cast<char*>(p.out) + t * p.out_stride * type_bytes(p.out_type);
    store_raw4(row, p.out_type, col, p.width, out_fits && col + 4 <= p.width, from_floats(x, p.out_type));
  }
}

int enqueue_lookup(LookupParams p, bool held, cudaStream_t st) {
  p.quads = (p.width + 3) / 4;
  const int across = (p.quads + kLookQuads - 1) / kLookQuads;
  p.per_cta = std::max(1, kLookQuads / p.quads);
  const long long grid = (p.count + p.per_cta - 1) / p.per_cta;
  if (grid > 0x7FFFFFFF) return QADAM_ERR_SIZE;
  if (held) lookup_kernel<true><<<dim3((unsigned)grid, across), kLookThreads, 0, st>>>(p);
  else lookup_kernel<false><<<dim3((unsigned)grid, across), kLookThreads, 0, st>>>(p);
  return cuda_call(cudaGetLastError()) ? QADAM_OK : QADAM_ERR_CUDA;
}

// ---------------------------------------------------------------- gradient: tokens sorted by id
//
// Stable sort of (id, place) by the bits of the id, at most 9 bits a pass: counts of each digit in each
// CTA's run of tokens, their running sum (all smaller digits, then the same digit in earlier runs), and
// every token to its place.  Stable, so a row's tokens stay in the order of the batch.

constexpr int kSortThreads = 512;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortItems = 8;                              // tokens per thread
constexpr int kSortRun = kSortThreads * kSortItems;        // 4096 tokens per CTA
constexpr int kDigitBits = 9;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kScanThreads = 1024;

struct SortParams {
  const void* ids;             // of the first pass; later passes read keys
  int id_bits;
  const unsigned* keys;
  const unsigned* places;
  unsigned* out_keys;
  unsigned* out_places;
  unsigned* counts;            // [digits][runs]
  int count, runs;
  int shift, digits;
  unsigned rows;
  long long padding;
  unsigned* status;
};

// The sort's key of a token: its row, or `rows` for one that is left out.
__device__ __forceinline__ unsigned sort_key(const SortParams& p, int t) {
  if (p.keys != nullptr) return p.keys[t];
  const long long id = load_id(p.ids, p.id_bits, t);
  if (id < 0 || id == p.padding) return p.rows;
  if (id >= (long long)p.rows) {
    if (p.status != nullptr) atomicOr(p.status, QADAM_ST_INDEX);
    return p.rows;
  }
  return (unsigned)id;
}

__global__ void __launch_bounds__(kSortThreads) count_digits_kernel(const __grid_constant__ SortParams p) {
  __shared__ unsigned n[kDigits];
  for (int d = threadIdx.x; d < p.digits; d += kSortThreads) n[d] = 0u;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kSortItems; ++j) {
    const long long t = (long long)blockIdx.x * kSortRun + j * kSortThreads + threadIdx.x;
    if (t < p.count) atomicAdd(&n[(sort_key(p, (int)t) >> p.shift) & (p.digits - 1)], 1u);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < p.digits; d += kSortThreads) p.counts[(size_t)d * p.runs + blockIdx.x] = n[d];
}

// Running sum of n counts in place, by one CTA: every thread a contiguous part.
__global__ void __launch_bounds__(kScanThreads) scan_counts_kernel(unsigned* counts, long long n) {
  __shared__ unsigned warp_total[kScanThreads / 32];
  const long long part = (n + kScanThreads - 1) / kScanThreads;
  const long long lo = min(n, threadIdx.x * part), hi = min(n, lo + part);
  unsigned sum = 0u;
  for (long long i = lo; i < hi; ++i) sum += counts[i];
  const int lane = threadIdx.x % 32;
  unsigned upto = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned other = __shfl_up_sync(0xFFFFFFFFu, upto, o);
    if (lane >= o) upto += other;
  }
  if (lane == 31) warp_total[threadIdx.x / 32] = upto;
  __syncthreads();
  if (threadIdx.x < 32) {
    unsigned w = warp_total[lane], s = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned other = __shfl_up_sync(0xFFFFFFFFu, s, o);
      if (lane >= o) s += other;
    }
    warp_total[lane] = s - w;
  }
  __syncthreads();
  unsigned at = warp_total[threadIdx.x / 32] + upto - sum;
  for (long long i = lo; i < hi; ++i) {
    const unsigned c = counts[i];
    counts[i] = at;
    at += c;
  }
}

__global__ void __launch_bounds__(kSortThreads) place_kernel(const __grid_constant__ SortParams p) {
  // tokens of each digit that a warp has seen, then where the warp's tokens of that digit begin
  __shared__ unsigned short seen[kSortWarps][kDigits];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  for (int i = threadIdx.x; i < kSortWarps * kDigits; i += kSortThreads) (&seen[0][0])[i] = 0;
  __syncthreads();
  unsigned key[kSortItems];
  unsigned short rank[kSortItems];
  const long long base = (long long)blockIdx.x * kSortRun + warp * (32 * kSortItems) + lane;
#pragma unroll
  for (int j = 0; j < kSortItems; ++j) {
    const long long t = base + 32 * j;
    const bool live = t < p.count;
    key[j] = live ? sort_key(p, (int)t) : 0u;
    const unsigned d = live ? (key[j] >> p.shift) & (p.digits - 1) : (unsigned)p.digits + lane;   // nobody's peer
    const unsigned peers = __match_any_sync(0xFFFFFFFFu, d);
    const int before = __popc(peers & ((1u << lane) - 1u));
    const int had = live ? seen[warp][d] : 0;
    __syncwarp();
    if (live && before == 0) seen[warp][d] = (unsigned short)(had + __popc(peers));
    __syncwarp();
    rank[j] = (unsigned short)(had + before);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < p.digits; d += kSortThreads) {
    unsigned at = 0u;
    for (int w = 0; w < kSortWarps; ++w) {
      const unsigned n = seen[w][d];
      seen[w][d] = (unsigned short)at;
      at += n;
    }
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kSortItems; ++j) {
    const long long t = base + 32 * j;
    if (t < p.count) {
      const unsigned d = (key[j] >> p.shift) & (p.digits - 1);
      const unsigned to = p.counts[(size_t)d * p.runs + blockIdx.x] + seen[warp][d] + rank[j];
      p.out_keys[to] = key[j];
      p.out_places[to] = p.places != nullptr ? p.places[t] : (unsigned)t;
    }
  }
}

// ---------------------------------------------------------------- gradient: sums
//
// The sorted tokens are cut into chunks of kChunk.  A warp adds up one chunk's rows in 128 columns, four to
// a lane, and writes a row that begins and ends in its chunk.  A row's tokens that cross a chunk's end leave
// a partial sum there; the rows that cross are put together from those in order.

constexpr int kChunk = 32;
constexpr int kSumThreads = 256;
constexpr int kSumWarps = kSumThreads / 32;
constexpr int kSumColumns = 128;
constexpr int kAhead = 8;                                  // rows asked for at a time

struct GradParams {
  const unsigned* keys;        // sorted; `rows` behind the last
  const unsigned* places;
  int count, chunks;
  const void* dy;
  int dy_type;
  long long dy_stride;
  float scale;
  void* grad;
  int grad_type;
  long long rows, grad_stride;
  int width, tiles;            // tiles: of 128 columns
  int accumulate;
  float* partial;              // [chunks][2][tiles * 128]: the run that began in an earlier chunk, the one that goes on
};

__global__ void __launch_bounds__(kSumThreads) zero_rows_kernel(const __grid_constant__ GradParams p) {
  const int quads = (p.width + 3) / 4;
  const bool fits = aligned4(p.grad, p.grad_type) && p.grad_stride % 4 == 0;
  const Raw4 zero = {{0u, 0u, 0u, 0u}};
  const long long n = p.rows * quads;
  for (long long q = (long long)blockIdx.x * kSumThreads + threadIdx.x; q < n; q += (long long)gridDim.x * kSumThreads) {
    const long long row = q / quads;
    const int col = 4 * (int)(q - row * quads);
    store_raw4(static_cast<char*>(p.grad) + row * p.grad_stride * type_bytes(p.grad_type), p.grad_type, col, p.width,
               fits && col + 4 <= p.width, zero);
  }
}

__device__ __forceinline__ void finish_row(const GradParams& p, unsigned row, int col, bool fits, const float (&sum)[4]) {
  if (col >= p.width) return;
  char* dst = static_cast<char*>(p.grad) + (long long)row * p.grad_stride * type_bytes(p.grad_type);
  const bool whole = fits && col + 4 <= p.width;
  float x[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = __fmul_rn(p.scale, sum[k]);
  if (p.accumulate) {
    float old[4];
    to_floats(load_raw4(dst, p.grad_type, col, p.width, whole), p.grad_type, old);
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = __fadd_rn(old[k], x[k]);
  }
  store_raw4(dst, p.grad_type, col, p.width, whole, from_floats(x, p.grad_type));
}

__device__ __forceinline__ float* partial_row(const GradParams& p, int chunk, int which, int col) {
  return p.partial + ((long long)chunk * 2 + which) * ((long long)p.tiles * kSumColumns) + col;
}

__global__ void __launch_bounds__(kSumThreads) sum_chunks_kernel(const __grid_constant__ GradParams p) {
  const long long unit = (long long)blockIdx.x * kSumWarps + threadIdx.x / 32;
  const int lane = threadIdx.x % 32;
  if (unit >= (long long)p.chunks * p.tiles) return;
  const int chunk = (int)(unit / p.tiles), col = (int)(unit % p.tiles) * kSumColumns + 4 * lane;
  const int begin = chunk * kChunk, n = min(kChunk, p.count - begin);
  const unsigned none = (unsigned)p.rows;
  unsigned key = none, place = 0u;
  if (lane < n) {
    key = p.keys[begin + lane];
    place = p.places[begin + lane];
  }
  const unsigned first = __shfl_sync(0xFFFFFFFFu, key, 0), last = __shfl_sync(0xFFFFFFFFu, key, n - 1);
  if (first == none) return;
  const bool from_before = begin > 0 && p.keys[begin - 1] == first;
  const bool goes_on = last != none && begin + n < p.count && p.keys[begin + n] == last;
  const bool dy_fits = aligned4(p.dy, p.dy_type) && p.dy_stride % 4 == 0;
  const bool grad_fits = aligned4(p.grad, p.grad_type) && p.grad_stride % 4 == 0;
  const int row_bytes_of = type_bytes(p.dy_type);
  float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  unsigned current = first;
  bool at_first = true;
  for (int j0 = 0; j0 < n; j0 += kAhead) {
    Raw4 raw[kAhead];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const unsigned row = __shfl_sync(0xFFFFFFFFu, place, j0 + a);
      const unsigned k = __shfl_sync(0xFFFFFFFFu, key, j0 + a);
      raw[a] = {{0u, 0u, 0u, 0u}};
      if (k != none && col < p.width)
        raw[a] = load_raw4(static_cast<const char*>(p.dy) + (long long)row * p.dy_stride * row_bytes_of, p.dy_type, col, p.width,
                           dy_fits && col + 4 <= p.width);
    }
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const unsigned k = __shfl_sync(0xFFFFFFFFu, key, j0 + a);
      if (k != current) {
        if (current != none) {
          if (at_first && from_before) *reinterpret_cast<float4*>(partial_row(p, chunk, 0, col)) = make_float4(sum[0], sum[1], sum[2], sum[3]);
          else finish_row(p, current, col, grad_fits, sum);
        }
        at_first = false;
        current = k;
        sum[0] = sum[1] = sum[2] = sum[3] = 0.0f;
      }
      float x[4];
      to_floats(raw[a], p.dy_type, x);
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] = __fadd_rn(sum[i], x[i]);
    }
  }
  if (current == none) return;
  if (at_first && from_before) *reinterpret_cast<float4*>(partial_row(p, chunk, 0, col)) = make_float4(sum[0], sum[1], sum[2], sum[3]);
  else if (goes_on) *reinterpret_cast<float4*>(partial_row(p, chunk, 1, col)) = make_float4(sum[0], sum[1], sum[2], sum[3]);
  else finish_row(p, current, col, grad_fits, sum);
}

// One CTA per chunk and 128 columns: the run that begins in the chunk and goes on beyond it, if there is one.
__global__ void __launch_bounds__(kSumThreads) join_chunks_kernel(const __grid_constant__ GradParams p) {
  __shared__ float4 part[kSumWarps][32];
  const int chunk = blockIdx.x, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int col = blockIdx.y * kSumColumns + 4 * lane;
  const int begin = chunk * kChunk, end = begin + kChunk;
  if (end >= p.count) return;
  const unsigned key = p.keys[end - 1];
  if (key == (unsigned)p.rows || p.keys[end] != key) return;                    // nothing goes on
  if (p.keys[begin] == key && begin > 0 && p.keys[begin - 1] == key) return;    // it began earlier
  int lo = end, hi = p.count;                                                   // first place behind the run
  while (lo < hi) {
    const int mid = lo + (hi - lo) / 2;
    if (p.keys[mid] == key) lo = mid + 1;
    else hi = mid;
  }
  const int last = (lo - 1) / kChunk;                                           // chunk the run ends in
  const int n = last - chunk + 1, each = (n + kSumWarps - 1) / kSumWarps;
  float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int i = warp * each; i < min(n, (warp + 1) * each); ++i) {
    const float4 x = *reinterpret_cast<const float4*>(partial_row(p, chunk + i, i == 0 ? 1 : 0, col));
    sum[0] = __fadd_rn(sum[0], x.x);
    sum[1] = __fadd_rn(sum[1], x.y);
    sum[2] = __fadd_rn(sum[2], x.z);
    sum[3] = __fadd_rn(sum[3], x.w);
  }
  part[warp][lane] = make_float4(sum[0], sum[1], sum[2], sum[3]);
  __syncthreads();
  if (warp != 0) return;
  for (int w = 1; w < min(kSumWarps, n); ++w) {
    const float4 x = part[w][lane];
    sum[0] = __fadd_rn(sum[0], x.x);
    sum[1] = __fadd_rn(sum[1], x.y);
    sum[2] = __fadd_rn(sum[2], x.z);
    sum[3] = __fadd_rn(sum[3], x.w);
  }
  finish_row(p, key, col, aligned4(p.grad, p.grad_type) && p.grad_stride % 4 == 0, sum);
}

// ---------------------------------------------------------------- host side

struct GradLayout {
  size_t keys[2], places[2], counts, partial, bytes;
  int runs, chunks, tiles;
};

int grad_layout(int64_t count, int64_t rows, int64_t width, GradLayout* l) {
  if (count < 0 || count > (int64_t)1 << 30 || rows < 1 || rows >= 0x7FFFFFFF || width < 1 || width > (int64_t)1 << 22)
    return QADAM_ERR_SIZE;
  l->runs = (int)((count + kSortRun - 1) / kSortRun);
  l->chunks = (int)((count + kChunk - 1) / kChunk);
  l->tiles = (int)((width + kSumColumns - 1) / kSumColumns);
  if ((int64_t)l->chunks * l->tiles > (int64_t)1 << 32) return QADAM_ERR_SIZE;      // (warps of one launch)
  size_t at = 0;
  const size_t list = round_up256((size_t)count * sizeof(unsigned));
  for (int i = 0; i < 2; ++i) {
    l->keys[i] = at;
    at += list;
    l->places[i] = at;
    at += list;
  }
  l->counts = at;
  at += round_up256((size_t)l->runs * kDigits * sizeof(unsigned));
  l->partial = at;
  at += (size_t)l->chunks * 2 * l->tiles * kSumColumns * sizeof(float);
  l->bytes = at + 256;
  return QADAM_OK;
}

int check_rows(const void* p, int type, int64_t width, int64_t stride) {
  if (!known_type(type)) return QADAM_ERR_TYPE;
  if (stride < width || stride > (int64_t)1 << 40) return QADAM_ERR_SIZE;
  return is_aligned(p, type_bytes(type)) ? QADAM_OK : QADAM_ERR_ALIGN;
}

int check_ids(const void* ids, int id_bits, int64_t count) {
  if (id_bits != 32 && id_bits != 64) return QADAM_ERR_TYPE;
  if (!ids && count > 0) return QADAM_ERR_NULL;
  return is_aligned(ids, id_bits / 8) ? QADAM_OK : QADAM_ERR_ALIGN;
}

int check_lookup(const void* table, int64_t rows, int64_t width, const void* ids, int32_t id_bits, int64_t count, float scale,
                 const void* out, int32_t out_type, int64_t out_stride, const uint32_t* status) {
  if (!table || (!out && count > 0)) return QADAM_ERR_NULL;
  if (rows < 1 || rows > (int64_t)1 << 40 || width < 1 || width > (int64_t)1 << 24 || count < 0 || count > (int64_t)1 << 40)
    return QADAM_ERR_SIZE;
  if (!std::isfinite(scale)) return QADAM_ERR_HYPER;
  int rc = check_rows(out, out_type, width, out_stride);
  if (rc == QADAM_OK) rc = check_ids(ids, id_bits, count);
  if (rc == QADAM_OK && !is_aligned(status, 4)) rc = QADAM_ERR_ALIGN;
  return rc;
}

}  // namespace

extern "C" {

int qadam_embedding_lookup(const void* table, int32_t type, int64_t rows, int64_t width, int64_t stride, const void* ids,
                           int32_t id_bits, int64_t count, float scale, void* out, int32_t out_type, int64_t out_stride,
                           uint32_t* status, void* stream) {
  int rc = check_lookup(table, rows, width, ids, id_bits, count, scale, out, out_type, out_stride, status);
  if (rc == QADAM_OK) rc = check_rows(table, type, width, stride);
  if (rc != QADAM_OK || count == 0) return rc;
  LookupParams p = {};
  p.table = table; p.type = type; p.rows = rows; p.stride = stride; p.width = (int)width;
  p.ids = ids; p.id_bits = id_bits; p.count = count; p.scale = scale;
  p.out = out; p.out_type = out_type; p.out_stride = out_stride; p.status = status;
  return enqueue_lookup(p, false, static_cast<cudaStream_t>(stream));
}

int qadam_held_lookup(const void* wcodes, size_t wcode_bytes, int32_t kx, int64_t first, int64_t rows, int64_t width,
                      const void* ids, int32_t id_bits, int64_t count, float scale, void* out, int32_t out_type,
                      int64_t out_stride, uint32_t* status, void* stream) {
  int rc = check_lookup(wcodes, rows, width, ids, id_bits, count, scale, out, out_type, out_stride, status);
  if (rc != QADAM_OK) return rc;
  if (kx < 0 || kx > 14) return QADAM_ERR_LEVEL;
  if (!is_aligned(wcodes, 16)) return QADAM_ERR_ALIGN;
  if (first < 0 || first > (int64_t)1 << 44 || wcode_bytes % 16 != 0 || wcode_bytes / 2 > (size_t)1 << 44) return QADAM_ERR_SIZE;
  const int64_t held = (int64_t)(wcode_bytes * 8 / (size_t)(kx + 2));            // elements
  if (first > held || rows > (held - first) / width) return QADAM_ERR_SIZE;
  if (count == 0) return QADAM_OK;
  LookupParams p = {};
  p.table = wcodes; p.rows = rows; p.width = (int)width;
  p.ids = ids; p.id_bits = id_bits; p.count = count; p.scale = scale;
  p.out = out; p.out_type = out_type; p.out_stride = out_stride; p.status = status;
  p.kx = kx; p.first = first; p.words = (long long)(wcode_bytes / 4);
  return enqueue_lookup(p, true, static_cast<cudaStream_t>(stream));
}

int qadam_embedding_grad_query_sizes(int64_t count, int64_t rows, int64_t width, size_t* workspace_bytes) {
  GradLayout l;
  const int rc = grad_layout(count, rows, width, &l);
  if (rc == QADAM_OK && workspace_bytes) *workspace_bytes = l.bytes;
  return rc;
}

int qadam_embedding_grad(const void* ids, int32_t id_bits, int64_t count, const void* dy, int32_t dy_type, int64_t dy_stride,
                         float scale, int64_t padding, void* grad, int32_t grad_type, int64_t rows, int64_t width,
                         int64_t grad_stride, int32_t accumulate, void* workspace, size_t workspace_bytes, uint32_t* status,
                         void* stream) {
  if (!grad || (!dy && count > 0)) return QADAM_ERR_NULL;
  GradLayout l;
  int rc = grad_layout(count, rows, width, &l);
  if (rc != QADAM_OK) return rc;
  if (accumulate != 0 && accumulate != 1) return QADAM_ERR_SIZE;
  if (!std::isfinite(scale)) return QADAM_ERR_HYPER;
  rc = check_rows(grad, grad_type, width, grad_stride);
  if (rc == QADAM_OK) rc = check_rows(dy, dy_type, width, dy_stride);
  if (rc == QADAM_OK) rc = check_ids(ids, id_bits, count);
  if (rc == QADAM_OK && !is_aligned(status, 4)) rc = QADAM_ERR_ALIGN;
  if (rc != QADAM_OK) return rc;
  if (count > 0 && !workspace) return QADAM_ERR_NULL;
  if (!is_aligned(workspace, 256)) return QADAM_ERR_ALIGN;
  if (count > 0 && workspace_bytes < l.bytes) return QADAM_ERR_WORKSPACE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  auto list = [&](size_t off) { return reinterpret_cast<unsigned*>(ws + off); };

  GradParams g = {};
  g.count = (int)count; g.chunks = l.chunks;
  g.dy = dy; g.dy_type = dy_type; g.dy_stride = dy_stride; g.scale = scale;
  g.grad = grad; g.grad_type = grad_type; g.rows = rows; g.grad_stride = grad_stride;
  g.width = (int)width; g.tiles = l.tiles; g.accumulate = accumulate;
  if (!accumulate) {
    const long long quads = rows * ((width + 3) / 4);
    zero_rows_kernel<<<(int)std::min<long long>((quads + kSumThreads - 1) / kSumThreads, 148 * 8), kSumThreads, 0, st>>>(g);
    if (!cuda_call(cudaGetLastError())) return QADAM_ERR_CUDA;
  }
  if (count == 0) return QADAM_OK;

  int bits = 1;
  while ((rows >> bits) != 0) ++bits;                        // keys 0 .. rows
  const int passes = (bits + kDigitBits - 1) / kDigitBits, digit = (bits + passes - 1) / passes;
  SortParams s = {};
  s.ids = ids; s.id_bits = id_bits; s.count = (int)count; s.runs = l.runs; s.rows = (unsigned)rows;
  s.padding = padding; s.status = status; s.digits = 1 << digit;
  s.counts = list(l.counts);
  for (int i = 0; i < passes; ++i) {
    s.shift = i * digit;
    s.keys = i == 0 ? nullptr : list(l.keys[(i + 1) % 2]);
    s.places = i == 0 ? nullptr : list(l.places[(i + 1) % 2]);
    s.out_keys = list(l.keys[i % 2]);
    s.out_places = list(l.places[i % 2]);
    count_digits_kernel<<<l.runs, kSortThreads, 0, st>>>(s);
    scan_counts_kernel<<<1, kScanThreads, 0, st>>>(s.counts, (long long)l.runs << digit);
    place_kernel<<<l.runs, kSortThreads, 0, st>>>(s);
    if (!cuda_call(cudaGetLastError())) return QADAM_ERR_CUDA;
  }
  g.keys = s.out_keys;
  g.places = s.out_places;
  g.partial = reinterpret_cast<float*>(ws + l.partial);
  const long long units = (long long)l.chunks * l.tiles;
  const long long grid = (units + kSumWarps - 1) / kSumWarps;
  sum_chunks_kernel<<<(unsigned)grid, kSumThreads, 0, st>>>(g);
  if (l.chunks > 1) join_chunks_kernel<<<dim3((unsigned)l.chunks, (unsigned)l.tiles), kSumThreads, 0, st>>>(g);
  return cuda_call(cudaGetLastError()) ? QADAM_OK : QADAM_ERR_CUDA;
}

}  // extern "C"
