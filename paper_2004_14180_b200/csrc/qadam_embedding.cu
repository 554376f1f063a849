// Rows of an embedding table and the table's gradient: qadam_embedding_*, qadam_held_lookup.
#include "qadam.h"

#include <cooperative_groups.h>

#include <algorithm>
#include <cmath>

#include "qadam_tensors.cuh"

using namespace qadam;

namespace {

__device__ __forceinline__ long long load_id(const void* ids, int id_bits, long long t) {
  return id_bits == 64 ? static_cast<const long long*>(ids)[t] : (long long)static_cast<const int*>(ids)[t];
}

// ---------------------------------------------------------------- lookup

//
// Reads the rows that the batch names, writes a row per token: bound by HBM for long batches, by two trips to memory
// (tokens, then rows) for short ones.  A CTA fetches its tokens first; a thread then has AHEAD pieces of eight columns
// under way.  Where rows do not begin on 16 bytes, a piece's columns are 32 apart, so that a warp's accesses are next to
// each other.

constexpr int kLookThreads = 256;
constexpr int kLookRounds = 4;                             // tokens that a thread takes (8192 held rows: 2 7.2 us, 4 6.4, 8 7.1)
constexpr int kLookTokens = kLookThreads * kLookRounds;
// What the rows are: elements of 16 or 32 bits, or packed codes of KIND = 2 .. 16 bits.
constexpr int kDense16 = 0, kDense32 = 1;
template <int KIND>
constexpr int kPieceWords = KIND == kDense32 ? 8 : KIND == kDense16 ? 4 : (8 * KIND + 31 + 31) / 32;
template <int KIND>
constexpr int kLookAhead = KIND == kDense32 ? 2 : 4;

struct LookupParams {
  const void* table;           // rows, or packed codes
  int type;
  long long rows, stride;
  int width, pieces;           // pieces: of a row
  int here, across;            // of a row in one CTA, at the most; CTAs of a row
  int at_once;                 // tokens that a CTA's threads take at a time
  const void* ids;
  int id_bits;
  long long count;
  int per_cta;                 // tokens
  float scale;
  void* out;
  int out_type;
  long long out_stride;
  int spread;                  // rows, of the table or of the result, do not begin on 16 bytes
  unsigned* status;
  long long first, words;      // packed codes
};

// Columns of a piece: first + k step.
__device__ __forceinline__ int piece_column(const LookupParams& p, int piece) {
  return p.spread ? piece / 32 * 256 + piece % 32 : 8 * piece;
}

// Eight elements of a row as they lie in memory (a word each, if spread).
template <int KIND>
struct Piece {
  uint32_t w[kPieceWords<KIND>];
};
struct SpreadPiece {
  uint32_t w[8];
};

template <int KIND>
__device__ __forceinline__ Piece<KIND> load_piece(const LookupParams& p, long long id, int col) {
  Piece<KIND> r = {};
  if constexpr (KIND == kDense16 || KIND == kDense32) {
    constexpr int kBytes = KIND == kDense32 ? 4 : 2;
    const char* row = static_cast<const char*>(p.table) + id * p.stride * kBytes;
    if (col + 8 <= p.width) {
      const uint4 a = *reinterpret_cast<const uint4*>(row + (size_t)col * kBytes);
      r.w[0] = a.x; r.w[1] = a.y; r.w[2] = a.z; r.w[3] = a.w;
      if constexpr (KIND == kDense32) {
        const uint4 b = *reinterpret_cast<const uint4*>(row + (size_t)col * 4 + 16);
        r.w[4] = b.x; r.w[5] = b.y; r.w[6] = b.z; r.w[7] = b.w;
      }
    } else {
      for (int k = 0; k < 8; ++k) {
        if (col + k >= p.width) break;
        if constexpr (KIND == kDense32) r.w[k] = reinterpret_cast<const uint32_t*>(row)[col + k];
        else r.w[k / 2] |= (uint32_t) reinterpret_cast<const unsigned short*>(row)[col + k] << (16 * (k % 2));
      }
    }
  } else {
    const long long at = (p.first + id * p.width + col) * KIND >> 5;
    const uint32_t* w = static_cast<const uint32_t*>(p.table) + at;
    if (at + kPieceWords<KIND> <= p.words) {
#pragma unroll
      for (int k = 0; k < kPieceWords<KIND>; ++k) r.w[k] = w[k];
    } else {
      const int last = (int)(p.words - 1 - at);              // (codes end in a word before the piece's last)
#pragma unroll
      for (int k = 0; k < kPieceWords<KIND>; ++k) r.w[k] = w[min(k, last)];
    }
  }
  return r;
}

// Code q + 2^kx stands for q 2^-(kx + 1).  The code becomes the last bits of 2^23 + code.
template <int KIND>
__device__ __forceinline__ float code_value(unsigned code) {
  const float q = __fadd_rn(__uint_as_float(0x4B000000u | (code & ((1u << KIND) - 1u))), -(8388608.0f + (float)(1 << (KIND - 2))));
  return __fmul_rn(q, 1.0f / (float)(1 << (KIND - 1)));
}

template <int KIND>
__device__ __forceinline__ void piece_floats(const LookupParams& p, const Piece<KIND>& r, long long id, int col, float (&x)[8]) {
  if constexpr (KIND == kDense32) {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = __uint_as_float(r.w[k]);
  } else if constexpr (KIND == kDense16) {
    float a[4], b[4];
    to_floats(Raw4{{r.w[0], r.w[1], 0u, 0u}}, p.type, a);
    to_floats(Raw4{{r.w[2], r.w[3], 0u, 0u}}, p.type, b);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[k] = a[k];
      x[4 + k] = b[k];
    }
  } else {
    const int shift = (int)((p.first + id * p.width + col) * KIND & 31);
    unsigned v[kPieceWords<KIND>];                         // 8 KIND bits
#pragma unroll
    for (int k = 0; k < kPieceWords<KIND>; ++k) v[k] = k + 1 < kPieceWords<KIND> ? __funnelshift_r(r.w[k], r.w[k + 1], shift) : r.w[k] >> shift;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int at = k * KIND, w = at / 32, bit = at % 32;
      unsigned code = v[w] >> bit;
      if (bit + KIND > 32) code |= v[w + 1] << (32 - bit);
      x[k] = code_value<KIND>(code);
    }
  }
}

template <int KIND>
__device__ __forceinline__ SpreadPiece load_spread(const LookupParams& p, long long id, int col) {
  SpreadPiece r = {};
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int at = col + 32 * k;
    if (at >= p.width) break;
    if constexpr (KIND == kDense32) {
      r.w[k] = static_cast<const uint32_t*>(p.table)[id * p.stride + at];
    } else if constexpr (KIND == kDense16) {
      r.w[k] = static_cast<const unsigned short*>(p.table)[id * p.stride + at];
    } else {
      // 32 bits from the 16 that the code begins in: it ends in them
      const long long half = (p.first + id * p.width + at) * KIND >> 4;
      const unsigned short* h = static_cast<const unsigned short*>(p.table);
      r.w[k] = h[half] | (uint32_t)h[min(half + 1, 2 * p.words - 1)] << 16;
    }
  }
  return r;
}

template <int KIND>
__device__ __forceinline__ void spread_floats(const LookupParams& p, const SpreadPiece& r, long long id, int col, float (&x)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if constexpr (KIND == kDense32) {
      x[k] = __uint_as_float(r.w[k]);
    } else if constexpr (KIND == kDense16) {
      x[k] = p.type == QADAM_BF16 ? __uint_as_float(r.w[k] << 16) : half_bits_to_float(r.w[k]);
    } else {
      x[k] = code_value<KIND>(r.w[k] >> (int)((p.first + id * p.width + col + 32 * k) * KIND & 15));
    }
  }
}

__device__ __forceinline__ void store_piece(const LookupParams& p, long long t, int col, const float (&x)[8]) {
  const float lo[4] = {x[0], x[1], x[2], x[3]}, hi[4] = {x[4], x[5], x[6], x[7]};
  const Raw4 a = from_floats(lo, p.out_type), b = from_floats(hi, p.out_type);
  char* row = static_cast<char*>(p.out) + t * p.out_stride * type_bytes(p.out_type);
  if (!p.spread && col + 8 <= p.width) {
    uint4* out = reinterpret_cast<uint4*>(row + (size_t)col * type_bytes(p.out_type));
    if (p.out_type == QADAM_F32) {
      out[0] = make_uint4(a.w[0], a.w[1], a.w[2], a.w[3]);
      out[1] = make_uint4(b.w[0], b.w[1], b.w[2], b.w[3]);
    } else {
      out[0] = make_uint4(a.w[0], a.w[1], b.w[0], b.w[1]);
    }
    return;
  }
  const int step = p.spread ? 32 : 1;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int at = col + k * step;
    if (at >= p.width) break;
    const Raw4& r = k < 4 ? a : b;
    if (p.out_type == QADAM_F32) reinterpret_cast<uint32_t*>(row)[at] = r.w[k % 4];
    else reinterpret_cast<unsigned short*>(row)[at] = (unsigned short)(r.w[k % 4 / 2] >> (16 * (k % 2)));
  }
}

template <int KIND>
__global__ void __launch_bounds__(kLookThreads, 6) lookup_kernel(const __grid_constant__ LookupParams p) {
  wait_for_previous_launch();
  constexpr int AHEAD = kLookAhead<KIND>;
  __shared__ long long ids[kLookTokens];
  const long long first = (long long)(blockIdx.x / p.across) * p.per_cta;
  const int tokens = (int)min((long long)p.per_cta, p.count - first);
  for (int t = threadIdx.x; t < tokens; t += blockDim.x) {
    long long id = load_id(p.ids, p.id_bits, first + t);
    if (id >= p.rows) {
      if (p.status != nullptr) atomicOr(p.status, QADAM_ST_INDEX);
      id = -1;
    }
    ids[t] = id;
  }
  __syncthreads();
  // a thread keeps its columns and goes from token to token
  const int row = threadIdx.x / p.here, piece = (int)(blockIdx.x % p.across) * p.here + (threadIdx.x - row * p.here);
  if (piece >= p.pieces) return;
  const int col = piece_column(p, piece), step = p.at_once;
  if (p.spread) {
    for (int t = row; t < tokens; t += step) {
      const long long id = ids[t];
      float x[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
      if (id >= 0) {
        spread_floats<KIND>(p, load_spread<KIND>(p, id, col), id, col, x);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = __fmul_rn(p.scale, x[k]);
      }
      store_piece(p, first + t, col, x);
    }
    return;
  }
  for (int t0 = row; t0 < tokens; t0 += AHEAD * step) {
    Piece<KIND> raw[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int t = t0 + j * step;
      const long long id = t < tokens ? ids[t] : -1;
      raw[j] = Piece<KIND>{};
      if (id >= 0) raw[j] = load_piece<KIND>(p, id, col);
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int t = t0 + j * step;
      if (t >= tokens) break;
      const long long id = ids[t];
      float x[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
      if (id >= 0) {
        piece_floats<KIND>(p, raw[j], id, col, x);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = __fmul_rn(p.scale, x[k]);
      }
      store_piece(p, first + t, col, x);
    }
  }
}

template <int KIND>
bool launch_lookup(const LookupParams& p, long long grid, int kind, cudaStream_t st) {
  if (kind == KIND) return launch(lookup_kernel<KIND>, grid, p.here * p.at_once, 0, 0, st, p);
  if constexpr (KIND < 16) return launch_lookup<KIND + 1>(p, grid, kind, st);
  return false;
}

int enqueue_lookup(LookupParams p, int kind, cudaStream_t st) {
  const bool in_fits = kind > kDense32 || (is_aligned(p.table, 16) && p.stride * type_bytes(p.type) % 16 == 0);
  p.spread = !in_fits || !is_aligned(p.out, 16) || p.out_stride * type_bytes(p.out_type) % 16 != 0;
  p.pieces = p.spread ? (p.width + 255) / 256 * 32 : (p.width + 7) / 8;
  p.here = std::min(p.pieces, kLookThreads);
  p.across = (p.pieces + p.here - 1) / p.here;
  p.at_once = kLookThreads / p.here;
  p.per_cta = p.at_once * kLookRounds;
  const long long ctas = (p.count + p.per_cta - 1) / p.per_cta;
  if (ctas > 0x7FFFFFFF / p.across) return QADAM_ERR_SIZE;
  return launch_lookup<kDense16>(p, ctas * p.across, kind, st) ? QADAM_OK : QADAM_ERR_CUDA;
}

// ---------------------------------------------------------------- gradient: tokens sorted by id
//
// (row, place) of every token, stable by row, so a row's tokens stay in the order of the batch.  The
// launches that sort leave most of the GPU idle: further CTAs of theirs clear the gradient meanwhile.

constexpr int kSortThreads = 512;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortItems = 8;                              // tokens per thread
constexpr int kSortRun = kSortThreads * kSortItems;        // 4096 tokens per CTA
constexpr int kDigitBits = 9;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kDirectRuns = 256;                           // up to so many runs every CTA adds up the counts for itself
// Up to so many tokens are ranked by comparing all pairs.  Whole calls that add to 30522 x 768, ranked / sorted by a cluster:
// 256 tokens 8.4 us / 12.9, 1024 11.5 / 15.5, 2048 14.3 / 16.6, 8192 25.7 / 20.2.
constexpr int kRankTokens = 2048;
constexpr int kCluster = 8;                                // CTAs that sort up to 8 x 4096 tokens through each other's shared memory
constexpr int kRankThreads = 512;
constexpr int kRankWarps = kRankThreads / 32;
constexpr int kRankPer = 64;                               // tokens that a CTA ranks
// Threads that clear beside the CTAs that sort.  Whole calls with 16 / 256 / 2048 / 8192 / 32768 tokens, binary32 gradients of 768
// columns, us:
//                  1000 rows                      30522                          400000
//   136 x  512     4.0   8.1                      18.0  20.2                     205   209
//   136 x 2048     4.2   8.2  15.6  19.7  33.5    18.5  20.9  24.3  28.8  45.2    186   188   192   223   237
//   136 x 4096     4.2   8.2  15.6  19.7  33.5    17.6  20.0  23.2  28.5  45.0    191   193   197   202   216
//   136 x 8192     4.2   8.2  15.6  19.7  33.5    17.0  19.4  23.1  27.9  44.3    183   185   189   190   204
// The last takes 8.3 us in place of 7.1 for 16 tokens and 8000 rows, and 82 in place of 79 for 10^5 tokens and 30522 rows.
constexpr int kClearThreads = 136 * 4096;

struct ClearParams {
  void* grad;
  int type, width;
  long long rows, stride;
  long long begin, end;        // this launch's share: aligned 16-byte words where rows touch, else rows
  int dense;                   // rows touch
  int head, tail;              // 2-byte pieces before and behind the words, cleared with the first of them
  int ctas;                    // CTAs of the launch that clear
};

struct SortParams {
  const void* ids;             // of the first pass; later passes read keys
  int id_bits;
  const unsigned* keys;
  const unsigned* places;
  unsigned* out_keys;
  unsigned* out_places;
  unsigned* counts;            // [runs][digits]
  int count, runs;
  int shift, digits;           // digits: 2^bits
  int bits, passes;
  int each;                    // a thread's tokens (sort_cluster_kernel)
  int scanned;                 // counts are places already (scan_counts_kernel)
  unsigned rows;
  long long padding;
  unsigned* status;
  unsigned* joined;            // counters of the sums, cleared by the first launch
  long long counters;
  ClearParams clear;
};

__device__ void clear_share(const ClearParams& c, int cta) {
  if (c.dense) {
    unsigned short* edge = static_cast<unsigned short*>(c.grad);
    uint4* w = reinterpret_cast<uint4*>(edge + c.head);
    if (c.begin == 0 && cta == 0 && threadIdx.x < 8) {
      if ((int)threadIdx.x < c.head) edge[threadIdx.x] = 0;
      unsigned short* end = edge + c.rows * c.width * (type_bytes(c.type) / 2) - c.tail;
      if ((int)threadIdx.x < c.tail) end[threadIdx.x] = 0;
    }
    for (long long i = c.begin + (long long)cta * blockDim.x + threadIdx.x; i < c.end; i += (long long)c.ctas * blockDim.x)
      w[i] = make_uint4(0u, 0u, 0u, 0u);
  } else {
    const bool fits = aligned4(c.grad, c.type) && c.stride % 4 == 0;
    const Raw4 zero = {{0u, 0u, 0u, 0u}};
    for (long long r = c.begin + cta; r < c.end; r += c.ctas) {
      char* row = static_cast<char*>(c.grad) + r * c.stride * type_bytes(c.type);
      for (int col = 4 * threadIdx.x; col < c.width; col += 4 * blockDim.x)
        store_raw4(row, c.type, col, c.width, fits && col + 4 <= c.width, zero);
    }
  }
}

constexpr int kClearCta = 512;
__global__ void __launch_bounds__(kClearCta) clear_kernel(const __grid_constant__ ClearParams c) {
  wait_for_previous_launch();
  clear_share(c, blockIdx.x);
}

// The sort's key of a token: its row, or `rows` for one that is left out.
__device__ __forceinline__ unsigned key_of(const SortParams& p, long long id) {
  if (id < 0 || id == p.padding) return p.rows;
  if (id >= (long long)p.rows) {
    if (p.status != nullptr) atomicOr(p.status, QADAM_ST_INDEX);
    return p.rows;
  }
  return (unsigned)id;
}

// Keys of the N tokens first, first + step, ...; 0 behind the last.  All loads are under way before the first is
// looked at.
template <int N>
__device__ __forceinline__ void load_keys(const SortParams& p, long long first, int step, unsigned (&key)[N]) {
  if (p.keys != nullptr) {
#pragma unroll
    for (int j = 0; j < N; ++j) key[j] = first + j * step < p.count ? p.keys[first + j * step] : 0u;
    return;
  }
  long long id[N];
#pragma unroll
  for (int j = 0; j < N; ++j) id[j] = first + j * step < p.count ? load_id(p.ids, p.id_bits, first + j * step) : 0;
#pragma unroll
  for (int j = 0; j < N; ++j) key[j] = key_of(p, id[j]);
}

__device__ __forceinline__ void clear_counters(const SortParams& p, int cta, int ctas) {
  for (long long i = (long long)cta * blockDim.x + threadIdx.x; i < p.counters; i += (long long)ctas * blockDim.x) p.joined[i] = 0u;
}

// Quads of tokens that each warp of rank_kernel goes over.
__host__ __device__ inline int rank_quads(int count) { return (count + 4 * kRankWarps - 1) / (4 * kRankWarps); }

// Few tokens: a token's place is the number of tokens before it, by row and place in one number (`shift` bits
// of place).  T^2 comparisons of a cycle or two on all lanes.
__global__ void __launch_bounds__(kRankThreads) rank_kernel(const __grid_constant__ SortParams p) {
  wait_for_previous_launch();
  extern __shared__ uint4 ranked[];                        // p.count numbers, filled up with the largest
  __shared__ unsigned before[kRankWarps][kRankPer];
  const int ctas = (p.count + kRankPer - 1) / kRankPer;
  if ((int)blockIdx.x >= ctas) {
    clear_share(p.clear, blockIdx.x - ctas);
    return;
  }
  clear_counters(p, blockIdx.x, ctas);
  unsigned* all = reinterpret_cast<unsigned*>(ranked);
  const int four = rank_quads(p.count);
  for (int t0 = threadIdx.x; t0 < 4 * kRankWarps * four; t0 += 8 * kRankThreads) {
    unsigned key[8];
    load_keys<8>(p, t0, kRankThreads, key);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int t = t0 + j * kRankThreads;
      if (t < 4 * kRankWarps * four) all[t] = t < p.count ? key[j] << p.shift | (unsigned)t : 0xFFFFFFFFu;
    }
  }
  __syncthreads();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int mine = blockIdx.x * kRankPer + lane;
  const unsigned x0 = all[min(mine, p.count - 1)], x1 = all[min(mine + 32, p.count - 1)];
  unsigned n0 = 0u, n1 = 0u;
#pragma unroll 4
  for (int q = warp * four; q < (warp + 1) * four; ++q) {
    const uint4 y = ranked[q];
    n0 += y.x < x0 ? 1u : 0u;
    n1 += y.x < x1 ? 1u : 0u;
    n0 += y.y < x0 ? 1u : 0u;
    n1 += y.y < x1 ? 1u : 0u;
    n0 += y.z < x0 ? 1u : 0u;
    n1 += y.z < x1 ? 1u : 0u;
    n0 += y.w < x0 ? 1u : 0u;
    n1 += y.w < x1 ? 1u : 0u;
  }
  before[warp][lane] = n0;
  before[warp][lane + 32] = n1;
  __syncthreads();
  const int t = blockIdx.x * kRankPer + threadIdx.x;
  if (threadIdx.x >= kRankPer || t >= p.count) return;
  unsigned n = 0u;
#pragma unroll
  for (int w = 0; w < kRankWarps; ++w) n += before[w][threadIdx.x];
  p.out_keys[n] = all[t] >> p.shift;
  p.out_places[n] = (unsigned)t;
}

// Lanes whose token has the same digit; a lane without a token has no peer but such lanes.  A ballot for each bit: with
// a match of the whole digit place_kernel took 24 us in place of 14 (200001 tokens).
__device__ __forceinline__ unsigned peers_of(unsigned digit, int bits, bool live) {
  unsigned peers = __ballot_sync(0xFFFFFFFFu, live);
  if (!live) peers = ~peers;
#pragma unroll
  for (int b = 0; b < kDigitBits; ++b) {
    if (b >= bits) break;
    const unsigned with = __ballot_sync(0xFFFFFFFFu, ((digit >> b) & 1u) != 0u);
    peers &= with ^ (((digit >> b) & 1u) - 1u);
  }
  return peers;
}

// A warp's tokens of a run, in order: each one's rank among the warp's tokens of its digit.  seen: the warp's count of
// each digit, 0 before.
template <int ITEMS>
__device__ __forceinline__ void rank_tokens(const unsigned (&key)[ITEMS], const bool (&live)[ITEMS], int shift, int bits,
                                            unsigned short* seen, unsigned short (&rank)[ITEMS]) {
  const int lane = threadIdx.x % 32;
#pragma unroll
  for (int j = 0; j < ITEMS; ++j) {
    const unsigned d = (key[j] >> shift) & ((1u << bits) - 1u);
    const unsigned peers = peers_of(d, bits, live[j]);
    const int before = __popc(peers & ((1u << lane) - 1u));
    const int had = seen[d];
    __syncwarp();
    if (live[j] && before == 0) seen[d] = (unsigned short)(had + __popc(peers));
    __syncwarp();
    rank[j] = (unsigned short)(had + before);
  }
}

// The warps' counts of a digit to where their tokens begin among the run's of that digit; the run's count is returned.
template <int WARPS>
__device__ __forceinline__ unsigned spread_counts(unsigned short (*seen)[kDigits], int d) {
  unsigned at = 0u;
#pragma unroll
  for (int w0 = 0; w0 < WARPS; w0 += 16) {
    unsigned n[16];
#pragma unroll
    for (int w = 0; w < 16; ++w) n[w] = seen[w0 + w][d];
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      seen[w0 + w][d] = (unsigned short)at;
      at += n[w];
    }
  }
  return at;
}

// Exclusive running sum of one number per thread over the first `digits` threads.
template <int WARPS>
__device__ __forceinline__ unsigned scan_digits(unsigned x, unsigned* warp_total) {
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  unsigned upto = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned other = __shfl_up_sync(0xFFFFFFFFu, upto, o);
    if (lane >= o) upto += other;
  }
  if (lane == 31) warp_total[warp] = upto;
  __syncthreads();
  unsigned at = upto - x;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) at += w < warp ? warp_total[w] : 0u;
  return at;
}

// All passes in one launch, by a cluster: every CTA has a run of tokens in registers and sends them to where they
// belong in the CTAs' shared memory.  Sorting leaves most of the GPU to what is cleared meanwhile.  8192 tokens: 16 us
// beside 94 MB of clearing, 27 us in four launches one after the other; 32768 tokens: 24 and 27 us.
template <int ITEMS>
__global__ void __launch_bounds__(kSortThreads) sort_cluster_kernel(const __grid_constant__ SortParams p) {
  wait_for_previous_launch();
  static_assert(kDigits <= kSortThreads, "a digit to a thread");
  extern __shared__ uint2 exchange[];                      // [kSortThreads * each]
  __shared__ unsigned short seen[kSortWarps][kDigits];
  __shared__ unsigned counts[kDigits], start[kDigits], warp_total[kSortWarps];
  if (blockIdx.x >= kCluster) {
    clear_share(p.clear, blockIdx.x - kCluster);
    return;
  }
  const cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
  const int cta = (int)cluster.block_rank();
  clear_counters(p, cta, kCluster);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const unsigned slots = kSortThreads * p.each;
  const int inside = warp * 32 * p.each + lane, base = cta * (int)slots + inside;
  // x / slots is the high word of x over, as x (over slots - 2^32) < x slots < 2^32
  const unsigned over = 0xFFFFFFFFu / slots + 1u;
  unsigned key[ITEMS], place[ITEMS];
  bool live[ITEMS];
  unsigned short rank[ITEMS];
  load_keys<ITEMS>(p, base, 32, key);
#pragma unroll
  for (int j = 0; j < ITEMS; ++j) {
    live[j] = j < p.each && base + 32 * j < p.count;
    place[j] = (unsigned)(base + 32 * j);
  }
  for (int pass = 0; pass < p.passes; ++pass) {
    const int shift = pass * p.bits;
    const bool last = pass + 1 == p.passes;
    for (int i = threadIdx.x; i < kSortWarps * kDigits / 2; i += kSortThreads) reinterpret_cast<unsigned*>(&seen[0][0])[i] = 0u;
    __syncthreads();
    if (pass > 0) {
#pragma unroll
      for (int j = 0; j < ITEMS; ++j)
        if (live[j]) {
          const uint2 e = exchange[inside + 32 * j];
          key[j] = e.x;
          place[j] = e.y;
        }
    }
    rank_tokens<ITEMS>(key, live, shift, p.bits, seen[warp], rank);
    __syncthreads();
    const int d = threadIdx.x;
    if (d < p.digits) counts[d] = spread_counts<kSortWarps>(seen, d);
    cluster.sync();                                        // counts are there; all tokens have left `exchange`
    unsigned all = 0u, earlier = 0u;
    if (d < p.digits) {
#pragma unroll
      for (int c = 0; c < kCluster; ++c) {
        const unsigned n = cluster.map_shared_rank(counts, c)[d];
        if (c < cta) earlier += n;
        all += n;
      }
    }
    const unsigned before = scan_digits<kSortWarps>(all, warp_total);
    if (d < p.digits) start[d] = before + earlier;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < ITEMS; ++j)
      if (live[j]) {
        const unsigned digit = (key[j] >> shift) & (p.digits - 1);
        const unsigned to = start[digit] + seen[warp][digit] + rank[j];
        if (last) {
          p.out_keys[to] = key[j];
          p.out_places[to] = place[j];
        } else {
          const unsigned there = __umulhi(to, over);
          cluster.map_shared_rank(exchange, there)[to - there * slots] = make_uint2(key[j], place[j]);
        }
      }
    cluster.sync();                                        // tokens have arrived; counts have been read
  }
}

// Many tokens: at most 9 bits a pass, lowest first.  Counts of each digit in each CTA's run of tokens; then
// every token to its place, behind all smaller digits and the same digit in earlier runs.
__global__ void __launch_bounds__(kSortThreads) count_digits_kernel(const __grid_constant__ SortParams p) {
  wait_for_previous_launch();
  __shared__ unsigned n[kDigits];
  if ((int)blockIdx.x >= p.runs) {
    clear_share(p.clear, blockIdx.x - p.runs);
    return;
  }
  if (p.keys == nullptr) clear_counters(p, blockIdx.x, p.runs);
  for (int d = threadIdx.x; d < p.digits; d += kSortThreads) n[d] = 0u;
  unsigned key[kSortItems];
  const long long first = (long long)blockIdx.x * kSortRun + threadIdx.x;
  load_keys<kSortItems>(p, first, kSortThreads, key);
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kSortItems; ++j)
    if (first + j * kSortThreads < p.count) atomicAdd(&n[(key[j] >> p.shift) & (p.digits - 1)], 1u);
  __syncthreads();
  for (int d = threadIdx.x; d < p.digits; d += kSortThreads) p.counts[(size_t)blockIdx.x * p.digits + d] = n[d];
}

// Counts to places for very many runs, by one CTA: a digit to a thread.
__global__ void __launch_bounds__(kSortThreads) scan_counts_kernel(unsigned* counts, int runs, int digits) {
  wait_for_previous_launch();
  static_assert(kDigits <= kSortThreads, "a digit to a thread");
  __shared__ unsigned warp_total[kSortWarps];
  const int d = threadIdx.x;
  unsigned n = 0u;
  if (d < digits) {
#pragma unroll 8
    for (int r = 0; r < runs; ++r) n += counts[(size_t)r * digits + d];
  }
  unsigned at = scan_digits<kSortWarps>(n, warp_total);
  if (d >= digits) return;
#pragma unroll 8
  for (int r = 0; r < runs; ++r) {
    const unsigned c = counts[(size_t)r * digits + d];
    counts[(size_t)r * digits + d] = at;
    at += c;
  }
}

__global__ void __launch_bounds__(kSortThreads) place_kernel(const __grid_constant__ SortParams p) {
  wait_for_previous_launch();
  __shared__ unsigned short seen[kSortWarps][kDigits];
  __shared__ unsigned start[kDigits], warp_total[kSortWarps];
  if ((int)blockIdx.x >= p.runs) {
    clear_share(p.clear, blockIdx.x - p.runs);
    return;
  }
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  for (int i = threadIdx.x; i < kSortWarps * kDigits / 2; i += kSortThreads) reinterpret_cast<unsigned*>(&seen[0][0])[i] = 0u;
  unsigned key[kSortItems], place[kSortItems];
  bool live[kSortItems];
  unsigned short rank[kSortItems];
  const long long base = (long long)blockIdx.x * kSortRun + warp * (32 * kSortItems) + lane;
  load_keys<kSortItems>(p, base, 32, key);
#pragma unroll
  for (int j = 0; j < kSortItems; ++j) {
    live[j] = base + 32 * j < p.count;
    place[j] = p.places == nullptr ? (unsigned)(base + 32 * j) : live[j] ? p.places[base + 32 * j] : 0u;
  }
  // this thread's digit in all runs, and in the runs before this one
  const int digit = threadIdx.x;
  unsigned earlier = 0u, all = 0u;
  if (digit < p.digits) {
    const unsigned* counts = p.counts + digit;
    if (p.scanned) {
      earlier = counts[(size_t)blockIdx.x * p.digits];
    } else {
      for (int r0 = 0; r0 < p.runs; r0 += 32) {
        unsigned x[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) x[j] = r0 + j < p.runs ? counts[(size_t)(r0 + j) * p.digits] : 0u;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          if (r0 + j == (int)blockIdx.x) earlier = all;
          all += x[j];
        }
      }
    }
  }
  const unsigned before = scan_digits<kSortWarps>(all, warp_total);          // (a barrier: `seen` is 0 everywhere)
  if (digit < p.digits) start[digit] = before + earlier;
  rank_tokens<kSortItems>(key, live, p.shift, p.bits, seen[warp], rank);
  __syncthreads();
  if (digit < p.digits) spread_counts<kSortWarps>(seen, digit);
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kSortItems; ++j) {
    if (live[j]) {
      const unsigned d = (key[j] >> p.shift) & (p.digits - 1);
      const unsigned to = start[d] + seen[warp][d] + rank[j];
      p.out_keys[to] = key[j];
      p.out_places[to] = place[j];
    }
  }
}

// ---------------------------------------------------------------- gradient: sums
//
// The sorted tokens are cut into chunks of at most 32.  A warp takes one chunk in a tile of columns, 16 bytes to a
// lane, and adds up the rows that begin in its chunk, following the last one into the next chunk.  Only a row that
// covers whole chunks beyond the one that it begins in is split: it leaves a partial sum in each of its chunks.
// Whoever leaves the last one in a group of 32 chunks adds up the group's, and whoever does that last adds up the
// groups': in the order of the tokens, whoever it is.

constexpr int kChunk = 32;
constexpr int kSumThreads = 128;
constexpr int kSumWarps = kSumThreads / 32;
constexpr int kAhead = 8;                                  // rows a warp has asked for
constexpr int kGroup = 32;                                 // chunks

struct GradParams {
  const unsigned* keys;        // sorted; `rows` behind the last
  const unsigned* places;
  int count, chunk, chunks;    // chunk: tokens
  const void* dy;
  int dy_type;
  long long dy_stride;
  float scale;
  void* grad;
  int grad_type;
  long long rows, grad_stride;
  int width, tiles;            // tiles: of 512 bytes of dy
  int vector, grad_vector;     // rows of dy are aligned to 16 bytes; of the gradient to four elements (1), to 16 bytes (2)
  int accumulate;
  float* partial;              // [chunks][2][tiles * columns]: of the row that began in an earlier chunk, of the one that goes on
  unsigned* joined;            // [3 chunks][tiles]: partial sums left in the group that begins there (2), groups
};

// A lane's columns: neighbours where rows are aligned to 16 bytes, else 32 apart, so that a warp's accesses stay
// next to each other.
template <int COLS>
struct Columns {
  int first;                   // column of k = 0
  int step;
  __device__ Columns(const GradParams& p, int tile) {
    const int lane = threadIdx.x % 32;
    step = p.vector ? 1 : 32;
    first = tile * 32 * COLS + (p.vector ? lane * COLS : lane);
  }
  __device__ int at(int k) const { return first + k * step; }
  __device__ bool together(int width) const { return step == 1 && first + COLS <= width; }
};

template <int TYPE>
constexpr int kCols = TYPE == QADAM_F32 ? 4 : 8;           // in 16 bytes

template <int TYPE>
__device__ __forceinline__ void row_floats(const uint4& r, float (&x)[kCols<TYPE>]) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
  if constexpr (TYPE == QADAM_F32) {
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = __uint_as_float(w[k]);
  } else if constexpr (TYPE == QADAM_BF16) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[2 * k] = __uint_as_float(w[k] << 16);
      x[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[2 * k] = half_bits_to_float(w[k] & 0xFFFFu);
      x[2 * k + 1] = half_bits_to_float(w[k] >> 16);
    }
  }
}

// A lane's parts of up to kGather rows that are not 16 aligned bytes, into its slots: all loads are under way before the
// first is stored.
constexpr int kGather = 4;
template <int COLS>
__device__ __noinline__ void gather_rows(uint4* slots, unsigned slot, const unsigned long long* where, int rows, Columns<COLS> c, int width) {
  // columns and rows that are not there take the last one's place: what becomes of them is not used
  unsigned v[kGather][COLS];
#pragma unroll
  for (int r = 0; r < kGather; ++r) {
    const void* row = reinterpret_cast<const void*>(where[min(r, rows - 1)]);
#pragma unroll
    for (int k = 0; k < COLS; ++k) {
      const int at = min(c.at(k), width - 1);
      if constexpr (COLS == 4) v[r][k] = static_cast<const uint32_t*>(row)[at];
      else v[r][k] = static_cast<const unsigned short*>(row)[at];
    }
  }
#pragma unroll
  for (int r = 0; r < kGather; ++r) {
    if (r >= rows) break;
    uint4 w;
    if constexpr (COLS == 4) w = make_uint4(v[r][0], v[r][1], v[r][2], v[r][3]);
    else w = make_uint4(v[r][0] | v[r][1] << 16, v[r][2] | v[r][3] << 16, v[r][4] | v[r][5] << 16, v[r][6] | v[r][7] << 16);
    slots[(slot + r) * 32] = w;
  }
}

__device__ __forceinline__ char* grad_row(const GradParams& p, unsigned row) {
  return static_cast<char*>(p.grad) + (long long)row * p.grad_stride * type_bytes(p.grad_type);
}

template <int COLS>
struct Sum {
  float x[COLS];
};

// A row's last step where its columns are not all there, or not aligned.
template <int COLS>
__device__ __noinline__ void finish_row_apart(const GradParams& p, char* dst, Columns<COLS> c, Sum<COLS> sum) {
#pragma unroll
  for (int k = 0; k < COLS; ++k) {
    const int col = c.at(k);
    if (col >= p.width) break;
    float x[4] = {__fmul_rn(p.scale, sum.x[k]), 0.0f, 0.0f, 0.0f};
    if (p.accumulate) {
      float old[4];
      to_floats(load_raw4(dst, p.grad_type, col, col + 1, false), p.grad_type, old);
      x[0] = __fadd_rn(old[0], x[0]);
    }
    store_raw4(dst, p.grad_type, col, col + 1, false, from_floats(x, p.grad_type));
  }
}

template <int COLS>
__device__ __forceinline__ void finish_row(const GradParams& p, unsigned row, const Columns<COLS>& c, const Sum<COLS>& sum) {
  char* dst = grad_row(p, row);
  if (p.grad_vector == 0 || !c.together(p.width)) {
    if (c.first < p.width) finish_row_apart<COLS>(p, dst, c, sum);
    return;
  }
  float x[COLS];
#pragma unroll
  for (int k = 0; k < COLS; k += 2) {
    const float2 r = mul2_rn(make_float2(sum.x[k], sum.x[k + 1]), make_float2(p.scale, p.scale));
    x[k] = r.x;
    x[k + 1] = r.y;
  }
  if (p.grad_type == QADAM_F32) {
    float4* out = reinterpret_cast<float4*>(dst) + c.first / 4;
#pragma unroll
    for (int q = 0; q < COLS / 4; ++q) {
      float4 r = make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
      if (p.accumulate) {
        const float4 old = out[q];
        r = make_float4(__fadd_rn(old.x, r.x), __fadd_rn(old.y, r.y), __fadd_rn(old.z, r.z), __fadd_rn(old.w, r.w));
      }
      out[q] = r;
    }
    return;
  }
  uint32_t w[COLS / 2];
#pragma unroll
  for (int q = 0; q < COLS; q += 4) {
    float y[4] = {x[q], x[q + 1], x[q + 2], x[q + 3]};
    if (p.accumulate) {
      float old[4];
      to_floats(load_raw4(dst, p.grad_type, c.first + q, 0, true), p.grad_type, old);
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] = __fadd_rn(old[k], y[k]);
    }
    const Raw4 r = p.grad_type == QADAM_BF16 ? from_floats(y, QADAM_BF16) : from_floats(y, QADAM_F16);
    w[q / 2] = r.w[0];
    w[q / 2 + 1] = r.w[1];
  }
  if (COLS == 8 && p.grad_vector == 2) {
    *reinterpret_cast<uint4*>(dst + (size_t)c.first * 2) = make_uint4(w[0], w[1], w[COLS / 2 - 2], w[COLS / 2 - 1]);
  } else {
#pragma unroll
    for (int q = 0; q < COLS; q += 4) reinterpret_cast<uint2*>(dst)[(c.first + q) / 4] = make_uint2(w[q / 2], w[q / 2 + 1]);
  }
}

// Partial sums lie lane by lane.
template <int COLS>
__device__ __forceinline__ float4* partial_of(const GradParams& p, int chunk, int which, int tile) {
  return reinterpret_cast<float4*>(p.partial + ((((long long)chunk * 2 + which) * p.tiles + tile) * 32 + threadIdx.x % 32) * COLS);
}

// First place in [lo, hi) whose key is not below `key` (AFTER: is above it), by the whole warp.
template <bool AFTER>
__device__ __forceinline__ int search(const unsigned* keys, unsigned key, int lo, int hi) {
  const int lane = threadIdx.x % 32;
  while (lo < hi) {
    const int step = (hi - lo + 31) / 32;
    const long long at = (long long)lo + (long long)lane * step;
    const unsigned k = keys[min(at, (long long)hi - 1)];
    const int n = __popc(__ballot_sync(0xFFFFFFFFu, at < hi && (AFTER ? k <= key : k < key)));
    if (n == 0) return lo;
    hi = (int)min((long long)hi, (long long)lo + (long long)n * step);
    lo += (n - 1) * step + 1;
  }
  return lo;
}

// Counts a partial sum that this warp has left; true if it is the last of `of`, whose sums can then be read.
// The lanes' stores come before the count of lane 0 (release), the sums that others counted before the reads (acquire).
__device__ __forceinline__ bool left_last(unsigned* counter, int of) {
  __syncwarp();
  unsigned n = 0u;
  if (threadIdx.x % 32 == 0) asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(n) : "l"(counter) : "memory");
  n = __shfl_sync(0xFFFFFFFFu, n, 0);
  __syncwarp();
  return n == (unsigned)of - 1u;
}

template <int COLS>
__device__ __forceinline__ void add_left(const GradParams& p, int chunk, bool begins, int tile, Sum<COLS>& sum) {
  const float4* from = partial_of<COLS>(p, chunk, begins ? 1 : 0, tile);
#pragma unroll
  for (int q = 0; q < COLS / 4; ++q) {
    const float4 x = __ldcg(from + q);
    sum.x[4 * q] = __fadd_rn(sum.x[4 * q], x.x);
    sum.x[4 * q + 1] = __fadd_rn(sum.x[4 * q + 1], x.y);
    sum.x[4 * q + 2] = __fadd_rn(sum.x[4 * q + 2], x.z);
    sum.x[4 * q + 3] = __fadd_rn(sum.x[4 * q + 3], x.w);
  }
}

// This chunk's part of a split row.  Its group's chunks of the row: those that begin with the row, and the one before
// them if it ends with it.
template <int COLS>
__device__ __forceinline__ void leave_part(const GradParams& p, unsigned row, int chunk, int tile, Columns<COLS> c, Sum<COLS> sum) {
  const int lane = threadIdx.x % 32, group = chunk / kGroup * kGroup;
  const long long head = (long long)(group + lane) * p.chunk;
  const bool with = group + lane < p.chunks && p.keys[head] == row;              // chunk `group + lane` begins with the row
  const bool more = group + lane < p.chunks && head > 0 && p.keys[head - 1] == row;      // and the one before ends with it
  const unsigned begins = __ballot_sync(0xFFFFFFFFu, with), follows = __ballot_sync(0xFFFFFFFFu, with && more);
  // `begins` is a run of ones, or empty where the row begins in the group's last chunk
  int first = begins == 0u ? kGroup - 1 : __ffs(begins) - 1;
  const int last = begins == 0u ? kGroup - 1 : 31 - __clz(begins);
  const bool before = begins != 0u && ((follows >> first) & 1u) != 0u;           // the row began before chunk `first`
  const bool in_group = begins == 0u || first > 0 || !before;                     // the row begins in this group
  if (before && first > 0) --first;
  const int g0 = group + first, g1 = group + last;
  const bool starts = in_group && chunk == g0;
  float4* out = partial_of<COLS>(p, chunk, starts ? 1 : 0, tile);
#pragma unroll
  for (int q = 0; q < COLS / 4; ++q) out[q] = make_float4(sum.x[4 * q], sum.x[4 * q + 1], sum.x[4 * q + 2], sum.x[4 * q + 3]);
  if (!left_last(p.joined + ((long long)g0 * 2 + (in_group ? 1 : 0)) * p.tiles + tile, g1 - g0 + 1)) return;
#pragma unroll
  for (int k = 0; k < COLS; ++k) sum.x[k] = 0.0f;
#pragma unroll 4
  for (int i = g0; i <= g1; ++i) add_left<COLS>(p, i, in_group && i == g0, tile, sum);
  const bool onward = last == kGroup - 1 && (long long)(g1 + 1) * p.chunk < p.count && p.keys[(long long)(g1 + 1) * p.chunk] == row;
  if (!in_group || onward) {
    // more groups: this one's sum takes the place of its first part
    float4* all = partial_of<COLS>(p, g0, in_group ? 1 : 0, tile);
#pragma unroll
    for (int q = 0; q < COLS / 4; ++q) all[q] = make_float4(sum.x[4 * q], sum.x[4 * q + 1], sum.x[4 * q + 2], sum.x[4 * q + 3]);
    const int row_first = in_group ? g0 : search<false>(p.keys, row, 0, group * p.chunk) / p.chunk;
    const int row_last = onward ? (search<true>(p.keys, row, (g1 + 1) * p.chunk, p.count) - 1) / p.chunk : g1;
    const int groups = row_last / kGroup - row_first / kGroup + 1;
    if (!left_last(p.joined + ((long long)p.chunks * 2 + row_first) * p.tiles + tile, groups)) return;
#pragma unroll
    for (int k = 0; k < COLS; ++k) sum.x[k] = 0.0f;
#pragma unroll 4
    for (int i = 0; i < groups; ++i) {
      const int at = max(row_first, (row_first / kGroup + i) * kGroup);
      add_left<COLS>(p, at, at == row_first, tile, sum);
    }
  }
  finish_row<COLS>(p, row, c, sum);
}

// Bound by HBM where few tokens share a row (rows of dy in, rows of the gradient out), if the loop stays short: a
// row of 512 bytes is one iteration, and everything that is the same for all lanes (addresses, where rows end) is
// worked out once per chunk.  Rows arrive through shared memory (cp.async), so that the ring of rows under way takes
// no registers.  200001 tokens of 1024 bf16 into 75 x 10^3 rows (410 MB in, 150 out): 98 us, 5.7 TB/s,
// 0.87 of the rate of a copy.
template <int TYPE>
__global__ void __launch_bounds__(kSumThreads, 7) sum_chunks_kernel(const __grid_constant__ GradParams p) {
  wait_for_previous_launch();
  constexpr int COLS = kCols<TYPE>;
  __shared__ uint4 ring[kSumWarps][kAhead][32];
  __shared__ unsigned long long address[kSumWarps][2 * kChunk];
  __shared__ unsigned rows[kSumWarps][2 * kChunk];
  const long long unit = (long long)blockIdx.x * kSumWarps + threadIdx.x / 32;
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  if (unit >= (long long)p.chunks * p.tiles) return;
  const int chunk = (int)(unit / p.tiles), tile = (int)(unit % p.tiles);
  const int begin = chunk * p.chunk, n = min(p.chunk, p.count - begin);
  const unsigned none = (unsigned)p.rows;
  // a window of 64 tokens from the chunk's first on, the rows before it and before the chunk before it
  const unsigned key0 = begin + lane < p.count ? p.keys[begin + lane] : none;
  const unsigned key1 = begin + 32 + lane < p.count ? p.keys[begin + 32 + lane] : none;
  const unsigned place0 = begin + lane < p.count ? p.places[begin + lane] : 0u;
  const unsigned place1 = begin + 32 + lane < p.count ? p.places[begin + 32 + lane] : 0u;
  const unsigned before = begin > 0 ? p.keys[begin - 1] : none;
  const unsigned long_before = begin > p.chunk ? p.keys[begin - p.chunk - 1] : none;
  const long long row_bytes = p.dy_stride * (16 / COLS);
  address[warp][lane] = reinterpret_cast<unsigned long long>(p.dy) + (unsigned long long)(place0 * row_bytes);
  address[warp][32 + lane] = reinterpret_cast<unsigned long long>(p.dy) + (unsigned long long)(place1 * row_bytes);
  rows[warp][lane] = key0;
  rows[warp][32 + lane] = key1;
  const unsigned first = __shfl_sync(0xFFFFFFFFu, key0, 0);
  if (first == none) return;
  // bit i: token i is the last of its row in the window
  const unsigned up0 = __shfl_down_sync(0xFFFFFFFFu, key0, 1), up1 = __shfl_down_sync(0xFFFFFFFFu, key1, 1);
  const unsigned second = __shfl_sync(0xFFFFFFFFu, key1, 0);
  unsigned long long ends = __ballot_sync(0xFFFFFFFFu, key0 != (lane == 31 ? second : up0));
  ends |= (unsigned long long)__ballot_sync(0xFFFFFFFFu, lane == 31 || key1 != up1) << 32;
  const int live = __popc(__ballot_sync(0xFFFFFFFFu, key0 != none)) + __popc(__ballot_sync(0xFFFFFFFFu, key1 != none));
  const bool from_before = before == first;
  const int end0 = __ffsll((long long)ends);                         // behind the first row
  const bool full = n == p.chunk;
  const bool whole = full && end0 >= n;                              // the chunk is part of one row
  const bool split_before = from_before && (whole || long_before == first);      // and leaves a partial sum here
  // tokens from .. to are this warp's: none of a row that the chunk before follows up to here, and all of its own last
  // one unless that goes on into a chunk that is part of it
  const int from = from_before && !split_before ? end0 : 0;
  const int last_end = __ffsll((long long)(ends >> (n - 1))) + n - 1;            // behind the row of the chunk's last token
  const bool split_after = full && live >= n && last_end >= 2 * p.chunk;
  const int to = min(live, split_after || (split_before && whole) ? n : last_end);
  if (from >= n || from >= live) return;
  __syncwarp();

  const Columns<COLS> c(p, tile);
  const bool together = c.together(p.width), some = c.first < p.width;
  const unsigned long long lane_bytes = (unsigned long long)c.first * (16 / COLS);
  const unsigned slot0 = (unsigned)__cvta_generic_to_shared(&ring[warp][0][lane]);
  // all lanes with columns have 16 aligned bytes of them (a lane without any asks for the row's first)
  const bool fast = __all_sync(0xFFFFFFFFu, together || !some);
  const unsigned long long column = some ? lane_bytes : 0ull;
  const unsigned long long* const where = address[warp];
  uint4* const slots = &ring[warp][0][lane];
  auto ask = [&](int i, unsigned slot) {
    if (i < to && fast)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(slot0 + slot * 512u), "l"(where[i] + column) : "memory");
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  if (p.accumulate && some) {
    // rows that will be added to are brought near while those of dy arrive
    for (int i = from; i < to; ++i)
      if (((ends >> i) & 1ull) != 0)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(grad_row(p, rows[warp][i]) + (size_t)c.first * type_bytes(p.grad_type)));
  }
#pragma unroll 1
  for (int i = 0; i < kAhead; ++i) ask(from + i, i);
  Sum<COLS> sum;
#pragma unroll
  for (int k = 0; k < COLS; ++k) sum.x[k] = 0.0f;
  bool leaves = split_before;                                        // the row's sum is a partial one
  // bit 0: this token ends its row, or what this warp has of it
  ends = (ends | 1ull << (to - 1)) >> from;
  unsigned slot = 0u;
#pragma unroll 1
  for (int i = from; i < to; ++i) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
    if (!fast && some && slot % kGather == 0u) gather_rows<COLS>(slots, slot, where + i, min(to - i, kGather), c, p.width);
    float x[COLS];
    row_floats<TYPE>(slots[slot * 32], x);
#pragma unroll
    for (int k = 0; k < COLS; k += 2) {
      const float2 r = add2_rn(make_float2(sum.x[k], sum.x[k + 1]), make_float2(x[k], x[k + 1]));
      sum.x[k] = r.x;
      sum.x[k + 1] = r.y;
    }
    ask(i + kAhead, slot);
    slot = (slot + 1) % kAhead;                            // (a multiple of kGather)
    if (((unsigned)ends & 1u) != 0u) {
      const bool goes_on = i + 1 == to && split_after;
      if (leaves || goes_on) {
        leave_part<COLS>(p, rows[warp][i], chunk, tile, c, sum);
      } else {
        finish_row<COLS>(p, rows[warp][i], c, sum);
      }
      leaves = false;
#pragma unroll
      for (int k = 0; k < COLS; ++k) sum.x[k] = 0.0f;
    }
    ends >>= 1;
  }
}

// ---------------------------------------------------------------- host side

// A chunk is 32 tokens, or fewer (down to 2) where that would leave SMs without enough warps to keep their loads in
// flight: below `kWarps` warps over 512 bytes of columns (8192 tokens added to 768 columns: 24.9 us; with twice as
// many warps 26.3, with half as many 29.6: shorter chunks split more rows).
constexpr int64_t kWarps = 148 * 8;
constexpr int kLeastChunk = 2;

struct GradLayout {
  size_t keys[2], places[2], counts, partial, joined, bytes;
  int runs, chunk, chunks;
};

int grad_layout(int64_t count, int64_t rows, int64_t width, GradLayout* l) {
  if (count < 0 || count > (int64_t)1 << 30 || rows < 1 || rows >= 0x7FFFFFFF || width < 1 || width > (int64_t)1 << 22)
    return QADAM_ERR_SIZE;
  const int64_t tiles = (width + 127) / 128;                 // 512 bytes of binary32; half as many of 16-bit types
  l->runs = (int)((count + kSortRun - 1) / kSortRun);
  int64_t room = 1;                                          // chunks of any batch up to this one
  for (int chunk = kLeastChunk;; chunk *= 2) {
    const int64_t enough = kWarps * 2 * chunk / ((width + 255) / 256);        // tokens for chunks of twice as many
    room = std::max<int64_t>(room, (std::min(count, enough) + chunk - 1) / chunk);
    l->chunk = chunk;
    if (chunk == kChunk || count < enough) break;
  }
  if (l->chunk == kChunk) room = std::max<int64_t>(room, (count + kChunk - 1) / kChunk);
  l->chunks = (int)((count + l->chunk - 1) / l->chunk);
  if (room * tiles > (int64_t)1 << 32) return QADAM_ERR_SIZE;      // (CTAs of one launch)
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
  l->joined = at;
  at += round_up256((size_t)(room * 3 * tiles) * sizeof(unsigned));
  l->partial = at;
  at += (size_t)room * 2 * ((width + 255) / 256 * 256) * sizeof(float);
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
  return enqueue_lookup(p, type == QADAM_F32 ? kDense32 : kDense16, static_cast<cudaStream_t>(stream));
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
  p.first = first; p.words = (long long)(wcode_bytes / 4);
  return enqueue_lookup(p, kx + 2, static_cast<cudaStream_t>(stream));
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
  g.count = (int)count; g.chunk = l.chunk; g.chunks = l.chunks;
  g.dy = dy; g.dy_type = dy_type; g.dy_stride = dy_stride; g.scale = scale;
  g.grad = grad; g.grad_type = grad_type; g.rows = rows; g.grad_stride = grad_stride;
  g.width = (int)width; g.accumulate = accumulate;
  const int cols = 16 / type_bytes(dy_type);
  g.tiles = (int)((width + 32 * cols - 1) / (32 * cols));

  int bits = 1;
  while ((rows >> bits) != 0) ++bits;                        // keys 0 .. rows
  int place_bits = 0;
  while (((count - 1) >> place_bits) > 0) ++place_bits;
  const bool ranked = count <= kRankTokens && bits + place_bits <= 32;
  const bool clustered = !ranked && count <= kCluster * kSortRun;
  const int passes = (bits + kDigitBits - 1) / kDigitBits, digit = (bits + passes - 1) / passes;
  const bool scanned = l.runs > kDirectRuns;

  SortParams s = {};
  ClearParams& c = s.clear;
  c.grad = grad; c.type = grad_type; c.width = (int)width; c.rows = rows; c.stride = grad_stride;
  const int64_t row_bytes = width * type_bytes(grad_type);
  // rows that touch and have a whole aligned word between them are one run of words with an edge at either end
  const int64_t to_word = -(int64_t)(reinterpret_cast<uintptr_t>(grad)) & 15, run = rows * row_bytes - to_word;
  c.dense = grad_stride == width && run >= 16;
  c.head = (int)(to_word / 2);
  c.tail = (int)(run % 16 / 2);
  // what there is to clear is dealt out evenly to the launches that sort
  const long long to_clear = accumulate ? 0 : c.dense ? run / 16 : rows;
  const int launches = count == 0 || ranked || clustered ? 1 : 2 * passes;
  int turn = 0;
  auto share = [&](int threads) {
    c.begin = to_clear * turn / launches;
    c.end = to_clear * (turn + 1) / launches;
    ++turn;
    const long long each = c.dense ? threads : 1;
    c.ctas = (int)std::min<long long>((c.end - c.begin + each - 1) / each, kClearThreads / threads);
  };
  if (count == 0) {
    share(kClearCta);
    if (c.ctas == 0) return QADAM_OK;
    return launch(clear_kernel, c.ctas, kClearCta, 0, 0, st, c) ? QADAM_OK : QADAM_ERR_CUDA;
  }
  s.ids = ids; s.id_bits = id_bits; s.count = (int)count; s.runs = l.runs; s.rows = (unsigned)rows;
  s.padding = padding; s.status = status; s.digits = 1 << digit; s.bits = digit; s.passes = passes;
  s.scanned = scanned;
  s.counts = list(l.counts);
  s.joined = list(l.joined);
  s.counters = (long long)l.chunks * 3 * g.tiles;
  s.out_keys = list(l.keys[0]);
  s.out_places = list(l.places[0]);
  if (ranked) {
    s.shift = place_bits;
    share(kRankThreads);
    if (!launch(rank_kernel, ((int)count + kRankPer - 1) / kRankPer + c.ctas, kRankThreads, (size_t)rank_quads((int)count) * kRankWarps * 16,
                0, st, s))
      return QADAM_ERR_CUDA;
  } else if (clustered) {
    // no more than the batch needs (whole calls, 8192 tokens: 2 each 27.2 us, 8 each 32.9; 20000: 5 each 38.7, 8 each 39.5)
    s.each = (int)((count + kCluster * kSortThreads - 1) / (kCluster * kSortThreads));
    share(kSortThreads);
    const auto kernel = s.each <= 2 ? sort_cluster_kernel<2> : sort_cluster_kernel<kSortItems>;
    const size_t smem = passes > 1 ? (size_t)kSortThreads * s.each * sizeof(uint2) : 0;
    // the limit of dynamic shared memory belongs to the kernel: every call that needs it raised sets the same
    if (smem > 12 * 1024 &&
        !cuda_call(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSortRun * (int)sizeof(uint2))))
      return QADAM_ERR_CUDA;
    c.ctas = (c.ctas + kCluster - 1) / kCluster * kCluster;
    if (!launch(kernel, kCluster + c.ctas, kSortThreads, smem, kCluster, st, s)) return QADAM_ERR_CUDA;
  } else {
    for (int i = 0; i < passes; ++i) {
      s.shift = i * digit;
      s.keys = i == 0 ? nullptr : list(l.keys[(i + 1) % 2]);
      s.places = i == 0 ? nullptr : list(l.places[(i + 1) % 2]);
      s.out_keys = list(l.keys[i % 2]);
      s.out_places = list(l.places[i % 2]);
      share(kSortThreads);
      if (!launch(count_digits_kernel, l.runs + c.ctas, kSortThreads, 0, 0, st, s)) return QADAM_ERR_CUDA;
      if (scanned && !launch(scan_counts_kernel, 1, kSortThreads, 0, 0, st, s.counts, l.runs, s.digits)) return QADAM_ERR_CUDA;
      share(kSortThreads);
      if (!launch(place_kernel, l.runs + c.ctas, kSortThreads, 0, 0, st, s)) return QADAM_ERR_CUDA;
    }
  }
  g.keys = s.out_keys;
  g.places = s.out_places;
  g.partial = reinterpret_cast<float*>(ws + l.partial);
  g.joined = s.joined;
  g.vector = is_aligned(dy, 16) && dy_stride % cols == 0;
  g.grad_vector = !is_aligned(grad, 4 * type_bytes(grad_type)) || grad_stride % 4 != 0 ? 0
                  : is_aligned(grad, 16) && grad_stride * type_bytes(grad_type) % 16 == 0 ? 2 : 1;
  const long long units = (long long)l.chunks * g.tiles;
  const long long grid = (units + kSumWarps - 1) / kSumWarps;
  const bool ok = dy_type == QADAM_F32    ? launch(sum_chunks_kernel<QADAM_F32>, grid, kSumThreads, 0, 0, st, g)
                  : dy_type == QADAM_BF16 ? launch(sum_chunks_kernel<QADAM_BF16>, grid, kSumThreads, 0, 0, st, g)
                                          : launch(sum_chunks_kernel<QADAM_F16>, grid, kSumThreads, 0, 0, st, g);
  return ok ? QADAM_OK : QADAM_ERR_CUDA;
}

}  // extern "C"
