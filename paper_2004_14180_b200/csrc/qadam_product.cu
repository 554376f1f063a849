// Products of rows in 8 bits with weights in 8 bits: qadam_row_product, qadam_held_product.
//
//   out[m][n] = round( a_scale[m] b_scale[n] (sum_k a[m][k] b[n][k] - zero a_sums[m]) + bias[n] (+ out[m][n]) )
//
// The sums are whole numbers of 32 bits, exact.  A packed weight of 8 bits is its code, 0 .. 128, level + 64: the codes go to
// the tensor cores as they lie in memory, as unsigned bytes, and 64 sum_k a[m][k] is taken off at the end.
//
// Few tokens are bound by the weights' bytes, many by the tensor cores' products (tcgen05, 8-bit integers) where the sum is long, and by the
// results' way out where it is short.  Tiles come by TMA, zeros where a matrix ends, so that sizes need not be multiples of anything.
#include "qadam.h"

#include <cuda.h>
#include <cooperative_groups.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "qadam_rows.cuh"

using namespace qadam;
namespace cg = cooperative_groups;

namespace {

constexpr int kChannels = 128;             // of a tile: the rows of the tensor cores' result
constexpr int kDepth = 128;                // bytes of a row in a stage
constexpr int kFewTokens = 128;            // at most: the columns of the result; more tokens take the kernel below
constexpr int kProductThreads = 192;       // a warp that loads, one that multiplies, four for the end
constexpr int kMaxStages = 8;
constexpr int kMaxSplit = 8;
constexpr unsigned kPolls = 1u << 23;      // of a wait, unless a call says otherwise: some tenths of a second at least, where a tile takes microseconds

struct ProductParams {
  const float* a_scale;
  const int* a_sums;
  const float* b_scale;
  float worth;                             // of a weight, where there is no b_scale
  int zero;
  const void* bias;
  int bias_type;
  char* out;
  int out_type;
  long long out_stride;
  int accumulate;
  long long rows, channels;
  int blocks;                              // of kDepth along the sum
  int tokens;                              // the rows rounded up to 16
  int transposed;
  int b_signed;
  int stages;
  unsigned polls;
  int missing;                             // bit r: CTA r of a cluster does not ask for its last block (tests)
  unsigned* status;
};

__device__ __forceinline__ unsigned shared_at(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void barrier_init(uint64_t* bar, unsigned count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(shared_at(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_expect(uint64_t* bar, unsigned bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(shared_at(bar)), "r"(bytes) : "memory");
}
// As if so many bytes had come.
__device__ __forceinline__ void barrier_complete(uint64_t* bar, unsigned bytes) {
  asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(shared_at(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool barrier_try(uint64_t* bar, unsigned parity) {
  unsigned ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(shared_at(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
// Gives up after so many polls, or once another thread has.
__device__ __forceinline__ bool barrier_wait(uint64_t* bar, unsigned parity, volatile int* gave_up, unsigned polls) {
  for (unsigned i = 0; i < polls; ++i) {
    if (barrier_try(bar, parity)) return true;
    if (*gave_up) return false;
  }
  *gave_up = 1;
  return false;
}

// The same for a whole warp, which goes on as one.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, unsigned parity, volatile int* gave_up, unsigned polls) {
  return __all_sync(0xFFFFFFFFu, barrier_wait(bar, parity, gave_up, polls)) != 0;
}
// For what is on its way when a kernel has given up: it has to end before memory is anyone else's.
__device__ __forceinline__ void settle(uint64_t* bar, unsigned parity) {
  for (unsigned n = 0; n < kPolls && !barrier_try(bar, parity); ++n) {}
}

__device__ __forceinline__ void load_tile(void* to, const CUtensorMap* map, int x, int y, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(shared_at(to)),
      "l"(map), "r"(x), "r"(y), "r"(shared_at(bar))
      : "memory");
}

// Where an operand lies in shared memory: rows of 128 bytes, swizzled in groups of eight (1024 bytes apart).
__device__ __forceinline__ uint64_t operand(unsigned at) {
  return (uint64_t)((at & 0x3FFFFu) >> 4) | (uint64_t)(16384u >> 4) << 16 | (uint64_t)(1024u >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

__device__ __forceinline__ void multiply(unsigned result, uint64_t a, uint64_t b, unsigned kind, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(result),
      "l"(a), "l"(b), "r"(kind), "r"((unsigned)add)
      : "memory");
}
__device__ __forceinline__ void commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(shared_at(bar)) : "memory");
}
__device__ __forceinline__ void before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Sixteen columns of the result, of the warp's 32 rows.
__device__ __forceinline__ void read_columns(unsigned from, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
        "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(from)
      : "memory");
}

// One lane of a warp whose lanes are all here.  What that lane alone issues stands in code that the warp runs as one, with values that
// are the same in all lanes: in a branch that lane 0 takes, a product cost 68 cycles to issue and a block of the sum 350 more.
__device__ __forceinline__ bool elected() {
  unsigned p;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xFFFFFFFF;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ int warp_of_thread() { return __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x / 32), 0); }

// The stages of a ring, one after the other, and the phase of their barriers.
struct RingPlace {
  int stage = 0;
  unsigned phase = 0;
  __device__ __forceinline__ void next(int stages) {
    if (++stage == stages) {
      stage = 0;
      phase ^= 1u;
    }
  }
  // How many places it has come along, modulo twice the ring.
  __device__ __forceinline__ int turns(int stages) const { return (int)phase * stages + stage; }
  __device__ __forceinline__ void back(int stages) {
    if (--stage < 0) {
      stage = stages - 1;
      phase ^= 1u;
    }
  }
};

struct ProductShared {
  uint64_t full[kMaxStages], empty[kMaxStages], done;
  unsigned result;                         // in tensor memory
  int gave_up;
};

// The end of the sums of a channel and up to N tokens, `step` apart from t on, of which those below `live` are there.
struct EndShared {
  float scale[kFewTokens];
  int less[kFewTokens];
};
template <int N>
__device__ __forceinline__ void finish(const ProductParams& p, const EndShared& e, float worth, float bias, long long channel, int t, int step,
                                       int live, const uint32_t (&sum)[N]) {
  float y[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int i = t + k * step < live ? t + k * step : t;
    y[k] = fmaf((float)(int)(sum[k] - (uint32_t)e.less[i]) * e.scale[i], worth, bias);
  }
  const long long first = t * p.out_stride + channel, next = (long long)step * p.out_stride;
  if (p.accumulate) {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (t + k * step < live) y[k] += load_one_of(p.out, p.out_type, first + k * next);
  }
  if (p.out_type == QADAM_F32) {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (t + k * step < live) store_one<QADAM_F32>(p.out, first + k * next, y[k]);
  } else if (p.out_type == QADAM_BF16) {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (t + k * step < live) store_one<QADAM_BF16>(p.out, first + k * next, y[k]);
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (t + k * step < live) store_one<QADAM_F16>(p.out, first + k * next, y[k]);
  }
}

// Few tokens: the weights' channels are the rows of the tensor cores' result, so that a tile is as wide as there are tokens.  One tile of
// kChannels x tokens to a cluster; its CTAs share the sum's blocks, so that enough SMs fetch weights, and add up in each other's
// shared memory (whole numbers: in any order the same).  1 x 4096 x 4096: 6.8 us (16.8 MB, 2.6 at the copy rate: launch, first load,
// last sum); 16 x 768 x 30522 packed codes, fp32: 5.8 us (25 MB, 3.9).
__global__ void __launch_bounds__(kProductThreads) product_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map,
                                                                  const __grid_constant__ ProductParams p) {
  extern __shared__ uint8_t raw[];
  __shared__ ProductShared s;
  __shared__ EndShared about;
  uint8_t* ring = raw + (1024u - (shared_at(raw) & 1023u)) % 1024u;
  const int warp = warp_of_thread(), lane = threadIdx.x % 32;
  cg::cluster_group cluster = cg::this_cluster();
  const int split = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const unsigned b_bytes = kChannels * kDepth, a_bytes = (unsigned)p.tokens * kDepth, stage_bytes = a_bytes + b_bytes;
  const long long channel = (long long)(blockIdx.x / split) * kChannels;
  const int from = (int)((long long)p.blocks * rank / split), to = (int)((long long)p.blocks * (rank + 1) / split);

  if (threadIdx.x == 0) {
    for (int i = 0; i < p.stages; ++i) {
      barrier_init(&s.full[i], 1);
      barrier_init(&s.empty[i], 1);
    }
    barrier_init(&s.done, 1);
    s.gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  const unsigned columns = p.tokens <= 32 ? 32 : p.tokens <= 64 ? 64 : 128;
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_at(&s.result)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  before_sync();
  __syncthreads();
  after_sync();
  const unsigned result = s.result;
  wait_for_previous_launch();

  RingPlace at;
  int loaded = 0;                          // stages' fills asked for (warp 0)
  if (warp == 0) {
    const int end = to - (p.missing >> rank & 1);
    for (int i = from; i < end; ++i, ++loaded, at.next(p.stages)) {
      if (!warp_wait(&s.empty[at.stage], at.phase ^ 1u, &s.gave_up, p.polls)) break;
      if (elected()) {
        uint8_t* b = ring + at.stage * stage_bytes;
        barrier_expect(&s.full[at.stage], stage_bytes);
        if (p.transposed) load_tile(b, &b_map, (int)channel, i * kDepth, &s.full[at.stage]);
        else load_tile(b, &b_map, i * kDepth, (int)channel, &s.full[at.stage]);
        load_tile(b + b_bytes, &a_map, i * kDepth, 0, &s.full[at.stage]);
      }
      __syncwarp();
    }
  } else if (warp == 1) {
    // result 32 bits signed; first operand by its type; second signed; sizes in eights and sixteens
    const unsigned kind = 2u << 4 | (unsigned)p.b_signed << 7 | 1u << 10 | (unsigned)p.transposed << 15 | (unsigned)(p.tokens / 8) << 17 |
                          (unsigned)(kChannels / 16) << 24;
    const unsigned step = p.transposed ? 32 * 128 / 16 : 32 / 16;
    for (int i = from; i < to; ++i, at.next(p.stages)) {
      if (!warp_wait(&s.full[at.stage], at.phase, &s.gave_up, p.polls)) break;
      after_sync();
      const unsigned b = shared_at(ring) + (unsigned)at.stage * stage_bytes;
      const uint64_t wd = operand(b), td = operand(b + b_bytes);
      if (elected()) {
#pragma unroll
        for (int k = 0; k < kDepth / 32; ++k) multiply(result, wd + (uint64_t)(k * step), td + (uint64_t)(k * 2), kind, i > from || k > 0);
        commit(&s.empty[at.stage]);
      }
      __syncwarp();
    }
    if (elected()) commit(&s.done);
    __syncwarp();
  }
  const int live = (int)p.rows;
  const long long mine = channel + warp % 4 * 32 + lane;     // a warp can read the rows of the result that its number names
  const bool in = warp >= 2 && mine < p.channels;
  float worth = p.worth, bias = 0.0f;
  if (warp >= 2) {                         // what the end needs is here when the sums are
    for (int i = threadIdx.x - 64; i < live; i += 128) {
      about.scale[i] = p.a_scale[i];
      about.less[i] = p.a_sums ? p.zero * p.a_sums[i] : 0;
    }
    if (in && p.b_scale) worth = p.b_scale[mine];
    if (in && p.bias) bias = load_one_of(p.bias, p.bias_type, mine);
  }
  __syncthreads();
  const bool ok = __all_sync(0xFFFFFFFFu, warp_wait(&s.done, 0, &s.gave_up, p.polls) && *static_cast<volatile int*>(&s.gave_up) == 0) != 0;
  after_sync();
  const unsigned from_result = result + (unsigned)(warp % 4 * 32) * 65536u;
  if (split == 1) {
    if (warp >= 2 && ok) {
      for (int t = 0; t < live; t += 16) {
        uint32_t v[16];
        read_columns(from_result + (unsigned)t, v);
        if (in) finish(p, about, worth, bias, mine, t, 1, live, v);
      }
    }
  } else {
    int* sums = reinterpret_cast<int*>(ring);              // [tokens][kChannels]; nothing is on its way into the ring any more
    const int of_warp = warp % 4 * 32 + lane;
    if (warp >= 2 && ok) {
      for (int t = 0; t < live; t += 16) {
        uint32_t v[16];
        read_columns(from_result + (unsigned)t, v);
#pragma unroll
        for (int k = 0; k < 16; ++k) sums[(t + k) * kChannels + of_warp] = (int)v[k];
      }
    }
    cluster.sync();
    if (warp >= 2) {
      bool all = true;
      for (int r = 0; r < split; ++r) all &= *cluster.map_shared_rank(&s.gave_up, r) == 0;
      if (all && in) {
        const int each = (live - rank + split - 1) / split;  // tokens that are this CTA's
        const auto add_up = [&](auto together) {
          constexpr int N = decltype(together)::value;
          for (int t = rank; t < live; t += N * split) {
            uint32_t v[N] = {};
#pragma unroll 4
            for (int r = 0; r < split; ++r) {
              const int* of = cluster.map_shared_rank(sums, r) + of_warp;
#pragma unroll
              for (int k = 0; k < N; ++k) v[k] += (uint32_t)of[(t + k * split < live ? t + k * split : t) * kChannels];
            }
            finish(p, about, worth, bias, mine, t, split, live, v);
          }
        };
        // what is on its way from other CTAs at a time: as many tokens as there are, up to eight
        if (each <= 1) add_up(std::integral_constant<int, 1>());
        else if (each <= 2) add_up(std::integral_constant<int, 2>());
        else if (each <= 4) add_up(std::integral_constant<int, 4>());
        else add_up(std::integral_constant<int, 8>());
      }
    }
    cluster.sync();
  }
  before_sync();
  __syncthreads();
  if (s.gave_up) {                         // the same for all threads: who sets it does so before the barrier
    if (warp == 0 && lane == 0) {
      for (int i = 0; i < loaded && i < p.stages; ++i) {
        at.back(p.stages);
        settle(&s.full[at.stage], at.phase);
      }
      settle(&s.done, 0);                  // (committed to in any case: behind it no product reads or writes)
      if (p.status) atomicOr(p.status, (unsigned)QADAM_ST_TIMEOUT);
    }
    __syncthreads();
  }
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(result), "r"(columns));
}

// ---------------------------------------------------------------- many tokens

// Tiles of 256 tokens x up to 256 channels to a pair of CTAs on two SMs, which multiply together: each has 128 tokens, half of the
// channels' weights in its shared memory, and the results of its 128 tokens in its tensor memory.  That halves the weights'
// way into shared memory.  The pairs go from tile to tile; results have two places, so that the end of a tile (eight warps: numbers of
// 32 bits times scales, rounded, through shared memory and out in boxes) runs beside the next one's products.  16384 x 8192 x 8192: 643 us
// (3.42 x 10^15 operations a second; twice the measured bf16 rate is 3.36), 4096 x 4096 x 4096 46 us (3.0); products alone, from shared memory as it
// is, take 0.25 us a block, with their loads 0.36: shared memory takes 32 KB in and gives 48 KB out for each block.  8192 x 768 x 2304
// (sums of six blocks): 17.8 us, of which 3.5 are start and end; before it was 18.7, without the results' stores 15.7, without their arithmetic too 13.0.
// (Weights that stay in shared memory from tile to tile, for short sums: 18.6 us, and 53 in place of 47 for 65536 x 768 x 768.)
constexpr int kPairThreads = 384;          // a warp that loads, one that multiplies, one for tensor memory, one idle, eight for the end
constexpr int kPairTokens = 256;
constexpr int kPairMaxStages = 5;
constexpr int kOperandBytes = 128 * kDepth;
constexpr int kPairStageBytes = 2 * kOperandBytes;
constexpr int kEndWarps = 8;
constexpr int kBoxBytes = 32 * 128;        // of 32 tokens, 128 bytes each
constexpr int kUnit = 64;                  // channels that a warp takes at a time
constexpr int kEndChannels = 128;          // of a tile, that a warp sees at most
// Shared memory: stages, boxes of results on their way out, what the end knows of its channels.  Five stages and one box a warp, or four and
// two: for sums of 8192 (8192 x 8192 results of 16 bits) five stages take 337 us and four 357, for sums of 768 (8192 x 768) two boxes
// take 9.9 us and one 10.7.  (Sixteen warps for the end in place of eight: no gain at 16 bits, 32 us against 25 for 8192 x 2304 fp32.)
constexpr int pair_bytes(int stages, int boxes) { return stages * kPairStageBytes + kEndWarps * (boxes * kBoxBytes + kEndChannels * 8); }
constexpr int kPairBytes = pair_bytes(4, 2);
static_assert(kPairBytes >= pair_bytes(5, 1), "");
constexpr int kLongSum = 16;               // blocks from which five stages are taken
constexpr int kTokenGroup = 8;             // tiles of so many token blocks lie next to each other in time: what they read stays in L2

struct PairParams {
  const float* a_scale;
  const int* a_sums;
  const float* b_scale;
  float worth;
  int zero;
  const void* bias;
  int bias_type;
  char* out;
  long long out_stride;
  int accumulate;
  long long rows, channels;
  int blocks;
  int half;                                // channels of a tile that a CTA's shared memory has the weights of: 32, 64, 96 or 128
  int token_tiles, channel_tiles;
  unsigned group_magic;                    // 2^32 / (kTokenGroup channel_tiles), rounded up
  int transposed, b_signed;
  int stages, boxes;
  unsigned polls;
  int missing;
  unsigned* status;
};

struct PairShared {
  uint64_t full[kPairMaxStages], empty[kPairMaxStages], result_full[2], result_empty[2];
  unsigned result;
  int gave_up;
  int asked, multiplied, ended;            // turns of the ring at the end: blocks asked for by this CTA, multiplied; of the results: tiles
};

__device__ __forceinline__ unsigned of_first(unsigned at) {                // the same place in the pair's first CTA
  unsigned r;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(at));
  return r;
}
__device__ __forceinline__ void pair_load(void* to, const CUtensorMap* map, int x, int y, unsigned bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];" ::"r"(
          shared_at(to)),
      "l"(map), "r"(x), "r"(y), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void pair_multiply(unsigned result, uint64_t a, uint64_t b, unsigned kind, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(result),
      "l"(a), "l"(b), "r"(kind), "r"((unsigned)add)
      : "memory");
}
__device__ __forceinline__ void pair_commit(uint64_t* bar) {               // arrives in both CTAs
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(shared_at(bar)),
               "h"((unsigned short)3)
               : "memory");
}
__device__ __forceinline__ void arrive_at(unsigned bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void read_unit(unsigned from, uint32_t (&v)[kUnit]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, "
      "%26, %27, %28, %29, %30, %31, %32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, %48, %49, "
      "%50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
        "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]),
        "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]),
        "=r"(v[31]), "=r"(v[32]), "=r"(v[33]), "=r"(v[34]), "=r"(v[35]), "=r"(v[36]), "=r"(v[37]), "=r"(v[38]), "=r"(v[39]), "=r"(v[40]),
        "=r"(v[41]), "=r"(v[42]), "=r"(v[43]), "=r"(v[44]), "=r"(v[45]), "=r"(v[46]), "=r"(v[47]), "=r"(v[48]), "=r"(v[49]), "=r"(v[50]),
        "=r"(v[51]), "=r"(v[52]), "=r"(v[53]), "=r"(v[54]), "=r"(v[55]), "=r"(v[56]), "=r"(v[57]), "=r"(v[58]), "=r"(v[59]), "=r"(v[60]),
        "=r"(v[61]), "=r"(v[62]), "=r"(v[63])
      : "r"(from)
      : "memory");
}
__device__ __forceinline__ void store_box(const CUtensorMap* map, const void* from, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(shared_at(from))
               : "memory");
}

// The same, added to what is there (binary32: one rounding, as a load, a sum and a store would have).
__device__ __forceinline__ void add_box(const CUtensorMap* map, const void* from, int x, int y) {
  asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y),
               "r"(shared_at(from))
               : "memory");
}

struct PairTile {
  int token, channel;                      // tiles
};
// (A division by multiplication, which may be one too large, and one by eight: with divisions for every tile the end of a tile took 0.3 us more.)
__device__ __forceinline__ PairTile pair_tile(const PairParams& p, int t) {
  const int wide = kTokenGroup * p.channel_tiles;
  int group = (int)__umulhi((unsigned)t, p.group_magic), in = t - group * wide;
  if (in < 0) {
    --group;
    in += wide;
  }
  const int first = group * kTokenGroup, tall = p.token_tiles - first;
  if (tall >= kTokenGroup) return {first + in % kTokenGroup, in / kTokenGroup};
  return {first + in % tall, in / tall};
}

// OUT: type of the result.  BOXES: it is written in boxes; else (rows that do not begin on 16 bytes, or 16-bit results to be added
// to, whose sums are rounded once) from shared memory element by element, 32 channels of a token at a time.
template <int OUT, bool BOXES>
__global__ void __launch_bounds__(kPairThreads, 1) pair_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map,
                                                               const __grid_constant__ CUtensorMap out_map, const __grid_constant__ PairParams p) {
  extern __shared__ uint8_t raw[];
  __shared__ PairShared s;
  uint8_t* ring = raw + (1024u - (shared_at(raw) & 1023u)) % 1024u;
  const int warp = warp_of_thread(), lane = threadIdx.x % 32;
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank();
  const int tiles = p.token_tiles * p.channel_tiles, step = gridDim.x / 2;

  if (threadIdx.x == 0) {
    for (int i = 0; i < p.stages; ++i) {
      barrier_init(&s.full[i], 1);
      barrier_init(&s.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      barrier_init(&s.result_full[i], 1);
      barrier_init(&s.result_empty[i], 2 * kEndWarps);
    }
    s.gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_at(&s.result)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
  before_sync();
  cluster.sync();
  after_sync();
  const unsigned result = s.result;
  wait_for_previous_launch();

  const unsigned b_bytes = p.transposed ? kOperandBytes : (unsigned)p.half * kDepth;
  RingPlace place;
  if (warp == 0) {
    bool ok = true;
    for (int t = blockIdx.x / 2; t < tiles && ok; t += step) {
      const PairTile tile = pair_tile(p, t);
      const int row = tile.token * kPairTokens + rank * 128, channel = tile.channel * 2 * p.half + rank * p.half;
      const int blocks = p.blocks - (t + step >= tiles ? p.missing >> rank & 1 : 0);
      for (int i = 0; i < blocks; ++i, place.next(p.stages)) {
        ok = warp_wait(&s.empty[place.stage], place.phase ^ 1u, &s.gave_up, p.polls);
        if (!ok) break;
        if (elected()) {
          uint8_t* a = ring + place.stage * kPairStageBytes;
          const unsigned bar = of_first(shared_at(&s.full[place.stage]));
          if (rank == 0) barrier_expect(&s.full[place.stage], 2 * (kOperandBytes + b_bytes));
          pair_load(a, &a_map, i * kDepth, row, bar);
          if (p.transposed) pair_load(a + kOperandBytes, &b_map, channel, i * kDepth, bar);
          else pair_load(a + kOperandBytes, &b_map, i * kDepth, channel, bar);
        }
        __syncwarp();
      }
    }
    if (lane == 0) s.asked = place.turns(p.stages);
  } else if (warp == 1 && rank == 0) {
    // result 32 bits signed; first operand signed, second by its type; sizes in eights and sixteens
    const unsigned kind = 2u << 4 | 1u << 7 | (unsigned)p.b_signed << 10 | (unsigned)p.transposed << 16 | (unsigned)(2 * p.half / 8) << 17 |
                          (unsigned)(kPairTokens / 16) << 24;
    const unsigned b_step = p.transposed ? 32 * 128 / 16 : 32 / 16;
    RingPlace turn;
    bool ok = true;
    for (int t = blockIdx.x / 2; t < tiles; t += step, turn.next(2)) {
      ok = warp_wait(&s.result_empty[turn.stage], turn.phase ^ 1u, &s.gave_up, p.polls);
      if (!ok) break;
      after_sync();
      const unsigned at = result + (unsigned)turn.stage * 256u;
      for (int i = 0; i < p.blocks; ++i, place.next(p.stages)) {
        ok = warp_wait(&s.full[place.stage], place.phase, &s.gave_up, p.polls);
        if (!ok) break;
        after_sync();
        const unsigned a = shared_at(ring) + (unsigned)place.stage * kPairStageBytes;
        const uint64_t ad = operand(a), bd = operand(a + kOperandBytes);
        if (elected()) {
#pragma unroll
          for (int k = 0; k < kDepth / 32; ++k) pair_multiply(at, ad + (uint64_t)(k * 2), bd + (uint64_t)(k * b_step), kind, i > 0 || k > 0);
          pair_commit(&s.empty[place.stage]);
          if (i + 1 == p.blocks) pair_commit(&s.result_full[turn.stage]);
        }
        __syncwarp();
      }
      if (!ok) break;
    }
    if (lane == 0) {
      s.multiplied = place.turns(p.stages);
      s.ended = turn.turns(2);
    }
  } else if (warp >= 4) {
    const int end = warp - 4, quarter = warp % 4, side = end / 4;
    uint8_t* boxes = ring + p.stages * kPairStageBytes + end * p.boxes * kBoxBytes;
    float2* about = reinterpret_cast<float2*>(ring + p.stages * kPairStageBytes + kEndWarps * p.boxes * kBoxBytes) + end * kEndChannels;   // two scales, two biases, ...
    constexpr bool kWide = BOXES && OUT != QADAM_F32;                        // a box has 64 channels of 16 bits, or 32 of 32 bits
    // what the end of a tile needs to know is asked for while the tile before it is at its end
    float2 channels[kEndChannels / 32];
    float a_scale = 0.0f;
    int less = 0;
    const auto ask = [&](int t) {
      if (t >= tiles) return;
      const PairTile tile = pair_tile(p, t);
      const int row = tile.token * kPairTokens + rank * 128 + quarter * 32 + lane;
      a_scale = row < (int)p.rows ? p.a_scale[row] : 0.0f;
      less = row < (int)p.rows && p.a_sums ? p.a_sums[row] : 0;
#pragma unroll
      for (int i = 0; i < kEndChannels / 32; ++i) {                          // this warp's: every other unit of the tile
        const int n = i * 32 + lane, c = (n / kUnit * 2 + side) * kUnit + n % kUnit;
        const int at = tile.channel * 2 * p.half + c;
        channels[i] = make_float2(p.worth, 0.0f);
        if (c < 2 * p.half && at < (int)p.channels) {
          if (p.b_scale) channels[i].x = p.b_scale[at];
          if (p.bias) channels[i].y = load_one_of(p.bias, p.bias_type, at);
        }
      }
    };
    ask(blockIdx.x / 2);
    RingPlace turn;
    int flip = 0;
    for (int t = blockIdx.x / 2; t < tiles; t += step, turn.next(2)) {
      const PairTile tile = pair_tile(p, t);
      const long long row0 = (long long)tile.token * kPairTokens + rank * 128 + quarter * 32;
      const long long channel0 = (long long)tile.channel * 2 * p.half;
      const int wide = (int)min((long long)2 * p.half, p.channels - channel0);
      __syncwarp();
#pragma unroll
      for (int i = 0; i < kEndChannels / 32; ++i) {
        float* to = reinterpret_cast<float*>(about) + (i * 32 + (lane & ~1)) * 2 + (lane & 1);
        to[0] = channels[i].x;
        to[2] = channels[i].y;
      }
      const float times = a_scale;
      const int off = less * p.zero;
      __syncwarp();
      if (!warp_wait(&s.result_full[turn.stage], turn.phase, &s.gave_up, p.polls)) break;
      after_sync();
      ask(t + step);
      const unsigned at = result + (unsigned)turn.stage * 256u + (unsigned)(quarter * 32) * 65536u;
      for (int j = 0; (j * 2 + side) * kUnit < wide; ++j) {
        const int c0 = (j * 2 + side) * kUnit;
        uint8_t* box = boxes + (kWide ? flip * kBoxBytes : 0);
        uint32_t v[kUnit];
        read_unit(at + (unsigned)c0, v);
        if constexpr (BOXES) {             // (this one's box has been read)
          if (kWide && p.boxes == 2) {
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
            flip ^= 1;
          } else {
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
          }
        }
        __syncwarp();
        const float4* f = reinterpret_cast<const float4*>(about + j * kUnit);
        uint8_t* line = box + lane * 128;
#pragma unroll
        for (int k = 0; k < kUnit; k += 8) {
          float y[8];
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            const float4 g = f[(k + i) / 2];
            const float2 sum = make_float2((float)((int)v[k + i] - off), (float)((int)v[k + i + 1] - off));
            const float2 z = fma2_rn(mul2_rn(sum, make_float2(times, times)), make_float2(g.x, g.y), make_float2(g.z, g.w));
            y[i] = z.x;
            y[i + 1] = z.y;
          }
          if constexpr (kWide) {
            store_raw8<OUT == QADAM_F32 ? QADAM_BF16 : OUT>(line + (((k / 8) ^ (lane & 7)) << 4), floats_to_raw8<OUT == QADAM_F32 ? QADAM_BF16 : OUT>(y));
          } else {
#pragma unroll
            for (int i = 0; i < 8; i += 4)
              *reinterpret_cast<float4*>(line + (k / 32) * kBoxBytes + ((((k + i) / 4 % 8) ^ (lane & 7)) << 4)) = make_float4(y[i], y[i + 1], y[i + 2], y[i + 3]);
          }
        }
        if constexpr (BOXES) {
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            if (row0 < p.rows) {
              if (!kWide && p.accumulate) {
                add_box(&out_map, box, (int)(channel0 + c0), (int)row0);
                if (c0 + 32 < wide) add_box(&out_map, box + kBoxBytes, (int)(channel0 + c0 + 32), (int)row0);
              } else {
                store_box(&out_map, box, (int)(channel0 + c0), (int)row0);
                if (!kWide && c0 + 32 < wide) store_box(&out_map, box + kBoxBytes, (int)(channel0 + c0 + 32), (int)row0);
              }
            }
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
          }
        } else {
          __syncwarp();
          const int live = (int)min((long long)32, p.rows - row0);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const bool in = c0 + h * 32 + lane < wide;
            char* to = p.out + (row0 * p.out_stride + channel0 + c0 + h * 32 + lane) * (OUT == QADAM_F32 ? 4 : 2);
            const long long row_bytes = p.out_stride * (OUT == QADAM_F32 ? 4 : 2);
#pragma unroll 1
            for (int r = 0; r < live; r += 16) {               // sixteen tokens' loads under way, if there is something to add to
              float y[16];
#pragma unroll
              for (int i = 0; i < 16; ++i) y[i] = p.accumulate && in && r + i < live ? load_one<OUT>(to + i * row_bytes, 0) : 0.0f;
#pragma unroll
              for (int i = 0; i < 16; ++i)
                y[i] += *reinterpret_cast<const float*>(box + h * kBoxBytes + (r + i) * 128 + (((lane / 4) ^ ((r + i) & 7)) << 4) + lane % 4 * 4);
#pragma unroll
              for (int i = 0; i < 16; ++i)
                if (in && r + i < live) store_one<OUT>(to + i * row_bytes, 0, y[i]);
              to += 16 * row_bytes;
            }
          }
          __syncwarp();
        }
      }
      before_sync();
      __syncwarp();
      if (lane == 0) arrive_at(of_first(shared_at(&s.result_empty[turn.stage])));
    }
    if constexpr (BOXES) {
      if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
  }
  if (*static_cast<volatile int*>(&s.gave_up)) *cluster.map_shared_rank(&s.gave_up, rank ^ 1) = 1;         // (who gave up comes by here afterwards)
  before_sync();
  cluster.sync();
  after_sync();
  if (s.gave_up) {                         // in both, then
    if (warp == 0 && lane == 0) {
      // The first CTA's barriers count both's copies, and one may have asked for more blocks than the other, both for no more than there are stages
      // since the last one that was multiplied: what only the second has asked for is expected alone, what only the first has is counted as there.
      const int ring = 2 * p.stages, multiplied = *cluster.map_shared_rank(&s.multiplied, 0), ended = *cluster.map_shared_rank(&s.ended, 0);
      const int first = (*cluster.map_shared_rank(&s.asked, 0) - multiplied + ring) % ring;
      const int second = (*cluster.map_shared_rank(&s.asked, 1) - multiplied + ring) % ring;
      if (rank == 0) {
        for (int i = 0; i < max(first, second); ++i) {
          const int at = (multiplied + i) % ring;
          uint64_t* full = &s.full[at % p.stages];
          if (i >= first) barrier_expect(full, kOperandBytes + b_bytes);
          if (i >= second) barrier_complete(full, kOperandBytes + b_bytes);
          settle(full, (unsigned)(at / p.stages));
        }
        if (p.status) atomicOr(p.status, (unsigned)QADAM_ST_TIMEOUT);
      }
      // products end in the order in which they were begun, each block's, and each tile's, with a commit to both CTAs (a place that nothing has come
      // by yet counts as left behind)
      const int last = (multiplied + ring - 1) % ring, tile = (ended + 3) % 4;
      settle(&s.empty[last % p.stages], (unsigned)(last / p.stages));
      settle(&s.result_full[tile % 2], (unsigned)(tile / 2));
    }
    __syncwarp();
    cluster.sync();
  }
  if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(result), "r"(512));
}

// ---------------------------------------------------------------- launches

using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                            const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

Encode encoder() {
  static std::atomic<Encode> known{nullptr};
  Encode e = known.load();
  if (e) return e;
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult found;
  if (!cuda_call(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found)) || found != cudaDriverEntryPointSuccess) return nullptr;
  e = reinterpret_cast<Encode>(fn);
  known.store(e);
  return e;
}

// A matrix of results, written in boxes of 32 rows of 128 bytes.
bool box_map(CUtensorMap* map, void* p, int type, int64_t channels, int64_t rows, int64_t stride) {
  const Encode encode = encoder();
  if (!encode) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)channels, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)(stride * type_bytes(type))};
  const cuuint32_t box[2] = {type == QADAM_F32 ? 32u : 64u, 32u}, unit[2] = {1, 1};
  return encode(map, type == QADAM_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : type == QADAM_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                2, p, dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A matrix of bytes [rows][stride], of which a copy takes boxes of 128 x `box_rows`; what lies beyond it reads as zero.
bool byte_map(CUtensorMap* map, const void* p, int64_t width, int64_t rows, int64_t stride, int box_rows) {
  const Encode encode = encoder();
  if (!encode) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)stride};
  const cuuint32_t box[2] = {128, (cuuint32_t)box_rows}, unit[2] = {1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(p), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// CTAs of a cluster wait for one another while they hold tensor memory, so no SM may be given more of those than its 512 columns serve.  Their
// shared memory sees to it.  Where few tokens share a sum, a CTA has two stages or more: up to 32 tokens 32 columns and 36 KB, up to 64
// 64 and 44 KB, up to 128 128 and 52 KB; pairs 512 columns and 201 KB, beside which none of those fits.  (A CTA with one stage does, or several, and may
// have to wait for columns, or a pair for its.  But one stage means one block, a sum that is not shared: it holds columns only while it waits
// for nothing but its own copies, and gives them back.)
constexpr int kSmBytes = 228 * 1024;
constexpr int two_stages(int tokens) { return 2 * (kChannels + tokens) * kDepth; }
static_assert(kPairBytes + two_stages(16) > kSmBytes, "no CTA that shares a sum beside a pair's");
static_assert(4 * two_stages(80) + two_stages(16) > kSmBytes, "the least that more than 512 columns of CTAs that share sums come with");
constexpr int kRingBytes = 208 * 1024;

using PairKernel = void (*)(CUtensorMap, CUtensorMap, CUtensorMap, PairParams);
constexpr PairKernel kPairKernels[3][2] = {{pair_kernel<QADAM_F32, false>, pair_kernel<QADAM_F32, true>},
                                           {pair_kernel<QADAM_BF16, false>, pair_kernel<QADAM_BF16, true>},
                                           {pair_kernel<QADAM_F16, false>, pair_kernel<QADAM_F16, true>}};

// Once for each device: how much shared memory the kernels may take; the pairs of SMs that there are.
constexpr int kDevices = 64;
int pairs_of_device() {
  static std::atomic<int> known[kDevices];
  int device = 0;
  if (!cuda_call(cudaGetDevice(&device))) return 0;
  std::atomic<int>& pairs = known[device % kDevices];
  if (const int n = pairs.load()) return n;
  if (!cuda_call(cudaFuncSetAttribute(product_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes + 1024))) return 0;
  for (const auto& of_type : kPairKernels)
    for (const PairKernel kernel : of_type)
      if (!cuda_call(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPairBytes + 1024))) return 0;
  cudaLaunchConfig_t config = {};
  config.gridDim = dim3(2);
  config.blockDim = dim3(kPairThreads);
  config.dynamicSmemBytes = kPairBytes + 1024;
  cudaLaunchAttribute cluster;
  cluster.id = cudaLaunchAttributeClusterDimension;
  cluster.val.clusterDim.x = 2;
  cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
  config.attrs = &cluster;
  config.numAttrs = 1;
  int n = 0;
  if (!cuda_call(cudaOccupancyMaxActiveClusters(&n, kPairKernels[0][0], &config)) || n < 1) return 0;
  pairs.store(n);
  return n;
}

constexpr int kSms = 148;

// What a block of 128 bytes along the sum takes a CTA, in cycles: its products (16384 operations a cycle: four for each of the 128
// rows that a CTA's results have), or the way of its operands into shared memory, at 64 bytes a cycle, whichever is longer.
int64_t block_cycles(int columns, int loaded_rows) { return std::max<int64_t>(2 * columns, 2 * loaded_rows); }
constexpr int kTileCycles = 1500;          // what a tile costs besides

// Channels of a pair's tile: the time of the pairs' rounds is to be least.  (Of transposed weights a copy takes 128 channels whatever `half` is.
// Counting those would choose wider tiles on fewer SMs, which take longer: 2048 x 4096 x 768 14.7 us in place of 12.2, 8192 x 768 x 768
// 10.5 in place of 9.6, 620 x 142 x 532 11.2 in place of 7.2; 5498 x 4436 x 134 would take 21.1 in place of 23.3.)
struct PairShape {
  int half;
  int64_t cycles;
};
PairShape pair_shape(int64_t rows, int64_t channels, int blocks, int pairs) {
  PairShape best = {128, INT64_MAX};
  const int64_t token_tiles = (rows + kPairTokens - 1) / kPairTokens;
  for (int half = 128; half >= 32; half -= 32) {             // (whole boxes of results)
    const int64_t tiles = token_tiles * ((channels + 2 * half - 1) / (2 * half));
    const int64_t cycles = (tiles + pairs - 1) / pairs * (blocks * block_cycles(2 * half, 128 + half) + kTileCycles);
    if (cycles < best.cycles) best = {half, cycles};
  }
  return best;
}

// How many CTAs share the sum of a tile of few tokens: as many as there are SMs for, up to eight, as long as each has two blocks.
struct FewShape {
  int tokens, split, resident;             // resident: CTAs of an SM
  int64_t cycles;
};
FewShape few_shape(int64_t rows, int64_t channels, int blocks) {
  FewShape f;
  f.tokens = (int)(rows + 15) / 16 * 16;
  const int64_t tiles = (channels + kChannels - 1) / kChannels;
  f.resident = f.tokens <= 32 ? 2 : 1;
  const int resident = f.resident;
  f.split = 1;
  while (f.split < kMaxSplit && tiles * f.split * 2 <= (int64_t)resident * kSms && blocks >= f.split * 4) f.split *= 2;
  const int64_t rounds = (tiles * f.split + resident * kSms - 1) / (resident * kSms);
  f.cycles = rounds * resident * ((blocks + f.split - 1) / f.split * block_cycles(f.tokens, kChannels + f.tokens) + kTileCycles) + (f.split > 1 ? 2500 : 0);
  return f;
}

int enqueue_pairs(const ProductParams& q, const int8_t* a, int64_t a_stride, int64_t depth, const void* b, int64_t b_stride, int pairs, cudaStream_t st) {
  PairParams p = {};
  p.a_scale = q.a_scale; p.a_sums = q.a_sums; p.b_scale = q.b_scale; p.worth = q.worth; p.zero = q.zero; p.bias = q.bias; p.bias_type = q.bias_type;
  p.out = q.out; p.out_stride = q.out_stride; p.accumulate = q.accumulate; p.rows = q.rows; p.channels = q.channels; p.blocks = q.blocks;
  p.transposed = q.transposed; p.b_signed = q.b_signed; p.polls = q.polls; p.missing = q.missing; p.status = q.status;
  p.token_tiles = (int)((p.rows + kPairTokens - 1) / kPairTokens);
  p.half = pair_shape(p.rows, p.channels, p.blocks, pairs).half;
  p.channel_tiles = (int)((p.channels + 2 * p.half - 1) / (2 * p.half));
  p.group_magic = (unsigned)((((uint64_t)1 << 32) + kTokenGroup * (uint64_t)p.channel_tiles - 1) / (kTokenGroup * (uint64_t)p.channel_tiles));
  const int64_t out_pitch = p.out_stride * type_bytes(q.out_type);
  const bool boxes = (!p.accumulate || q.out_type == QADAM_F32) && is_aligned(p.out, 16) && out_pitch % 16 == 0 && out_pitch < (int64_t)1 << 40;
  p.boxes = boxes && q.out_type != QADAM_F32 && p.blocks >= kLongSum ? 1 : 2;
  p.stages = p.boxes == 1 ? 5 : 4;
  CUtensorMap a_map, b_map, out_map = {};
  const bool maps = byte_map(&a_map, a, depth, p.rows, a_stride, 128) &&
                    (p.transposed ? byte_map(&b_map, b, p.channels, depth, b_stride, kDepth) : byte_map(&b_map, b, depth, p.channels, b_stride, p.half)) &&
                    (!boxes || box_map(&out_map, p.out, q.out_type, p.channels, p.rows, p.out_stride));
  if (!maps) return QADAM_ERR_CUDA;
  const int64_t tiles = (int64_t)p.token_tiles * p.channel_tiles;
  if (tiles >= (int64_t)1 << 30) return QADAM_ERR_SIZE;
  return launch(kPairKernels[q.out_type][boxes], 2 * std::min<int64_t>(tiles, pairs), kPairThreads, kPairBytes + 1024, 2, st, a_map, b_map, out_map, p)
             ? QADAM_OK : QADAM_ERR_CUDA;
}

int enqueue_product(ProductParams& p, const int8_t* a, int64_t a_stride, int64_t depth, const void* b, int64_t b_stride, cudaStream_t st) {
  p.blocks = (int)((depth + kDepth - 1) / kDepth);
  const int pairs = pairs_of_device();
  if (pairs == 0) return QADAM_ERR_CUDA;
  // up to 32 tokens the pairs' 256 are a waste in any case; up to 128 it is the longer sum's or the many channels' turn
  const FewShape few = few_shape(p.rows, p.channels, p.blocks);
  if (p.rows > kFewTokens || (p.rows > 32 && pair_shape(p.rows, p.channels, p.blocks, pairs).cycles <= few.cycles))
    return enqueue_pairs(p, a, a_stride, depth, b, b_stride, pairs, st);
  const int tokens = few.tokens, split = few.split;
  const int64_t tiles = (p.channels + kChannels - 1) / kChannels;
  p.tokens = tokens;
  const int stage = (kChannels + tokens) * kDepth;
  const int needed = (p.blocks + split - 1) / split;
  p.stages = std::min({kMaxStages, kRingBytes / few.resident / stage, std::max(needed, (tokens * kChannels * 4 + stage - 1) / stage)});
  if (tiles * split >= (int64_t)1 << 31) return QADAM_ERR_SIZE;
  CUtensorMap a_map, b_map;
  const bool maps = byte_map(&a_map, a, depth, p.rows, a_stride, tokens) &&
                    (p.transposed ? byte_map(&b_map, b, p.channels, depth, b_stride, kDepth) : byte_map(&b_map, b, depth, p.channels, b_stride, kChannels));
  if (!maps) return QADAM_ERR_CUDA;
  return launch(product_kernel, tiles * split, kProductThreads, (size_t)p.stages * stage + 1024, split, st, a_map, b_map, p) ? QADAM_OK : QADAM_ERR_CUDA;
}

constexpr int64_t kMostRows = ((int64_t)1 << 31) - 512, kMostDepth = 131072;                         // (places in a tile's rows stay below 2^31)

int check_product(const qadam_product_args& p) {
  if (p.rows < 0 || p.rows > kMostRows || p.channels < 1 || p.channels > kMostRows || p.depth < 1 || p.depth > kMostDepth) return QADAM_ERR_SIZE;
  if ((p.transposed != 0 && p.transposed != 1) || (p.accumulate != 0 && p.accumulate != 1)) return QADAM_ERR_SIZE;
  if (p.wait_polls < 0 || p.test_missing_blocks < 0 || p.test_missing_blocks >= 1 << kMaxSplit) return QADAM_ERR_SIZE;
  if (!known_type(p.out_type) || (p.bias && !known_type(p.bias_type))) return QADAM_ERR_TYPE;
  if (p.rows > 0 && (!p.a || !p.a_scale || !p.out)) return QADAM_ERR_NULL;
  if (p.a_stride < p.depth || p.a_stride >= (int64_t)1 << 40 || p.out_stride < p.channels || p.out_stride > (int64_t)1 << 40) return QADAM_ERR_SIZE;
  if (!is_aligned(p.a, 16) || p.a_stride % 16 != 0 || !is_aligned(p.a_scale, 4) || (p.bias && !is_aligned(p.bias, type_bytes(p.bias_type))) ||
      !is_aligned(p.out, type_bytes(p.out_type)) || !is_aligned(p.status, 4))
    return QADAM_ERR_ALIGN;
  return QADAM_OK;
}

ProductParams product_params(const qadam_product_args& g) {
  ProductParams p = {};
  p.a_scale = g.a_scale;
  p.bias = g.bias; p.bias_type = g.bias_type;
  p.out = static_cast<char*>(g.out); p.out_type = g.out_type; p.out_stride = g.out_stride; p.accumulate = g.accumulate;
  p.rows = g.rows; p.channels = g.channels; p.transposed = g.transposed; p.status = g.status;
  p.polls = g.wait_polls ? (unsigned)g.wait_polls : kPolls; p.missing = g.test_missing_blocks;
  return p;
}

}  // namespace

extern "C" {

int qadam_row_product(const qadam_product_args* args, void* stream) {
  if (!args) return QADAM_ERR_NULL;
  const qadam_product_args& g = *args;
  const int rc = check_product(g);
  if (rc != QADAM_OK) return rc;
  if (g.rows > 0 && !g.b) return QADAM_ERR_NULL;
  if (g.transposed && g.b_scale) return QADAM_ERR_SIZE;
  if (g.b_stride < (g.transposed ? g.channels : g.depth) || g.b_stride >= (int64_t)1 << 40) return QADAM_ERR_SIZE;
  if (!is_aligned(g.b, 16) || g.b_stride % 16 != 0 || !is_aligned(g.b_scale, 4)) return QADAM_ERR_ALIGN;
  if (g.rows == 0) return QADAM_OK;
  ProductParams p = product_params(g);
  p.b_scale = g.b_scale; p.worth = g.b_worth; p.b_signed = 1;
  return enqueue_product(p, g.a, g.a_stride, g.depth, g.b, g.b_stride, static_cast<cudaStream_t>(stream));
}

int qadam_held_product(const qadam_product_args* args, void* stream) {
  if (!args) return QADAM_ERR_NULL;
  const qadam_product_args& g = *args;
  const int rc = check_product(g);
  if (rc != QADAM_OK) return rc;
  if (g.kx != 6) return QADAM_ERR_LEVEL;
  if (!g.b || (g.rows > 0 && !g.a_sums)) return QADAM_ERR_NULL;
  const int64_t width = g.transposed ? g.channels : g.depth, table = g.transposed ? g.depth : g.channels;
  if (!is_aligned(g.b, 16) || g.first % 16 != 0 || width % 16 != 0 || !is_aligned(g.a_sums, 4)) return QADAM_ERR_ALIGN;
  if (g.first < 0 || g.wcode_bytes < 0 || g.first > g.wcode_bytes || table > (g.wcode_bytes - g.first) / width) return QADAM_ERR_SIZE;
  if (g.rows == 0) return QADAM_OK;
  ProductParams p = product_params(g);
  p.a_sums = g.a_sums; p.zero = 64; p.worth = 1.0f / 128.0f; p.b_signed = 0;
  return enqueue_product(p, g.a, g.a_stride, g.depth, static_cast<const uint8_t*>(g.b) + g.first, width, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
