// filter.cu - sampling rules per row: top-k, top-p and min-p on softmax(z / T)
// (memspec_op_sample_filtered, memspec_op_filter_logits).
//
// Order a row's ids by descending logit, equal logits by ascending id.  Each rule keeps a
// prefix of that order and all of them together the shortest: top-k the first k; top-p the
// shortest whose weights (expfix.cuh) hold p of the sum over the first k; min-p the ids
// with weight >= min_p of the largest.  So a rule's result is a cut (key, id): an id is
// kept if its logit's key is larger, or equal and its id not above the cut's.
//
// A cluster of C = 1, 2, 4 or 8 CTAs per row; each keeps its slice of the row in shared
// memory, so that the row is read once however many passes its rule takes:
//   1. load; the maximum, and a bound: if each CTA has j groups of threads with a logit
//      above its bound, C j logits of the row lie above the least of the bounds;
//   2. top-k up to some hundred: the candidates, the logits above the bound (two or three
//      times as many as top-k keeps), are listed; the list holds what the rule keeps, and
//      each entry is counted against the others for its place in the order, the sum of
//      weights before it and, among the kept ones, the sum before it in id order;
//   3. top-p alone, draws: the candidates are listed the same way and the sum of the rest is
//      formed roughly, by one ex2 each.  If the candidates hold p of the sum they are all
//      that is looked at (end_of); if they hold most of it, the ids a few octaves below them
//      are queued and searched alone (search_above).  Draws under larger k queue the ids
//      above the bound, or a little below it, and search those by count, then by weights;
//   4. else a search per part (top-k, then top-p among what top-k left): a histogram of the
//      elements.  For top-k counts, by depth below the maximum, 16 bins an octave of it; for
//      top-p counts and sums of weights (exact in 64 bits by two 32-bit atomics), by weight, nine
//      bins an octave of it (the queues of 3. have bins of one width).  The CTAs add up each other's
//      bins through distributed shared memory to find the bin with the cut, and list
//      its elements - or all up to there, where they are few enough; top-p alone lists
//      candidates on the way (masks), and is done where they hold p of the sum.  A bin with
//      more than the list takes (flat rows, many equal logits) is divided by key as often as
//      it needs; a single key, by id;
//   5. the draw: from the list where it holds all that is kept, else the kept weights' sums
//      slice by slice, then warp by warp; or the mask.
// Every CTA of a cluster takes the same decisions from the same numbers, so no result is
// passed back but an id among more equal logits than the list takes, and what the first
// CTA found where it goes on alone.
//
// Measured (us, one launch in a graph; 4 V bytes a row at 6780 GB/s are 0.02 to 11):
//                       no cut  top-k 50  k, p  k 1000, p 0.9  top-p 0.9  flat, top-p 0.9
//     1 x  32000           5.5       6.9   7.6          15.4       14.3             17.9
//     1 x 128256           9.6       7.9   8.7          19.3       14.9             30.2
//    16 x 128256          14.1      10.2  11.3          25.5       22.5             42.5
//   144 x 128256          56.2      36.2  37.3          84.4       76.2            161.8
// (op_sample, which knows no rule, takes 19.1 for the last one without a cut; greedy rows 32.2
// here, 13.3 there.)  One row is bound by latency: load, three to ten barriers of the cluster at
// 0.7 us each, list and draw.  A batch is bound by how rows are held: a row keeps a cluster of 8
// CTAs and its shared memory from load to draw, 51 rows fit, so that 144 run in three waves whose
// CTAs load, then wait, then search together.  An SM has a CTA for 70 to 79% of the time, and
// then 37 to 47% of its issue slots are used; warps wait at barriers most, without a cut for the
// weights' arithmetic (50 instructions an element, 8 of them load and maximum, some 30 the weight;
// 8 for a rough weight).
#include <cuda_runtime.h>

#include <math.h>
#include <stddef.h>

#include <atomic>
#include <string>

#include "../../include/memspec_ops.h"
#include "expfix.cuh"
#include "internal.h"
#include "ptx.cuh"

namespace memspec {
namespace {

constexpr int kMaxVocab = 131072;
constexpr int kMaxSlice = 16388;             // floats of a CTA's slice: three CTAs per SM
constexpr int kMaxCluster = 8;
constexpr uint32_t kCopyBytes = 16384;
constexpr float kLargest = 3.402823466e38f;
constexpr int kBins = 416;                   // of a search's histogram
constexpr int kBinBits = 8;                  // of one that divides a bin
constexpr int kSupers = kBins / 32;          // groups of 32 bins
constexpr int kMantissa = 4;                 // counts: 16 bins an octave of max - z, from 2^-10 on
constexpr int kFirstOctave = (127 - 10) << kMantissa;
constexpr int kPlacesPerBin = 28;            // weights: a bin per ninth of log2 of the weight
static_assert(-kNoWeight / kPlacesPerBin <= kBins, "every weight has a bin");
constexpr uint32_t kList = 256;              // list entries of a CTA and of the cluster
constexpr int kQueue = 4 * kList;            // places in the slice, in the list's memory
constexpr int kGroups = 64;                  // groups of threads whose maxima give the bound
constexpr int kMostAbove = 56;               // of them above it at most
constexpr int kMostBelow = 200;              // of logits of a CTA an octave below the bound
constexpr int kTopPAbove = 96;               // logits above the bound for top-p alone (144 rows of 32000:
                                             // 31 us; with 112 the queues overflow, 50; with 80 at p =
                                             // 0.95 43 against 39)

typedef unsigned long long u64;

// NaN as -inf, +inf as the largest finite number.
__device__ __forceinline__ float sane(float z) { return fminf(fmaxf(z, -INFINITY), kLargest); }

struct alignas(16) Smem {
  u64 table[kExpSteps];
  union {
    struct {
      uint32_t cnt[kBins], lo[kBins], hi[kBins];     // count, sum of weights in two words
    } h;
    u64 entry[2][kList];                     // the cluster's list, and sorted
    struct {
      u64 weight[kList];                     // draw_from_list: weights in the rule's order,
      uint32_t by_id[2][kList];              // ids with places in it, and sorted
    } d;
  };
  union {
    struct {                                 // find_bin: the sums of all CTAs
      u64 mass[kMaxCluster][32];
      uint32_t cnt[kMaxCluster][32];
    } p;
    uint16_t queue[kQueue];                  // then places in the slice, of a bin to divide
    u64 list[kList];                         // then this CTA's entries: (~key << 32) | id
  };
  // of this CTA, read by the others
  uint32_t sup_cnt[kSupers];
  u64 sup_mass[kSupers];
  u64 sum, listed_sum;                       // of the slice's weights, of the candidates'
  uint32_t n_list, n_candidates, n_queue;
  uint2 peer_max[kMaxCluster];               // pushed: keys of the maximum and the bound
  float2 log_min_p;                          // T log(min_p) in two floats, scaled
  u64 peer_sum[kMaxCluster];                 // pushed
  u64 scan[48];
  uint32_t group[kGroups];                   // keys
  uint64_t loaded;                           // mbarrier of the slice's copies
  uint32_t tie_id;                           // pushed
  u64 cut;
  u64 deep_sum;                              // of the slice's weights below a bound, roughly; read by the others
};
static_assert(3 * (sizeof(Smem) + kMaxSlice * 4 + 1024) <= 228 * 1024, "three CTAs per SM");
// Shared memory begins on a 16-byte boundary: what is accessed by 8 bytes (plainly or from other
// CTAs) lies on multiples of 8, the slice behind it, by 16, on one of 16.
static_assert(offsetof(Smem, table) % 8 == 0 && offsetof(Smem, h) % 8 == 0 && offsetof(Smem, p) % 8 == 0 &&
                  offsetof(Smem, sup_mass) % 8 == 0 && offsetof(Smem, sum) % 8 == 0 &&
                  offsetof(Smem, listed_sum) % 8 == 0 && offsetof(Smem, deep_sum) % 8 == 0 &&
                  offsetof(Smem, peer_max) % 8 == 0 && offsetof(Smem, log_min_p) % 8 == 0 &&
                  offsetof(Smem, peer_sum) % 8 == 0 && offsetof(Smem, scan) % 8 == 0 &&
                  offsetof(Smem, loaded) % 8 == 0 && offsetof(Smem, cut) % 8 == 0 && sizeof(Smem) % 16 == 0 &&
                  offsetof(Smem, entry) == offsetof(Smem, h) && offsetof(Smem, d) == offsetof(Smem, h) &&
                  offsetof(Smem, list) == offsetof(Smem, p) && offsetof(Smem, queue) == offsetof(Smem, p),
              "aligned");

// A row's rule, with what "off" means resolved.
struct Rule {
  float temperature, top_p, min_p;
  int top_k;
};
__device__ __forceinline__ Rule rule_of(const FilterArgs& a, int row) {
  const int i = row / a.rows_per_rule;
  Rule r;
  r.temperature = a.temperatures != nullptr ? a.temperatures[i] : a.temperature;
  r.top_k = a.top_ks != nullptr ? a.top_ks[i] : a.top_k;
  r.top_p = a.top_ps != nullptr ? a.top_ps[i] : a.top_p;
  r.min_p = a.min_ps != nullptr ? a.min_ps[i] : a.min_p;
  if (!(r.temperature > 0.f)) {   // greedy: the first id of the largest logit
    r.temperature = 1.f;
    r.top_k = 1;
    r.top_p = 1.f;
    r.min_p = 0.f;
  }
  r.temperature = fmaxf(r.temperature, kLowest);
  return r;
}

// ------------------------------------------------ sums over a warp and a CTA of NT threads
__device__ __forceinline__ u64 warp_sum(u64 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <class T>
__device__ __forceinline__ T warp_scan(T v) {   // inclusive
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T n = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += n;
  }
  return v;
}
// N sums over the block, to thread 0.
template <int NT, int N>
__device__ void block_sums(u64 (&v)[N], u64* scratch) {
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = warp_sum(v[k]);
  __syncthreads();
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int k = 0; k < N; ++k) scratch[k * (NT / 32) + (threadIdx.x >> 5)] = v[k];
  __syncthreads();
  if (threadIdx.x > 0) return;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    v[k] = 0;
#pragma unroll
    for (int i = 0; i < NT / 32; ++i) v[k] += scratch[k * (NT / 32) + i];
  }
}
// Inclusive sum over the threads up to this one; *total over all.
template <int NT>
__device__ u64 block_scan(u64 v, u64* scratch, u64* total) {
  const u64 incl = warp_scan(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 31) scratch[threadIdx.x >> 5] = incl;
  __syncthreads();
  u64 before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < NT / 32; ++i) {
    const u64 x = scratch[i];
    if (i < static_cast<int>(threadIdx.x >> 5)) before += x;
    all += x;
  }
  *total = all;
  return before + incl;
}
// The n <= kList different values of `in`, ascending, to `out`: each counted against the
// others by as many threads as there are to an entry (a bitonic network took twice as long
// at 100 entries).  `in` is padded with larger values to rank_padded(n).  All threads.
template <int NT>
__device__ __forceinline__ int rank_bits(uint32_t n) {   // 2^bits threads to an entry, 16 at most
  int bits = 0;
  while (bits < 4 && n << (bits + 1) <= NT) ++bits;
  return bits;
}
template <int NT>
__device__ __forceinline__ uint32_t rank_padded(uint32_t n) {
  const uint32_t step = 8u << rank_bits<NT>(n);
  return (n + step - 1) & ~(step - 1);
}
static_assert(kList % (8 << 4) == 0, "the padding fits the list");
template <int NT, class T>
__device__ void rank_sort(const T* in, T* out, uint32_t n) {
  const int bits = rank_bits<NT>(n);
  const uint32_t i = threadIdx.x >> bits, part = threadIdx.x & ((1u << bits) - 1), end = rank_padded<NT>(n);
  uint32_t rank = 0;
  T v{};
  if (i < n) {
    v = in[i];
    for (uint32_t j = part; j < end; j += 8u << bits) {
      T x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = in[j + (u << bits)];
#pragma unroll
      for (int u = 0; u < 8; ++u) rank += x[u] < v;
    }
  }
  for (int o = 1 << bits >> 1; o > 0; o >>= 1) rank += __shfl_xor_sync(0xffffffffu, rank, o);
  if (i < n && part == 0) out[rank] = v;
  __syncthreads();
}
// All threads of the cluster: what they wrote before is read after.
__device__ __forceinline__ void cluster_sync() {
  cluster_arrive_release();
  cluster_wait_acquire();
}

// An element's place in a row's order: (~key << 32) | id.  The cut is the last kept one.
__device__ __forceinline__ u64 entry_of(uint32_t key, uint32_t id) {
  return (static_cast<u64>(~key) << 32) | id;
}
__device__ __forceinline__ float entry_logit(u64 e) { return key_logit(~static_cast<uint32_t>(e >> 32)); }

// A CTA's slice of a row in shared memory: ids base .. base + len - 1, -inf where there is
// none.
struct Slice {
  float* z;
  int base, len;            // len a multiple of 4
};

// Four elements at a time, those of which one at least reaches z_min.  Passes work on the
// four together, so that their arithmetic and their atomics overlap.
template <int NT, class Each>
__device__ __forceinline__ void for_quads(const Slice& s, float z_min, Each each) {
  const float4* z4 = reinterpret_cast<const float4*>(s.z);
  for (int i = threadIdx.x; i < s.len / 4; i += NT) {
    const float4 v = z4[i];
    if (fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)) < z_min) continue;
    const float z[4] = {v.x, v.y, v.z, v.w};
    each(z, s.base + 4 * i);
  }
}

// The same with all of a warp's threads (nothing past the end, for which z is -inf).
template <int NT, class Each>
__device__ __forceinline__ void for_warp_quads(const Slice& s, float z_min, Each each) {
  const float4* z4 = reinterpret_cast<const float4*>(s.z);
  const int quads = s.len / 4, lane = threadIdx.x & 31;
  for (int i0 = static_cast<int>(threadIdx.x) - lane; i0 < quads; i0 += NT) {
    const int i = i0 + lane;
    const float4 v = i < quads ? z4[i] : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    if (!__any_sync(0xffffffffu, fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)) >= z_min)) continue;
    const float z[4] = {v.x, v.y, v.z, v.w};
    each(z, s.base + 4 * i);
  }
}
// Places in a list for the chosen elements of a warp's quads, by one atomic.
struct Places {
  uint32_t at[4];
};
__device__ __forceinline__ bool reserve(const bool (&in)[4], uint32_t* counter, Places& p) {
  const unsigned below = (1u << (threadIdx.x & 31)) - 1;
  uint32_t all = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const unsigned m = __ballot_sync(0xffffffffu, in[q]);
    p.at[q] = all + __popc(m & below);
    all += __popc(m);
  }
  if (all == 0) return false;
  uint32_t base = 0;
  if ((threadIdx.x & 31) == 0) base = atomicAdd(counter, all);
  base = __shfl_sync(0xffffffffu, base, 0);
#pragma unroll
  for (int q = 0; q < 4; ++q) p.at[q] += base;
  return true;
}

// ------------------------------------------------ one search: top-k or top-p
struct Part {
  u64 need;                 // the count, or (weights) the fraction of the sum, in 2^-64
  int n_min;                // weights: places below this one are not the cut, only their sum counts
  float bound;              // weights of all ids: candidates are listed on the way
  u64 within;               // entries up to this one take part
};

__device__ __forceinline__ int count_bin(float depth) {
  const int b = static_cast<int>(__float_as_uint(depth) >> (23 - kMantissa)) - kFirstOctave;
  return max(0, min(b, kBins - 1));
}

// A histogram's bin that holds the cut, by the same steps in every CTA of the cluster.
struct Found {
  int bin;
  u64 above, own;           // sum (count or weights) before the bin, and its own
  uint32_t count;           // elements in it
  uint32_t count_above;     // and before it
  u64 total;                // of all bins
  u64 need;                 // what the prefix has to reach
  bool all;                 // the whole set does not exceed it (a count): nothing is cut
};

// After the histogram of every CTA is complete and the cluster has synchronised; need_of: what
// the prefix has to reach, from the sum of all bins.
template <int NT, bool kMass, class NeedOf>
__device__ Found find_bin(NeedOf need_of, int C, Smem& sm) {
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  Found f;
  // the groups' sums of all CTAs
  if (tid < C * kSupers) {
    const int peer = tid / kSupers, g = tid % kSupers;
    sm.p.cnt[peer][g] = ld_cluster_u32(mapa_shared(smem_addr(&sm.sup_cnt[g]), peer));
    if (kMass) sm.p.mass[peer][g] = ld_cluster_u64(mapa_shared(smem_addr(&sm.sup_mass[g]), peer));
  }
  __syncthreads();
  u64 v = 0;
  uint32_t n = 0;
  if (lane < kSupers)
    for (int c = 0; c < C; ++c) {
      n += sm.p.cnt[c][lane];
      if (kMass) v += sm.p.mass[c][lane];
    }
  if (!kMass) v = n;
  u64 incl = warp_scan(v);
  const uint32_t n_incl = warp_scan(n);
  const u64 total = __shfl_sync(0xffffffffu, incl, 31);
  const u64 need = need_of(total);
  f.total = total;
  f.need = need;
  f.all = !kMass && need >= total;
  const unsigned reach = __ballot_sync(0xffffffffu, lane < kSupers && incl >= need);
  const int g = reach ? __ffs(reach) - 1 : kSupers - 1;
  const u64 before = __shfl_sync(0xffffffffu, incl - v, g);
  const uint32_t n_before = __shfl_sync(0xffffffffu, n_incl - n, g);
  __syncthreads();                                        // p is read
  if (w < C) {
    sm.p.cnt[w][lane] = ld_cluster_u32(mapa_shared(smem_addr(&sm.h.cnt[g * 32 + lane]), w));
    if (kMass)
      sm.p.mass[w][lane] = ld_cluster_u32(mapa_shared(smem_addr(&sm.h.lo[g * 32 + lane]), w)) |
                           (static_cast<u64>(ld_cluster_u32(mapa_shared(smem_addr(&sm.h.hi[g * 32 + lane]), w))) << 32);
  }
  __syncthreads();
  n = 0;
  v = 0;
  for (int c = 0; c < C; ++c) {
    n += sm.p.cnt[c][lane];
    if (kMass) v += sm.p.mass[c][lane];
  }
  if (!kMass) v = n;
  incl = before + warp_scan(v);
  const unsigned hit = __ballot_sync(0xffffffffu, incl >= need);
  const int b = hit ? __ffs(hit) - 1 : 31;
  f.bin = g * 32 + b;
  f.above = __shfl_sync(0xffffffffu, incl - v, b);
  f.own = __shfl_sync(0xffffffffu, v, b);
  f.count = __shfl_sync(0xffffffffu, n, b);
  f.count_above = n_before + __shfl_sync(0xffffffffu, warp_scan(n) - n, b);
  return f;
}
static_assert(256 / 32 >= kMaxCluster && 256 >= kMaxCluster * kSupers, "a warp per CTA of the cluster");

// N elements into their bins: counts, and weights as 64-bit sums in two words.
template <bool kMass, int N>
__device__ __forceinline__ void add_to_bins(Smem& sm, const bool (&in)[N], const int (&bin)[N], const u64 (&w)[N]) {
#pragma unroll
  for (int q = 0; q < N; ++q)
    if (in[q]) atomicAdd(&sm.h.cnt[bin[q]], 1u);
  if constexpr (kMass) {
    uint32_t old[N];
#pragma unroll
    for (int q = 0; q < N; ++q) old[q] = in[q] ? atomicAdd(&sm.h.lo[bin[q]], static_cast<uint32_t>(w[q])) : 0;
#pragma unroll
    for (int q = 0; q < N; ++q) {
      const uint32_t lo = static_cast<uint32_t>(w[q]);
      const uint32_t hi = static_cast<uint32_t>(w[q] >> 32) + (old[q] + lo < old[q] ? 1u : 0u);
      if (in[q] && hi != 0) atomicAdd(&sm.h.hi[bin[q]], hi);
    }
  }
}
template <int NT>
__device__ void clear_histogram(Smem& sm) {
  uint32_t* h = reinterpret_cast<uint32_t*>(&sm.h);
  for (int i = threadIdx.x; i < static_cast<int>(sizeof(sm.h) / 4); i += NT) h[i] = 0;
  __syncthreads();
}
// The groups' sums of this CTA's histogram, then the cluster's barrier.
template <int NT, bool kMass>
__device__ void close_histogram(Smem& sm) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  __syncthreads();
  for (int g = w; g < kSupers; g += NT / 32) {
    const uint32_t n = __reduce_add_sync(0xffffffffu, sm.h.cnt[g * 32 + lane]);
    u64 m = 0;
    if (kMass) m = warp_sum(sm.h.lo[g * 32 + lane] | (static_cast<u64>(sm.h.hi[g * 32 + lane]) << 32));
    if (lane == 0) {
      sm.sup_cnt[g] = n;
      sm.sup_mass[g] = m;
    }
  }
  cluster_sync();
}

// The fraction (in 2^-64) of a sum, rounded up, but 1 at least: what a prefix has to reach.
__device__ __forceinline__ u64 part_of(u64 fraction, u64 sum) {
  return max(__umul64hi(fraction, sum) + (fraction * sum != 0 ? 1 : 0), 1ull);
}

// The CTAs' lists (`count` of each), an entry per thread (~0 past the last), sorted; returns
// how many.
template <int NT>
__device__ uint32_t pull_list(int C, const uint32_t* count, u64& e, Smem& sm) {
  // a warp per CTA: lane c has CTA c's count
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  uint32_t n = lane < C ? ld_cluster_u32(mapa_shared(smem_addr(count), lane)) : 0;
  const uint32_t incl = warp_scan(n), all = min(__shfl_sync(0xffffffffu, incl, 31), kList);
  const uint32_t off = __shfl_sync(0xffffffffu, incl - n, w);
  n = __shfl_sync(0xffffffffu, n, w);
  if (w < C)
    for (uint32_t i = lane; i < n && off + i < kList; i += 32)
      sm.entry[0][off + i] = ld_cluster_u64(mapa_shared(smem_addr(&sm.list[i]), w));
  if (threadIdx.x >= all && threadIdx.x < rank_padded<NT>(all)) sm.entry[0][threadIdx.x] = ~0ull;
  __syncthreads();
  rank_sort<NT>(sm.entry[0], sm.entry[1], all);
  e = threadIdx.x < all ? sm.entry[1][threadIdx.x] : ~0ull;
  return all;
}

// A margin for the roundings of a place or a depth, and of a logit z from it.
__device__ __forceinline__ float slack_at(float z, const WeightScale& ws) {
  return 4e-7f * (fabsf(ws.max) + fabsf(z)) + 1e-37f;
}

struct Ended {
  u64 cut;
  uint32_t listed;          // > 0: the threads hold so many sorted entries, all up to the cut among them
  u64 entry;
  bool gone;                // kAlone: this CTA has nothing more to do
};

// The entry at which the prefix that p asks for ends.  kMass: by weights, else by count;
// kWhole: every id takes part; kAlone: where all that is kept is listed, the first CTA goes
// on alone (the others' `gone`).
template <int NT, bool kMass, bool kWhole, bool kAlone>
__device__ Ended search(const Part& p, const Slice& s, const WeightScale& ws, int C, int rank, Smem& sm) {
  const int tid = threadIdx.x;
  const float z_in = kWhole ? -kLargest : entry_logit(p.within);
  const uint32_t id_in = static_cast<uint32_t>(p.within);
  auto takes_part = [&](float z, int id) {
    return kWhole ? z > -INFINITY : z > z_in || (z == z_in && static_cast<uint32_t>(id) <= id_in);
  };
  // an element's bin, or one past the last: it takes no part or is not the cut
  auto bin_of = [&](float z, int id) {
    int b;
    if (kMass) {
      float f;
      const int n = weight_place(z, ws, f);
      b = n < p.n_min ? kBins : static_cast<int>(static_cast<unsigned>(-n) / kPlacesPerBin);
    } else {
      b = count_bin(ws.max - z);
    }
    return takes_part(z, id) ? b : kBins;
  };
  if (tid == 0) {             // before the barrier in clear_histogram: the pass counts candidates
    sm.n_list = sm.n_candidates = sm.n_queue = 0;
    sm.cut = p.within;
  }
  clear_histogram<NT>(sm);
  constexpr bool kCandidates = kMass && kWhole && !kAlone;   // draws (kAlone) have tried them before
  u64 sum = 0, listed_sum = 0;
  for_quads<NT>(s, z_in, [&](const float (&z)[4], int id) {
    bool in[4];
    int bin[4];
    u64 w[4];
    if (kMass) {
      int n[4];
      float f[4];
      weight_places(z, ws, n, f);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        w[q] = weight_at(n[q], f[q], sm.table);
        if (!kWhole && !takes_part(z[q], id + q)) w[q] = 0;
        in[q] = n[q] >= p.n_min && (kWhole || w[q] != 0);
        sum += w[q];
        bin[q] = static_cast<int>(static_cast<unsigned>(-n[q]) / kPlacesPerBin);
      }
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        in[q] = takes_part(z[q], id + q);
        w[q] = 0;
        bin[q] = count_bin(ws.max - z[q]);
      }
    }
    add_to_bins<kMass>(sm, in, bin, w);
    if (kCandidates && fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])) >= p.bound) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (z[q] >= p.bound) {
          listed_sum += w[q];
          const uint32_t i = atomicAdd(&sm.n_candidates, 1u);
          if (i < kList) sm.list[i] = entry_of(logit_key(z[q]), static_cast<uint32_t>(id + q));
        }
    }
  });
  if (kMass) {
    u64 sums[2] = {sum, listed_sum};
    block_sums<NT>(sums, sm.scan);
    if (tid == 0) {
      sm.sum = sums[0];
      sm.listed_sum = sums[1];
    }
  }
  close_histogram<NT, kMass>(sm);
  u64 need = p.need;
  if (kMass) {
    // lane c: CTA c's sums
    const int lane = tid & 31;
    const bool peer = lane < C;
    need = part_of(p.need, warp_sum(peer ? ld_cluster_u64(mapa_shared(smem_addr(&sm.sum), lane)) : 0));
    if (kCandidates) {
      const uint32_t n =
          __reduce_add_sync(0xffffffffu, peer ? ld_cluster_u32(mapa_shared(smem_addr(&sm.n_candidates), lane)) : 0u);
      const u64 listed = warp_sum(peer ? ld_cluster_u64(mapa_shared(smem_addr(&sm.listed_sum), lane)) : 0);
      if (n <= kList && listed >= need) {   // what is kept is among the candidates
        u64 e, all;
        pull_list<NT>(C, &sm.n_candidates, e, sm);
        cluster_sync();       // the others have read this CTA's list and sums
        const u64 own = static_cast<uint32_t>(tid) < n ? weight(entry_logit(e), ws, sm.table) : 0;
        const u64 incl = block_scan<NT>(own, sm.scan, &all);
        if (incl - own < need && need <= incl) sm.cut = e;
        __syncthreads();
        return {sm.cut, n, e, false};
      }
    }
  }
  Found f = find_bin<NT, kMass>([&](u64) { return need; }, C, sm);
  if (f.all) {
    cluster_sync();           // the others have read this CTA's histogram
    return {p.within, 0, 0, false};
  }
  const int bin = f.bin;
  // the keys that the bin's elements can have: from the depths at its ends
  uint32_t k_lo, k_hi;
  {
    float d0, d1;             // max - z
    if (kMass) {
      d0 = static_cast<float>(bin * kPlacesPerBin - 1) / (ws.hi256 * ws.scale);
      d1 = static_cast<float>((bin + 1) * kPlacesPerBin + 1) / (ws.hi256 * ws.scale);
    } else {
      d0 = __uint_as_float(static_cast<uint32_t>(bin + kFirstOctave) << (23 - kMantissa));
      d1 = __uint_as_float(static_cast<uint32_t>(bin + 1 + kFirstOctave) << (23 - kMantissa));
    }
    const float z1 = ws.max - d0, z0 = ws.max - d1;
    const float slack = slack_at(z0, ws);
    k_hi = bin == 0 || !(z1 + slack < ws.max) ? logit_key(ws.max) : logit_key(z1 + slack);
    k_lo = (!kMass && bin == kBins - 1) || !(z0 - slack > -kLargest) ? logit_key(-kLargest) : logit_key(z0 - slack);
  }
  int shift = 32;             // keys per bin of the last division: 2^shift
  float z_lo = key_logit(k_lo), z_hi = key_logit(k_hi);
  auto narrow = [&] {         // to the keys of bin f.bin of the last division
    k_hi -= static_cast<uint32_t>(f.bin) << shift;
    if (k_hi - k_lo >= 1u << shift) k_lo = k_hi - ((1u << shift) - 1);
    z_lo = key_logit(k_lo);
    z_hi = key_logit(k_hi);
  };
  // for the draw it pays to have all of the kept elements
  const bool whole_list = kMass && f.count_above + f.count <= kList;
  // the elements of the bin (whole_list: up to it) of a quad; false: none
  auto choose = [&](const float (&z)[4], int id, bool (&in)[4]) {
    const float top = whole_list ? kLargest : z_hi;
    bool any = false;
#pragma unroll
    for (int q = 0; q < 4; ++q) any |= in[q] = z[q] >= z_lo && z[q] <= top;
    if (!any) return false;
    any = false;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int b = bin_of(z[q], id + q);
      any |= in[q] = in[q] && (whole_list ? b <= bin : b == bin);
    }
    return any;
  };
  u64 above = f.above;
  // To divide a bin, its elements' places in the slice (of those in its range of keys) are
  // queued, up to kQueued per thread, and a thread keeps its share in registers.  (A pass
  // over the slice spends its whole body on every 128 elements with one of them.)
  constexpr int kQueued = kQueue / NT;
  float mine_z[kQueued];
  int mine_id[kQueued];
  bool queued = false;
  if (f.count > kList) {
    __syncthreads();          // sm.p, in the queue's place, is read
    for_warp_quads<NT>(s, z_lo, [&](const float (&z)[4], int id) {
      bool in[4];
      Places at;
#pragma unroll
      for (int q = 0; q < 4; ++q) in[q] = z[q] >= z_lo && z[q] <= z_hi;
      if (!reserve(in, &sm.n_queue, at)) return;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (in[q] && at.at[q] < kQueue) sm.queue[at.at[q]] = static_cast<uint16_t>(id + q - s.base);
    });
    __syncthreads();
    const uint32_t n = sm.n_queue;
    queued = n <= kQueue;     // each CTA for itself
    if (queued)
#pragma unroll
      for (int q = 0; q < kQueued; ++q) {
        const uint32_t i = q * NT + tid;
        mine_z[q] = -INFINITY;
        mine_id[q] = 0;
        if (i < n) {
          const int at = sm.queue[i];
          const float z = s.z[at];
          mine_id[q] = s.base + at;
          if (bin_of(z, mine_id[q]) == bin) mine_z[q] = z;
        }
      }
  }
  while (f.count > kList) {
    if (shift == 32) {        // the first division of [k_lo, k_hi]
      shift = max(0, 32 - __clz(k_hi - k_lo) - kBinBits);
    } else {
      if (shift == 0) break;
      narrow();
      shift = max(0, shift - kBinBits);
    }
    cluster_sync();           // the others have read this CTA's histogram
    clear_histogram<NT>(sm);
    auto divide = [&](const float (&z)[4], const bool (&in)[4]) {
      int b[4];
      u64 w[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        b[q] = static_cast<int>((k_hi - logit_key(z[q])) >> shift) & ((1 << kBinBits) - 1);
        w[q] = kMass ? weight(z[q], ws, sm.table) : 0;
      }
      add_to_bins<kMass>(sm, in, b, w);
    };
    if (queued) {
#pragma unroll
      for (int q4 = 0; q4 < kQueued; q4 += 4) {
        float z[4];
        bool in[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          z[q] = q4 + q < kQueued ? mine_z[q4 + q < kQueued ? q4 + q : 0] : -INFINITY;
          in[q] = z[q] >= z_lo && z[q] <= z_hi;
        }
        if (in[0] || in[1] || in[2] || in[3]) divide(z, in);
      }
    } else {
      for_quads<NT>(s, z_lo, [&](const float (&z)[4], int id) {
        bool in[4];
        if (choose(z, id, in)) divide(z, in);
      });
    }
    close_histogram<NT, kMass>(sm);
    f = find_bin<NT, kMass>([&](u64) { return f.need - above; }, C, sm);
    f.need += above;
    above += f.above;
  }
  if (shift < 32) narrow();
  if (f.count > kList) {      // one key: which of its ids
    const u64 one = kMass ? weight(z_hi, ws, sm.table) : 1;
    u64 left = (f.need - above + one - 1) / one;       // so many of them, in all CTAs
    // the bin's counts of the CTAs are still in sm.p
    int owner = 0;
    while (owner < C - 1 && left > sm.p.cnt[owner][f.bin & 31]) left -= sm.p.cnt[owner++][f.bin & 31];
    if (owner == rank) {
      // element order is id order: contiguous parts of the slice per thread
      const int per = (s.len + NT - 1) / NT, lo = min(tid * per, s.len), hi = min(lo + per, s.len);
      auto tied = [&](int i) { return s.z[i] == z_hi && takes_part(s.z[i], s.base + i); };
      u64 n = 0, all;
      for (int i = lo; i < hi; ++i) n += tied(i);
      u64 seen = block_scan<NT>(n, sm.scan, &all) - n;
      if (seen < left && left <= seen + n) {
        for (int i = lo; i < hi; ++i)
          if (tied(i) && ++seen == left) {
            for (int c = 0; c < C; ++c)
              st_cluster_u32(mapa_shared(smem_addr(&sm.tie_id), c), static_cast<uint32_t>(s.base + i));
            break;
          }
      }
    }
    cluster_sync();
    const u64 cut = entry_of(k_hi, sm.tie_id);
    __syncthreads();
    return {cut, 0, 0, false};
  }
  __syncthreads();            // sm.p, in the list's place, is read (the queue is in registers)
  if (queued) {
#pragma unroll
    for (int q = 0; q < kQueued; ++q)
      if (mine_z[q] >= z_lo && mine_z[q] <= z_hi) {
        const uint32_t i = atomicAdd(&sm.n_list, 1u);
        if (i < kList) sm.list[i] = entry_of(logit_key(mine_z[q]), static_cast<uint32_t>(mine_id[q]));
      }
  } else {
    for_warp_quads<NT>(s, z_lo, [&](const float (&z)[4], int id) {
      bool in[4];
      Places at;
      choose(z, id, in);
      if (!reserve(in, &sm.n_list, at)) return;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (in[q] && at.at[q] < kList) sm.list[at.at[q]] = entry_of(logit_key(z[q]), static_cast<uint32_t>(id + q));
    });
  }
  cluster_sync();
  if (kAlone && whole_list && rank != 0) {
    cluster_sync();           // the first CTA has read this one's list
    return {0, 0, 0, true};
  }
  u64 e, all;
  const uint32_t n = pull_list<NT>(C, &sm.n_list, e, sm);   // into the histogram's place: nobody reads that any more
  const u64 own = static_cast<uint32_t>(tid) >= n ? 0 : kMass ? weight(entry_logit(e), ws, sm.table) : 1;
  const u64 incl = (whole_list ? 0 : above) + block_scan<NT>(own, sm.scan, &all);
  if (incl - own < f.need && f.need <= incl) sm.cut = e;
  __syncthreads();
  const u64 cut = sm.cut;
  cluster_sync();             // the others have read this CTA's list
  return {cut, whole_list ? n : 0, e, false};
}

// 2^x, off by at most 2^-22 of itself; subnormal results as 0.
__device__ __forceinline__ float rough_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// What a prefix has to reach: a count, or `fraction` of a sum known to within `error`.
struct Need {
  u64 fraction, least, most;
  __device__ __forceinline__ explicit Need(u64 count) : fraction(0), least(count), most(count) {}
  __device__ __forceinline__ Need(u64 f, u64 sum, u64 error)
      : fraction(f), least(part_of(f, sum - error)), most(part_of(f, sum + error)) {}
};
// The entry where the prefix ends, among sorted ones e of weight `own` behind a sum of
// `before`, which the threads of the first CTA hold (alone) or of every one; then every list
// has been read.  Within the error of a border (of a row where every id takes part) all CTAs
// sum their slices exactly.
template <int NT>
__device__ __forceinline__ u64 end_of(const Need& need, u64 before, u64 own, u64 e, bool alone, const Slice& s,
                                      const WeightScale& ws, int C, int rank, Smem& sm) {
  const int tid = threadIdx.x;
  const bool here = !alone || rank == 0;
  u64 incl = 0, all;
  if (here) {
    incl = before + block_scan<NT>(own, sm.scan, &all);
    if (incl - own < need.least && need.most <= incl) sm.cut = e;
    __syncthreads();
    if (alone && tid > 0 && tid < C) st_cluster_u64(mapa_shared(smem_addr(&sm.cut), tid), sm.cut);
  }
  cluster_sync();
  u64 cut = sm.cut;
  if (cut == 0 && need.least < need.most) {
    u64 sums[1] = {0};
    for_quads<NT>(s, -kLargest, [&](const float (&z)[4], int) {
      int n[4];
      float f[4];
      weight_places(z, ws, n, f);
#pragma unroll
      for (int q = 0; q < 4; ++q) sums[0] += weight_at(n[q], f[q], sm.table);
    });
    block_sums<NT>(sums, sm.scan);
    if (tid == 0) sm.sum = sums[0];
    cluster_sync();
    const int lane = tid & 31;
    const u64 exact =
        part_of(need.fraction, warp_sum(lane < C ? ld_cluster_u64(mapa_shared(smem_addr(&sm.sum), lane)) : 0));
    if (here && incl - own < exact && exact <= incl) sm.cut = e;
    cluster_sync();           // the others have read this CTA's sum
    cut = sm.cut;
  }
  return cut;
}
// A search (kMass: by weights, need a fraction of their sum; else by count) among the ids from
// z_min on, which have to be few, up to the entry `within`: they are queued and go into the
// histogram.  Those below z_min weigh `deep` together, within `error`, and are not the cut.  No
// cut (0) where it takes more: more ids, or a bin's division.  may_leave: where all that is
// kept is listed, the first CTA goes on alone.
template <int NT, bool kMass>
__device__ Ended search_above(u64 wanted, u64 deep, u64 error, float z_min, u64 within, bool may_leave, const Slice& s,
                              const WeightScale& ws, int C, int rank, Smem& sm) {
  const int tid = threadIdx.x, lane = tid & 31;
  __syncthreads();            // sm.cut is read
  if (tid == 0) {
    sm.n_list = sm.n_queue = 0;
    sm.cut = 0;
  }
  clear_histogram<NT>(sm);
  for_warp_quads<NT>(s, z_min, [&](const float (&z)[4], int id) {
    bool in[4];
    Places at;
#pragma unroll
    for (int q = 0; q < 4; ++q) in[q] = z[q] >= z_min;
    if (!reserve(in, &sm.n_queue, at)) return;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (in[q] && at.at[q] < kQueue) sm.queue[at.at[q]] = static_cast<uint16_t>(id + q - s.base);
  });
  __syncthreads();
  // bins of equal width (by weights' places or depth's octaves, 256 ids and more stand in one)
  const float per = ws.max > z_min ? kBins / (ws.max - z_min) : 0.f;
  constexpr int kQueued = kQueue / NT;
  u64 mine[kQueued], w[kQueued];
  bool in[kQueued];
  int bin[kQueued];
#pragma unroll
  for (int q = 0; q < kQueued; ++q) {
    const uint32_t i = q * NT + tid;
    in[q] = i < min(sm.n_queue, static_cast<uint32_t>(kQueue));
    w[q] = 0;
    bin[q] = kBins;
    if (!in[q]) continue;
    const int at = sm.queue[i];
    const float z = s.z[at];
    mine[q] = entry_of(logit_key(z), static_cast<uint32_t>(s.base + at));
    if (kMass) w[q] = weight(z, ws, sm.table);
    in[q] = mine[q] <= within && (!kMass || w[q] != 0);
    if (in[q]) bin[q] = min(static_cast<int>((ws.max - z) * per), kBins - 1);
  }
  add_to_bins<kMass>(sm, in, bin, w);
  close_histogram<NT, kMass>(sm);
  const bool fits = __all_sync(
      0xffffffffu, lane >= C || ld_cluster_u32(mapa_shared(smem_addr(&sm.n_queue), min(lane, C - 1))) <= kQueue);
  const Found f = find_bin<NT, kMass>(
      [&](u64 total) { return kMass ? part_of(wanted, total + deep - error) : wanted; }, C, sm);
  const Need need = kMass ? Need(wanted, f.total + deep, error) : Need(wanted);
  if (!fits || need.most > f.above + f.own || f.count > kList) {
    cluster_sync();           // the others have read this CTA's histogram
    return {0, 0, 0, false};
  }
  const bool whole_list = f.count_above + f.count <= kList;
  __syncthreads();            // sm.p, in the list's place, is read (the queue is in registers)
#pragma unroll
  for (int q = 0; q < kQueued; ++q)
    if (whole_list ? bin[q] <= f.bin : bin[q] == f.bin) {
      const uint32_t i = atomicAdd(&sm.n_list, 1u);
      if (i < kList) sm.list[i] = mine[q];
    }
  cluster_sync();
  const bool alone = whole_list && may_leave;
  u64 e = ~0ull, own = 0;
  uint32_t n = 0;
  if (!alone || rank == 0) {
    n = pull_list<NT>(C, &sm.n_list, e, sm);   // into the histogram's place: nobody reads that any more
    own = static_cast<uint32_t>(tid) >= n ? 0 : kMass ? weight(entry_logit(e), ws, sm.table) : 1;
  }
  const u64 cut = end_of<NT>(need, whole_list ? 0 : f.above, own, e, alone, s, ws, C, rank, sm);
  return {cut, whole_list ? n : 0, e, alone && rank != 0};
}

// The draw from the entries up to the cut among the n that the threads hold in order.
template <int NT>
__device__ void draw_from_list(const FilterArgs& a, int row, uint32_t n, u64 e, u64 cut, const WeightScale& ws,
                               Smem& sm) {
  const uint32_t tid = threadIdx.x, t = __syncthreads_count(tid < n && e <= cut);   // kept: the first t
  if (tid < t) {
    sm.d.weight[tid] = weight(entry_logit(e), ws, sm.table);
    sm.d.by_id[0][tid] = static_cast<uint32_t>(e) << 8 | tid;
  } else if (tid < rank_padded<NT>(t)) {
    sm.d.by_id[0][tid] = ~0u;
  }
  __syncthreads();
  rank_sort<NT>(sm.d.by_id[0], sm.d.by_id[1], t);   // the kept ids ascending
  const uint32_t by_id = tid < t ? sm.d.by_id[1][tid] : 0;
  u64 total;
  const u64 own = tid < t ? sm.d.weight[by_id & 255u] : 0;
  const u64 incl = block_scan<NT>(own, sm.scan, &total);
  const u64 target = __umul64hi(fraction64(a.u[row]), total);
  if (incl - own <= target && target < incl) a.out_tok[row] = static_cast<int>(by_id >> 8);
}
static_assert(kMaxVocab <= 1 << 24 && kList == 256, "an id and a place in 32 bits");

// NT = 512: a shorter pass over the slice (1 x 128256: no cut 9.7 us, 12.2 with 256 threads;
// flat top-p 31.5, 39.3); 256: three CTAs per SM and fewer instructions a row (what a thread
// does once per row), where not all of a launch's clusters fit at once (144 x 128256: top-k
// 35.9 us, 47.0 with 512; top-p then 112, 124).
template <int NT, bool kMask>
__global__ void __launch_bounds__(NT, NT == 256 ? 3 : 2) filter_kernel(const __grid_constant__ FilterArgs a, int C,
                                                                      int len) {
  extern __shared__ __align__(16) uint8_t raw[];
  Smem& sm = *reinterpret_cast<Smem*>(raw);
  Slice s;
  s.z = reinterpret_cast<float*>(raw + sizeof(Smem));
  s.len = len;
  constexpr int kWarps = NT / 32;
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  const int rank = static_cast<int>(cluster_ctarank()), row = blockIdx.x / C, V = a.vocab;
  for (int i = tid; i < kExpSteps; i += NT) sm.table[i] = exp_table()[i];
  if (tid == 0) {
    sm.n_list = 0;
    mbar_init(&sm.loaded, 1);
    fence_mbar_init();
  }
  cluster_arrive_release();   // waited for before the first push
  pdl_wait();
  pdl_launch_dependents();
  const float* z = a.logits + row * a.ld;
  // ids are shifted so that the slice's float4s are aligned in memory
  const int shift = static_cast<int>((reinterpret_cast<uintptr_t>(z) >> 2) & 3);
  s.base = rank * len - shift;
  // ------------------------------------------------ load; maximum and bound
  // whole float4s of the row by bulk copies (all of a slice's bytes are under way at once:
  // with loads through registers a quarter), its ragged ends by single loads
  float4* const s4 = reinterpret_cast<float4*>(s.z);
  const int q_lo = s.base < 0 ? 1 : 0, q_hi = max(q_lo, min(len, V - s.base) / 4);
  if (tid == 0 && q_hi > q_lo) {
    const uint32_t bytes = static_cast<uint32_t>(q_hi - q_lo) * 16;
    mbar_arrive_expect_tx(&sm.loaded, bytes);
    for (uint32_t at = 0; at < bytes; at += kCopyBytes)
      bulk_load(s.z + 4 * q_lo + at / 4, z + s.base + 4 * q_lo + at / 4, min(kCopyBytes, bytes - at), &sm.loaded,
                l2_policy_evict_normal());
  }
  const Rule r = rule_of(a, row);
  const bool by_k = r.top_k > 0 && r.top_k < V;
  bool by_p = r.top_p < 1.f;
  if (r.min_p > 0.f && tid == NT - 1) {   // 64-bit arithmetic: one thread's, beside the loads
    const double l = static_cast<double>(r.temperature) * (r.min_p < 1.f ? logit_scale(r.temperature) : 1.f) *
                     log(static_cast<double>(fminf(r.min_p, 1.f)));
    const float hi = static_cast<float>(l);
    sm.log_min_p = make_float2(hi, static_cast<float>(l - static_cast<double>(hi)));
  }
  float m = -INFINITY;
  auto take = [&](int i, float4 v) {
    const float4 o = make_float4(sane(v.x), sane(v.y), sane(v.z), sane(v.w));
    m = fmaxf(fmaxf(fmaxf(o.x, o.y), fmaxf(o.z, o.w)), m);
    if (v.x != o.x || v.y != o.y || v.z != o.z || v.w != o.w) s4[i] = o;
  };
  auto load_quad = [&](int i) {
    const int x = s.base + 4 * i;
    float4 v;
    v.x = x >= 0 && x < V ? __ldcg(z + x) : -INFINITY;
    v.y = x + 1 >= 0 && x + 1 < V ? __ldcg(z + x + 1) : -INFINITY;
    v.z = x + 2 >= 0 && x + 2 < V ? __ldcg(z + x + 2) : -INFINITY;
    v.w = x + 3 >= 0 && x + 3 < V ? __ldcg(z + x + 3) : -INFINITY;
    s4[i] = v;
    take(i, v);
  };
  if (tid < q_lo) load_quad(tid);
  for (int i = q_hi + tid; i < len / 4; i += NT) load_quad(i);
  if (q_hi > q_lo) {
    // the copies may be waited for once the barrier is initialised and they are announced
    __syncthreads();
    if (!mbar_wait_bounded(&sm.loaded, 0, nullptr, nullptr)) {
      mbar_wait_drain(&sm.loaded, 0);
      for (int i = q_lo + tid; i < q_hi; i += NT) load_quad(i);   // a thread takes what it loads
    }
#pragma unroll 4
    for (int i = q_lo + tid; i < q_hi; i += NT) take(i, s4[i]);
  }
  constexpr int kPerGroup = NT / kGroups;
#pragma unroll
  for (int o = 1; o < kPerGroup; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (tid % kPerGroup == 0) sm.group[tid / kPerGroup] = logit_key(m);
  __syncthreads();
  // the bound: the j-th largest group maximum, j = what this CTA owes to the top k (if that
  // is more than the groups can give, the bound is not used)
  const int owed = ((by_k ? r.top_k : kTopPAbove) + C - 1) / C, j = min(owed, kMostAbove);
  cluster_wait_acquire();
  if (w < kGroups / 32) {
    // the groups' keys less their last bits, made different by the group's number: at
    // least j groups reach the bound without those bits
    const uint32_t own = (sm.group[tid] & ~(kGroups - 1u)) | tid;
    int above = 0;
#pragma unroll 16
    for (int i = 0; i < kGroups; ++i) above += ((sm.group[i] & ~(kGroups - 1u)) | i) > own;
    const uint32_t top = __reduce_max_sync(0xffffffffu, max(sm.group[lane], sm.group[lane + 32]));
    if (above == j - 1)
      for (int c = 0; c < C; ++c)
        st_cluster_u64(mapa_shared(smem_addr(&sm.peer_max[rank]), c),
                       top | (static_cast<u64>(own & ~(kGroups - 1u)) << 32));
  }
  cluster_sync();
  uint32_t top = 0, least = ~0u;
  if (lane < C) {
    const uint2 v = sm.peer_max[lane];
    top = v.x;
    least = v.y;
  }
  m = key_logit(__reduce_max_sync(0xffffffffu, top));
  const float bound =
      r.top_k == 1 ? m : key_logit(max(__reduce_min_sync(0xffffffffu, least), logit_key(-kLargest)));
  // ------------------------------------------------ the cut
  const bool empty = m == -INFINITY;
  const WeightScale ws = weight_scale(m, r.temperature);
  const u64 no_cut = entry_of(logit_key(-kLargest), ~0u);
  u64 cut = no_cut;
  if (r.min_p > 0.f && !empty) {
    // the least float z with z >= max + T log(min_p), the product in two floats; all of it
    // scaled where T may take the product past the largest float
    const float2 l = sm.log_min_p;
    const float scale = r.min_p < 1.f ? ws.scale : 1.f, top = m * scale, lowest = -kLargest * scale;
    const float c = top + l.x, part = c - top;
    const float rest = ((top - (c - part)) + (l.x - part)) + l.y;  // what c lacks
    uint32_t key = c > lowest ? logit_key(scale == 1.f ? c : c * 18446744073709551616.f) : logit_key(-kLargest);
    if (c > lowest && rest > 0.f) ++key;
    cut = entry_of(min(key, logit_key(m)), ~0u);
  }
  const u64 fraction = fraction64(r.top_p);
  uint32_t n = 0;             // > 0: so many candidates were listed and hold what is kept
  if constexpr (!kMask) {
    // Top-p alone: the candidates' weights are summed exactly, all others' to 2^-17 of their
    // sum: that tells what the prefix has to reach but for the last bits, and with them where
    // it ends unless that is within those bits of a border.  (x - max, c and their product are
    // off by 2^-24 of themselves each, so an exponent above -46 by 2^-16.9 and the power by
    // 2^-17.4 of itself, besides the instruction's 2^-22; a thread's sums by 19
    // roundings: 2^-17.1 in all.)
    // Rows whose candidates lie within 4 octaves are flat: more ids than these hold the sum.
    // (Past T = 2^64 x - m may overflow where its weight does not vanish.)
    if (by_p && !by_k && !empty && ws.scale == 1.f && (m - bound) * ws.c() > 4.f) {
      float sum = 0.f, deep4[4] = {};
      u64 listed = 0;
      // 3 to 6 octaves below the bound: the queues hold what lies above of a row whose weights
      // fall by rank^-1.4
      const float z_deep = fmaxf(bound - static_cast<float>(34 - __clz(C)) / ws.c(), -kLargest);
      for_quads<NT>(s, -INFINITY, [&](const float (&x)[4], int id) {
        float e[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) e[q] = rough_exp2((x[q] - m) * ws.c());
        if (fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) >= bound) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (x[q] >= bound) {
              e[q] = 0.f;
              listed += weight(x[q], ws, sm.table);
              const uint32_t i = atomicAdd(&sm.n_list, 1u);
              if (i < kList) sm.list[i] = entry_of(logit_key(x[q]), static_cast<uint32_t>(id + q));
            }
        }
        sum += (e[0] + e[1]) + (e[2] + e[3]);
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (x[q] < z_deep) deep4[q] += e[q];
      });
      constexpr float kOne = 70368744177664.f;   // 2^46
      u64 sums[3] = {listed, __float2ull_rn(sum * kOne), 
                     __float2ull_rn(((deep4[0] + deep4[1]) + (deep4[2] + deep4[3])) * kOne)};
      block_sums<NT>(sums, sm.scan);
      if (tid == 0) {
        sm.listed_sum = sums[0];
        sm.sum = sums[1];
        sm.deep_sum = sums[2];
        sm.cut = 0;                        // no entry
      }
      cluster_sync();
      const bool peer = lane < C;
      n = __reduce_add_sync(0xffffffffu, peer ? ld_cluster_u32(mapa_shared(smem_addr(&sm.n_list), lane)) : 0u);
      listed = warp_sum(peer ? ld_cluster_u64(mapa_shared(smem_addr(&sm.listed_sum), lane)) : 0);
      const u64 rest = warp_sum(peer ? ld_cluster_u64(mapa_shared(smem_addr(&sm.sum), lane)) : 0);
      const u64 deep = warp_sum(peer ? ld_cluster_u64(mapa_shared(smem_addr(&sm.deep_sum), lane)) : 0);
      // weights are whole numbers, and 0 where the power is below 2^-45: 4 per id for both
      const u64 whole = 4 * static_cast<u64>(V);
      const u64 error = rest == 0 ? 0 : (rest >> 17) + whole;
      const Need need(fraction, listed + rest, error);
      if (n <= kList && listed >= need.most) {
        u64 e = ~0ull, own = 0;
        if (rank == 0) {                   // the rest is the first CTA's
          pull_list<NT>(C, &sm.n_list, e, sm);
          own = static_cast<uint32_t>(tid) < n ? weight(entry_logit(e), ws, sm.table) : 0;
        }
        cut = min(cut, end_of<NT>(need, 0, own, e, true, s, ws, C, rank, sm));
        if (rank == 0) draw_from_list<NT>(a, row, n, e, cut, ws, sm);
        return;
      }
      n = 0;
      cluster_sync();                      // the others have read this CTA's counts and sums
      // more than the list takes, but not by far: most of the sum is the candidates', and the
      // ids that are not deep hold all that is kept
      const u64 deep_error = deep == 0 ? 0 : (deep >> 17) + whole;
      if (rest <= listed && listed + rest - error >= need.most + deep + deep_error) {
        const Ended e = search_above<NT, true>(fraction, deep, deep_error, z_deep, ~0ull, true, s, ws, C, rank, sm);
        if (e.gone) return;
        if (e.cut != 0) {
          cut = min(cut, e.cut);
          if (e.listed > 0) {
            draw_from_list<NT>(a, row, e.listed, e.entry, cut, ws, sm);
            return;
          }
          by_p = false;                    // done
        }
      }
    }
  }
  bool search_k = by_k && !empty;
  // j groups' maxima of 64 stand for 64 log(64 / (64 - j)) logits of the CTA: where those of the
  // cluster would pass 9/10 of the list, draws go to the queues at once (144 x 128256, k 240: 64 us
  // for 75)
  const int most = kMask ? kMostAbove : C == 8 ? 23 : C == 4 ? 37 : C == 2 ? 53 : kMostAbove;
  if (search_k && owed <= most) {
    for_warp_quads<NT>(s, bound, [&](const float (&x)[4], int id) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (x[q] >= bound) {
          const uint32_t i = atomicAdd(&sm.n_list, 1u);
          if (i < kList) sm.list[i] = entry_of(logit_key(x[q]), static_cast<uint32_t>(id + q));
        }
    });
    cluster_sync();
    n = __reduce_add_sync(0xffffffffu, lane < C ? ld_cluster_u32(mapa_shared(smem_addr(&sm.n_list), lane)) : 0u);
    if (n <= kList) {
      search_k = false;
      if (!kMask && rank != 0) {           // the rest is the first CTA's
        cluster_sync();
        return;
      }
      u64 e;
      pull_list<NT>(C, &sm.n_list, e, sm);
      if (kMask)
        cluster_sync();                    // the others have read this CTA's list
      else
        cluster_arrive_release();          // they may leave; nobody reads this CTA's
      const uint32_t k = min(n, static_cast<uint32_t>(r.top_k));
      if (by_p) {
        u64 total;
        const u64 own = static_cast<uint32_t>(tid) < k ? weight(entry_logit(e), ws, sm.table) : 0;
        const u64 incl = block_scan<NT>(own, sm.scan, &total);
        const u64 need = part_of(fraction, total);
        if (incl - own < need && need <= incl) sm.cut = e;
      } else if (static_cast<uint32_t>(tid) == k - 1) {
        sm.cut = e;
      }
      __syncthreads();
      cut = min(cut, sm.cut);
      if (!kMask) {
        draw_from_list<NT>(a, row, n, e, cut, ws, sm);
        cluster_wait_acquire();
        return;
      }
    } else {
      n = 0;
      cluster_sync();                      // the others have read this CTA's count
    }
  }
  u64 within = no_cut;
  if constexpr (!kMask) {
    // Large k: the ids above the bound, or an octave below it where that is not sure to leave
    // so many (for 200 per CTA it mostly does: 144 x 128256, k 1000, p 0.9 131 -> 84 us; for more
    // it would be tried in vain, 144 x 32000 37 us for 32); then top-p among what is left of them.
    if (search_k && owed <= kMostBelow && ws.c() > 0.f) {
      const float z_low = owed <= kMostAbove ? bound : fmaxf(bound - 1.f / ws.c(), -kLargest);
      Ended e = search_above<NT, false>(static_cast<u64>(r.top_k), 0, 0, z_low, ~0ull, !by_p, s, ws, C, rank, sm);
      if (e.gone) return;
      if (e.cut != 0) {
        search_k = false;
        within = e.cut;
        if (by_p) {
          e = search_above<NT, true>(fraction, 0, 0, entry_logit(within), within, true, s, ws, C, rank, sm);
          if (e.gone) return;
          by_p = e.cut == 0;
        }
        cut = min(cut, e.cut != 0 ? e.cut : within);
        if (e.cut != 0 && e.listed > 0) {
          draw_from_list<NT>(a, row, e.listed, e.entry, cut, ws, sm);
          return;
        }
      }
    }
  }
  if (search_k) {
    within = search<NT, false, true, false>(Part{static_cast<u64>(r.top_k), 0, 0.f, ~0ull}, s, ws, C, rank, sm).cut;
    cut = min(cut, within);
  }
  if (by_p && !empty && n == 0) {
    // ids deeper than log2(2 V / (1 - p)) hold less than half of 1 - p of the mass together
    const float deepest = log2f(2.f * V / (1.f - fmaxf(r.top_p, 0.f))) + 0.01f;
    const int n_min = max(-static_cast<int>(deepest * kExpSteps), kNoWeight + 1);
    const Part part{fraction, n_min, bound, within >= no_cut ? ~0ull : within};
    const Ended e = within >= no_cut ? search<NT, true, true, !kMask>(part, s, ws, C, rank, sm)
                                     : search<NT, true, false, !kMask>(part, s, ws, C, rank, sm);
    if (e.gone) return;
    cut = min(cut, e.cut);
    if (!kMask && e.listed > 0) {
      draw_from_list<NT>(a, row, e.listed, e.entry, cut, ws, sm);
      return;
    }
  }
  const float cut_z = entry_logit(cut);
  const uint32_t cut_id = static_cast<uint32_t>(cut);
  auto kept = [&](float x, int id) { return x > cut_z || (x == cut_z && static_cast<uint32_t>(id) <= cut_id); };
  if constexpr (kMask) {
    float* out = a.out + row * a.out_ld;
    const bool aligned = ((reinterpret_cast<uintptr_t>(out) >> 2) & 3) == static_cast<uintptr_t>(shift);
    const bool inside = aligned && s.base >= 0 && s.base + len <= V;
    for (int i = tid; i < len / 4; i += NT) {
      const int x = s.base + 4 * i;
      float4 o = reinterpret_cast<const float4*>(s.z)[i];
      if (fmaxf(fmaxf(o.x, o.y), fmaxf(o.z, o.w)) < cut_z) {
        o = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
      } else {
        o.x = kept(o.x, x) ? o.x : -INFINITY;
        o.y = kept(o.y, x + 1) ? o.y : -INFINITY;
        o.z = kept(o.z, x + 2) ? o.z : -INFINITY;
        o.w = kept(o.w, x + 3) ? o.w : -INFINITY;
      }
      if (inside || (aligned && x >= 0 && x + 3 < V)) {
        *reinterpret_cast<float4*>(out + x) = o;
      } else {
        if (x >= 0 && x < V) out[x] = o.x;
        if (x + 1 >= 0 && x + 1 < V) out[x + 1] = o.y;
        if (x + 2 >= 0 && x + 2 < V) out[x + 2] = o.z;
        if (x + 3 >= 0 && x + 3 < V) out[x + 3] = o.w;
      }
    }
    return;
  }
  // ------------------------------------------------ the draw
  // a warp's part of the slice: whole 128-id tiles, in id order
  const int tiles = (len + 127) / 128, per = (tiles + kWarps - 1) / kWarps;
  const int t_lo = min(w * per, tiles), t_hi = min(t_lo + per, tiles);
  auto tile_weights = [&](int t, u64 (&wt)[4]) {   // false: none of the tile is kept
    const int i = t * 128 + lane * 4;
    float4 v = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    if (i < len) v = *reinterpret_cast<const float4*>(s.z + i);
    const bool some = fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)) >= cut_z;
    if (!__any_sync(0xffffffffu, some)) return false;
    const int x = s.base + i;
    const float z[4] = {v.x, v.y, v.z, v.w};
    int n[4];
    float f[4];
    weight_places(z, ws, n, f);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      wt[q] = weight_at(n[q], f[q], sm.table);
      if (cut != no_cut && !kept(z[q], x + q)) wt[q] = 0;
    }
    return true;
  };
  u64 mine = 0;
  if (cut == no_cut && !empty) {   // nothing is cut: two tiles' arithmetic at a time (56 us for 65
                                   // over 144 rows of 128256)
    const float4 none = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    for (int t = t_lo; t < t_hi; t += 2) {
      const int i = t * 128 + lane * 4;
      const float4 v0 = i < len ? *reinterpret_cast<const float4*>(s.z + i) : none;
      const float4 v1 = t + 1 < t_hi && i + 128 < len ? *reinterpret_cast<const float4*>(s.z + i + 128) : none;
      const float z[8] = {v0.x, v0.y, v0.z, v0.w, v1.x, v1.y, v1.z, v1.w};
      int n[8];
      float f[8];
      weight_places(z, ws, n, f);
#pragma unroll
      for (int q = 0; q < 8; ++q) mine += weight_at(n[q], f[q], sm.table);
    }
  } else if (!empty) {
    for (int t = t_lo; t < t_hi; ++t) {
      u64 wt[4];
      if (tile_weights(t, wt)) mine += (wt[0] + wt[1]) + (wt[2] + wt[3]);
    }
  }
  mine = warp_sum(mine);
  __syncthreads();
  if (lane == 0) sm.scan[w] = mine;
  __syncthreads();
  u64 slice = 0, before = 0;
#pragma unroll
  for (int i = 0; i < kWarps; ++i) {
    if (i < w) before += sm.scan[i];
    slice += sm.scan[i];
  }
  if (tid < C) st_cluster_u64(mapa_shared(smem_addr(&sm.peer_sum[rank]), tid), slice);
  cluster_sync();
  u64 total = 0;
#pragma unroll
  for (int c = 0; c < kMaxCluster; ++c) {
    const u64 v = c < C ? sm.peer_sum[c] : 0;
    if (c < rank) before += v;
    total += v;
  }
  if (empty) {
    if (rank == 0 && tid == 0) a.out_tok[row] = -1;
    return;
  }
  const u64 target = __umul64hi(fraction64(a.u[row]), total);
  if (!(before <= target && target < before + mine)) return;   // another warp's
  for (int t = t_lo; t < t_hi; ++t) {
    u64 wt[4];
    if (!tile_weights(t, wt)) continue;
    const u64 own = wt[0] + wt[1] + wt[2] + wt[3];
    const u64 incl = before + warp_scan(own);
    const u64 end = __shfl_sync(0xffffffffu, incl, 31);
    if (target < end) {
      u64 sum = incl - own;
      if (sum <= target && target < incl) {
        int q = 0;
        while (q < 3 && sum + wt[q] <= target) sum += wt[q++];
        a.out_tok[row] = s.base + t * 128 + lane * 4 + q;
      }
      return;
    }
    before = end;
  }
}

}  // namespace

cudaError_t launch_filter(const FilterArgs& a, cudaStream_t s, bool pdl) {
  if (a.vocab > kMaxVocab) return cudaErrorInvalidValue;
  // as many CTAs per row as its slices need, more while the launch is small (1 x 32000, no cut:
  // 5.4 us with 8 CTAs, 7.5 with 4; 64 x 32000: top-k and -p 10.9 us with 4, 15.9 with 8)
  int C = 1;
  while (C < kMaxCluster &&
         ((a.vocab + 3 + C - 1) / C > kMaxSlice - 3 || (a.rows * C * 2 <= 304 && a.vocab >= 2 * C * 2048)))
    C *= 2;
  const int len = ((a.vocab + 3 + C - 1) / C + 3) / 4 * 4;
  // 512 threads, two CTAs per SM, while all clusters fit at once: 34 of 8 CTAs, 72 of 4 (38 rows
  // of 128256, top-k 13.0 us with 256 threads and 17.2 with 512; 34 rows, top-p 41.5 and 34.7)
  const bool wide = a.rows * C <= (C == 8 ? 272 : C == 4 ? 288 : 304), mask = a.out != nullptr;
  void (*const kernel)(FilterArgs, int, int) = wide ? (mask ? filter_kernel<512, true> : filter_kernel<512, false>)
                                                    : (mask ? filter_kernel<256, true> : filter_kernel<256, false>);
  static std::atomic<bool> set[4][64];
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.rows) * C);
  cfg.blockDim = dim3(wide ? 512 : 256);
  cfg.dynamicSmemBytes = sizeof(Smem) + static_cast<size_t>(len) * 4;
  cfg.stream = s;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  std::atomic<bool>* done = e == cudaSuccess && dev < 64 ? &set[wide * 2 + mask][dev] : nullptr;
  if (e == cudaSuccess && (done == nullptr || !done->load(std::memory_order_relaxed))) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             static_cast<int>(sizeof(Smem) + kMaxSlice * 4));
    if (e == cudaSuccess && done != nullptr) done->store(true, std::memory_order_relaxed);
  }
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, a, C, len);
}

namespace {
// Arguments that both calls take; false: op error set.
bool filter_args(FilterArgs& a, const float* logits, int64_t ld, int32_t rows, int32_t vocab,
                 const memspec_filter* f) {
  const char* why = nullptr;
  if (logits == nullptr || f == nullptr)
    why = "null pointer";
  else if (reinterpret_cast<uintptr_t>(logits) & 3)
    why = "logits must be 4-byte aligned";
  else if (rows < 1 || rows > 65535 || vocab < 1 || vocab > kMaxVocab)
    why = "rows must be in 1..65535 and vocab in 1..131072";
  else if (rows > 1 && (ld < vocab || ld > INT64_C(1) << 40))
    why = "the row stride must be at least vocab";
  else if (f->temperature_dev == nullptr && !(f->temperature >= 0.f))
    why = "temperature must be >= 0";
  else if (f->top_k_dev == nullptr && f->top_k < 0)
    why = "top_k must be >= 0";
  else if (f->top_p_dev == nullptr && !(f->top_p > 0.f && f->top_p <= 1.f))
    why = "top_p must be in (0, 1]";
  else if (f->min_p_dev == nullptr && !(f->min_p >= 0.f && f->min_p <= 1.f))
    why = "min_p must be in [0, 1]";
  else if ((reinterpret_cast<uintptr_t>(f->temperature_dev) | reinterpret_cast<uintptr_t>(f->top_k_dev) |
            reinterpret_cast<uintptr_t>(f->top_p_dev) | reinterpret_cast<uintptr_t>(f->min_p_dev)) & 3)
    why = "rule arrays must be 4-byte aligned";
  if (why != nullptr) {
    set_op_error(why);
    return false;
  }
  a.logits = logits;
  a.ld = ld;
  a.rows = rows;
  a.vocab = vocab;
  a.rows_per_rule = 1;
  a.temperature = f->temperature;
  a.top_k = f->top_k;
  a.top_p = f->top_p;
  a.min_p = f->min_p;
  a.temperatures = f->temperature_dev;
  a.top_ks = f->top_k_dev;
  a.top_ps = f->top_p_dev;
  a.min_ps = f->min_p_dev;
  return true;
}

memspec_status filter_launch(const FilterArgs& a, void* stream) {
  const cudaError_t e = launch_filter(a, static_cast<cudaStream_t>(stream), true);
  if (e == cudaSuccess) return MEMSPEC_OK;
  set_op_error(std::string("filter launch: ") + cudaGetErrorString(e));
  return MEMSPEC_ERR_CUDA;
}
}  // namespace

}  // namespace memspec

extern "C" {

memspec_status memspec_op_sample_filtered(const float* logits, int64_t ld, int32_t rows, int32_t vocab,
                                          const memspec_filter* filter, const float* u, int32_t* out,
                                          void* stream) {
  memspec::FilterArgs a{};
  if (!memspec::filter_args(a, logits, ld, rows, vocab, filter)) return MEMSPEC_ERR_INVALID_ARG;
  if (u == nullptr || out == nullptr) {
    memspec::set_op_error("null pointer");
    return MEMSPEC_ERR_INVALID_ARG;
  }
  if ((reinterpret_cast<uintptr_t>(u) | reinterpret_cast<uintptr_t>(out)) & 3) {
    memspec::set_op_error("u and out must be 4-byte aligned");
    return MEMSPEC_ERR_INVALID_ARG;
  }
  a.u = u;
  a.out_tok = out;
  return memspec::filter_launch(a, stream);
}

memspec_status memspec_op_filter_logits(const float* logits, int64_t ld, int32_t rows, int32_t vocab,
                                        const memspec_filter* filter, float* out, int64_t out_ld,
                                        void* stream) {
  memspec::FilterArgs a{};
  if (!memspec::filter_args(a, logits, ld, rows, vocab, filter)) return MEMSPEC_ERR_INVALID_ARG;
  if (out == nullptr || (reinterpret_cast<uintptr_t>(out) & 3)) {
    memspec::set_op_error("out must be a 4-byte aligned pointer");
    return MEMSPEC_ERR_INVALID_ARG;
  }
  if (rows > 1 && (out_ld < vocab || out_ld > INT64_C(1) << 40 || (out == logits && out_ld != ld))) {
    memspec::set_op_error("out's row stride must be at least vocab, and in place the logits' own");
    return MEMSPEC_ERR_INVALID_ARG;
  }
  a.out = out;
  a.out_ld = out_ld;
  return memspec::filter_launch(a, stream);
}

}  // extern "C"
