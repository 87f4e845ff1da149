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
//   3. else a search per part (top-k, then top-p among what top-k left): a histogram of the
//      elements' depth below the maximum, 16 bins an octave, with counts and for top-p the
//      weights' sums, exact in 64 bits by two 32-bit atomics; the CTAs add up each other's
//      bins through distributed shared memory to find the bin with the cut, and list
//      its elements - or all up to there, where they are few enough.  A bin with more
//      than the list takes (flat rows, many equal logits) is divided by key as often as it
//      needs; a single key, by id;
//   4. the draw: from the list where it holds all that is kept, else the kept weights' sums
//      slice by slice, then warp by warp; or the mask.
// Every CTA of a cluster takes the same decisions from the same numbers, so no result is
// passed back but an id among more equal logits than the list takes.
#include <cuda_runtime.h>

#include <math.h>

#include <atomic>
#include <string>

#include "../../include/memspec_ops.h"
#include "expfix.cuh"
#include "internal.h"
#include "ptx.cuh"

namespace memspec {
namespace {

constexpr int kThreads = 256;     // 64 elements each of the longest slice: what a thread does
                                  // once per row is a third of its instructions at 512
constexpr int kWarps = kThreads / 32;
constexpr int kMaxVocab = 131072;
constexpr uint32_t kCopyBytes = 16384;
constexpr float kLargest = 3.402823466e38f;

typedef unsigned long long u64;

// NaN as -inf, +inf as the largest finite number.
__device__ __forceinline__ float sane(float z) { return fminf(fmaxf(z, -INFINITY), kLargest); }

constexpr int kMaxCluster = 8;
constexpr int kMantissa = 4;                 // bins per octave of depth: 2^4
constexpr int kBins = 16 << kMantissa;       // depths 2^-10 .. 2^6, clamped
constexpr int kSupers = kBins / 32;          // groups of 32 bins
constexpr uint32_t kList = 256;              // list entries of a CTA and of the cluster
constexpr int kGroups = 64;                  // groups of 4 threads whose maxima give the bound
constexpr int kMostAbove = 56;               // of them above it at most

struct alignas(16) Smem {
  u64 table[kExpSteps];
  union {
    struct {
      struct {
        uint32_t cnt[kBins], lo[kBins], hi[kBins];   // count, sum of weights in two words
      } h;
      struct {                               // find_bin: the sums of all CTAs
        u64 mass[kMaxCluster][32];
        uint32_t cnt[kMaxCluster][32];
      } p;
    };
    struct {
      u64 entry[kList], weight[kList];
    } all;                                   // the cluster's list
  };
  u64 list[kList];                           // this CTA's: (~key << 32) | id
  // of this CTA, read by the others
  uint32_t sup_cnt[kSupers];
  u64 sup_mass[kSupers];
  u64 tail;
  uint32_t n_list;
  u64 p_tail[kMaxCluster];                   // of all CTAs
  uint2 peer_max[kMaxCluster];               // pushed: keys of the maximum and the bound
  float2 log_min_p;                          // T log(min_p) in two floats
  u64 peer_sum[kMaxCluster];                 // pushed
  u64 scan[kWarps];
  uint32_t group[kGroups];                   // keys
  uint64_t loaded;                           // mbarrier of the slice's copies
  uint32_t tie_id;                           // pushed
  u64 cut, total;
};
static_assert(3 * (sizeof(Smem) + 16388 * 4 + 1024) <= 228 * 1024, "three CTAs per SM");

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
  return r;
}

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
__device__ u64 block_sum(u64 v, u64* scratch) {
  v = warp_sum(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  u64 s = 0;
#pragma unroll
  for (int i = 0; i < kWarps; ++i) s += scratch[i];
  return s;
}
// All threads of the cluster: what they wrote before is read after.
__device__ __forceinline__ void cluster_sync() {
  cluster_arrive_release();
  cluster_wait_acquire();
}

// The cut after the last kept id of a row's order: (~key << 32) | id; entries up to it are kept.
__device__ __forceinline__ u64 entry_of(uint32_t key, uint32_t id) {
  return (static_cast<u64>(~key) << 32) | id;
}

// A CTA's slice of a row in shared memory: ids base .. base + len - 1, -inf where there is
// none.  Element i of the slice is held by nobody in particular: passes deal float4s.
struct Slice {
  float* z;
  int base, len;            // len a multiple of 4
};

struct Part {               // one search: what it looks at and for
  bool mass;                // top-p: `need` is a fraction of the sum; else a count
  u64 need;
  float scale;              // depth = (max - z) * scale
  float max, deepest;       // elements deeper than `deepest` are not the cut (only their weight counts)
  u64 within;               // entries up to this one take part
};

__device__ __forceinline__ int bin_of(float depth) {
  const int b = static_cast<int>(__float_as_uint(depth) >> (23 - kMantissa)) - ((127 - 10) << kMantissa);
  return max(0, min(b, kBins - 1));
}

// A histogram's bin that holds the cut, by the same steps in every CTA of the cluster.
struct Found {
  int bin;
  u64 above;                // sum (count or mass) before the bin
  uint32_t count;           // elements in it
  uint32_t count_above;     // and before it
  u64 need;                 // what the prefix has to reach
  bool all;                 // the whole set does not exceed it (a count): nothing is cut
};

// After the histogram of every CTA is complete and the cluster has synchronised.
__device__ Found find_bin(const Part& p, bool first, u64 need, int C, Smem& sm) {
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  Found f;
  // the groups' sums of all CTAs
  if (tid < C * kSupers) {
    const int peer = tid / kSupers, g = tid % kSupers;
    sm.p.cnt[peer][g] = ld_cluster_u32(mapa_shared(smem_addr(&sm.sup_cnt[g]), peer));
    if (p.mass) sm.p.mass[peer][g] = ld_cluster_u64(mapa_shared(smem_addr(&sm.sup_mass[g]), peer));
  }
  if (p.mass && first && tid < C) sm.p_tail[tid] = ld_cluster_u64(mapa_shared(smem_addr(&sm.tail), tid));
  __syncthreads();
  u64 v = 0, tail = 0;
  uint32_t n = 0;
  if (lane < kSupers)
    for (int c = 0; c < C; ++c) {
      n += sm.p.cnt[c][lane];
      if (p.mass) v += sm.p.mass[c][lane];
    }
  if (!p.mass) v = n;
  u64 incl = warp_scan(v);
  const uint32_t n_incl = warp_scan(n);
  const u64 total = __shfl_sync(0xffffffffu, incl, 31);
  if (p.mass && first) {
    for (int c = 0; c < C; ++c) tail += sm.p_tail[c];
    const u64 s = total + tail, part = need * s;          // the fraction times the sum, rounded up
    need = __umul64hi(need, s) + (part != 0 ? 1 : 0);
    if (need == 0) need = 1;
  }
  f.need = need;
  f.all = !p.mass && need >= total;
  const unsigned reach = __ballot_sync(0xffffffffu, lane < kSupers && incl >= need);
  const int g = reach ? __ffs(reach) - 1 : kSupers - 1;
  const u64 before = __shfl_sync(0xffffffffu, incl - v, g);
  const uint32_t n_before = __shfl_sync(0xffffffffu, n_incl - n, g);
  __syncthreads();                                        // p is read
  if (w < C) {
    sm.p.cnt[w][lane] = ld_cluster_u32(mapa_shared(smem_addr(&sm.h.cnt[g * 32 + lane]), w));
    if (p.mass)
      sm.p.mass[w][lane] = ld_cluster_u32(mapa_shared(smem_addr(&sm.h.lo[g * 32 + lane]), w)) |
                           (static_cast<u64>(ld_cluster_u32(mapa_shared(smem_addr(&sm.h.hi[g * 32 + lane]), w))) << 32);
  }
  __syncthreads();
  n = 0;
  v = 0;
  for (int c = 0; c < C; ++c) {
    n += sm.p.cnt[c][lane];
    if (p.mass) v += sm.p.mass[c][lane];
  }
  if (!p.mass) v = n;
  incl = before + warp_scan(v);
  const unsigned hit = __ballot_sync(0xffffffffu, incl >= need);
  const int b = hit ? __ffs(hit) - 1 : 31;
  f.bin = g * 32 + b;
  f.above = __shfl_sync(0xffffffffu, incl - v, b);
  f.count = __shfl_sync(0xffffffffu, n, b);
  f.count_above = n_before + __shfl_sync(0xffffffffu, warp_scan(n) - n, b);
  return f;
}

// The elements of at least z_min (four at a time: some below it too).
template <class Each>
__device__ __forceinline__ void for_slice(const Slice& s, float z_min, Each each) {
  const float4* z4 = reinterpret_cast<const float4*>(s.z);
  for (int i = threadIdx.x; i < s.len / 4; i += kThreads) {
    const float4 v = z4[i];
    if (fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)) < z_min) continue;
    each(v.x, s.base + 4 * i);
    each(v.y, s.base + 4 * i + 1);
    each(v.z, s.base + 4 * i + 2);
    each(v.w, s.base + 4 * i + 3);
  }
}

__device__ __forceinline__ void add_mass(Smem& sm, int bin, u64 w) {
  const uint32_t lo = static_cast<uint32_t>(w);
  const uint32_t old = atomicAdd(&sm.h.lo[bin], lo);
  const uint32_t hi = static_cast<uint32_t>(w >> 32) + (old + lo < old ? 1u : 0u);
  if (hi != 0) atomicAdd(&sm.h.hi[bin], hi);
}
__device__ void clear_histogram(Smem& sm) {
  uint32_t* h = reinterpret_cast<uint32_t*>(&sm.h);
  for (int i = threadIdx.x; i < static_cast<int>(sizeof(sm.h) / 4); i += kThreads) h[i] = 0;
  __syncthreads();
}
// The groups' sums of this CTA's histogram, then the cluster's barrier.
__device__ void close_histogram(const Part& p, Smem& sm) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  __syncthreads();
  for (int g = w; g < kSupers; g += kWarps) {
    const uint32_t n = __reduce_add_sync(0xffffffffu, sm.h.cnt[g * 32 + lane]);
    u64 m = 0;
    if (p.mass) m = warp_sum(sm.h.lo[g * 32 + lane] | (static_cast<u64>(sm.h.hi[g * 32 + lane]) << 32));
    if (lane == 0) {
      sm.sup_cnt[g] = n;
      sm.sup_mass[g] = m;
    }
  }
  cluster_sync();
}

// The CTAs' lists into sm.all; returns the number of entries.  All threads.
template <class Mass>
__device__ uint32_t pull_list(int C, bool weighted, Mass mass, Smem& sm) {
  // a warp per CTA: lane c has CTA c's count
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  uint32_t n = lane < C ? ld_cluster_u32(mapa_shared(smem_addr(&sm.n_list), lane)) : 0;
  const uint32_t incl = warp_scan(n), all = min(__shfl_sync(0xffffffffu, incl, 31), kList);
  const uint32_t off = __shfl_sync(0xffffffffu, incl - n, w);
  n = __shfl_sync(0xffffffffu, n, w);
  if (w < C)
    for (uint32_t i = lane; i < n && off + i < kList; i += 32) {
      const u64 e = ld_cluster_u64(mapa_shared(smem_addr(&sm.list[i]), w));
      sm.all.entry[off + i] = e;
      sm.all.weight[off + i] = weighted ? mass(key_logit(~static_cast<uint32_t>(e >> 32))) : 1;
    }
  __syncthreads();
  return all;
}
static_assert(kWarps >= kMaxCluster, "a warp per CTA of the cluster");

// Over the n entries of sm.all, 2^bits threads to an entry: the sum of value(e, j) over all
// j, then use(i, e, sum) in the first of them.
template <class Value, class Use>
__device__ __forceinline__ void for_pairs(uint32_t n, Smem& sm, Value value, Use use) {
  const int bits = n <= kThreads / 8 ? 3 : n <= kThreads / 4 ? 2 : n <= kThreads / 2 ? 1 : 0;
  const uint32_t i = threadIdx.x >> bits, part = threadIdx.x & ((1u << bits) - 1);
  const u64 e = i < n ? sm.all.entry[i] : 0;
  u64 sum = 0;
  if (i < n)
    for (uint32_t j = part; j < n; j += 1u << bits) sum += value(e, j);
  for (int o = 1 << bits >> 1; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (i < n && part == 0) use(i, e, sum);
}
static_assert(kList <= kThreads, "an entry per thread");

struct Ended {
  u64 cut;
  uint32_t listed;          // > 0: sm.all holds so many entries, all up to the cut among them
};

// The entry at which the prefix that p asks for ends.
template <class Mass>
__device__ Ended search(const Part& p, const Slice& s, int C, int rank, Mass mass, Smem& sm) {
  const int tid = threadIdx.x;
  auto depth = [&](float z) { return (p.max - z) * p.scale; };
  auto takes_part = [&](float z, int id) {
    return z > -INFINITY && entry_of(logit_key(z), static_cast<uint32_t>(id)) <= p.within;
  };
  const bool whole = p.within == ~0ull;
  const float z_in = whole ? -kLargest : key_logit(~static_cast<uint32_t>(p.within >> 32));
  clear_histogram(sm);
  if (tid == 0) {
    sm.n_list = 0;
    sm.cut = p.within;
  }
  u64 tail = 0;
  for_slice(s, z_in, [&](float z, int id) {
    if (whole ? z == -INFINITY : !takes_part(z, id)) return;
    const float d = depth(z);
    const u64 w = p.mass ? mass(z) : 0;
    if (d > p.deepest) {
      tail += w;
      return;
    }
    const int b = bin_of(d);
    atomicAdd(&sm.h.cnt[b], 1u);
    if (p.mass) add_mass(sm, b, w);
  });
  if (p.mass) {
    tail = block_sum(tail, sm.scan);
    if (tid == 0) sm.tail = tail;
  }
  close_histogram(p, sm);
  Found f = find_bin(p, true, p.need, C, sm);
  if (f.all) {
    cluster_sync();           // the others have read this CTA's histogram
    return {p.within, 0};
  }
  const int bin = f.bin;
  // the keys that the bin's elements can have: those of its depths with a margin (depth is
  // (max - z) * scale, off by some units in the last place of the larger term)
  uint32_t k_lo, k_hi;
  {
    constexpr int kFirst = (127 - 10) << kMantissa;
    const float a0 = __uint_as_float(static_cast<uint32_t>(bin + kFirst) << (23 - kMantissa));
    const float a1 = __uint_as_float(static_cast<uint32_t>(bin + 1 + kFirst) << (23 - kMantissa));
    const float z1 = p.max - a0 / p.scale, z0 = p.max - a1 / p.scale;
    const float slack = 4e-7f * (fabsf(p.max) + fabsf(z0)) + 1e-37f;
    k_hi = bin == 0 || !(z1 + slack < p.max) ? logit_key(p.max) : logit_key(z1 + slack);
    k_lo = bin == kBins - 1 || !(z0 - slack > -kLargest) ? logit_key(-kLargest) : logit_key(z0 - slack);
  }
  int shift = 32;             // keys per bin of the last division: 2^shift
  auto in_bin = [&](float z, int id) {
    if (whole ? z == -INFINITY : !takes_part(z, id)) return false;
    const float d = depth(z);
    if (d > p.deepest || bin_of(d) != bin) return false;
    const uint32_t k = logit_key(z);
    return k >= k_lo && k <= k_hi;
  };
  auto narrow = [&] {         // to the keys of bin f.bin of the last division
    k_hi -= static_cast<uint32_t>(f.bin) << shift;
    if (k_hi - k_lo >= 1u << shift) k_lo = k_hi - ((1u << shift) - 1);
  };
  u64 above = f.above;
  // for the draw it pays to have all of the kept elements
  const bool whole_list = p.mass && f.count_above + f.count <= kList;
  while (f.count > kList) {
    if (shift == 32) {        // the first division of [k_lo, k_hi]
      shift = max(0, 32 - __clz(k_hi - k_lo) - (4 + kMantissa));
    } else {
      if (shift == 0) break;
      narrow();
      shift = max(0, shift - (4 + kMantissa));
    }
    cluster_sync();           // the others have read this CTA's histogram
    clear_histogram(sm);
    for_slice(s, key_logit(k_lo), [&](float z, int id) {
      if (!in_bin(z, id)) return;
      const int b = static_cast<int>((k_hi - logit_key(z)) >> shift);
      atomicAdd(&sm.h.cnt[b], 1u);
      if (p.mass) add_mass(sm, b, mass(z));
    });
    close_histogram(p, sm);
    f = find_bin(p, false, f.need - above, C, sm);
    f.need += above;
    above += f.above;
  }
  if (shift < 32) narrow();
  if (f.count > kList) {      // one key: which of its ids
    const u64 one = p.mass ? mass(key_logit(k_hi)) : 1;
    u64 left = (f.need - above + one - 1) / one;       // so many of them, in all CTAs
    // the bin's counts of the CTAs are still in sm.p
    int owner = 0;
    while (owner < C - 1 && left > sm.p.cnt[owner][f.bin & 31]) left -= sm.p.cnt[owner++][f.bin & 31];
    if (owner == rank) {
      // element order is id order: contiguous parts of the slice per thread
      const int per = (s.len + kThreads - 1) / kThreads, lo = min(tid * per, s.len), hi = min(lo + per, s.len);
      u64 n = 0;
      for (int i = lo; i < hi; ++i) n += in_bin(s.z[i], s.base + i);
      const u64 incl = warp_scan(n);
      if ((tid & 31) == 31) sm.scan[tid >> 5] = incl;
      __syncthreads();
      u64 before = incl - n;
      for (int i = 0; i < (tid >> 5); ++i) before += sm.scan[i];
      if (before < left && left <= before + n) {
        u64 seen = before;
        for (int i = lo; i < hi; ++i)
          if (in_bin(s.z[i], s.base + i) && ++seen == left) {
            for (int c = 0; c < C; ++c)
              st_cluster_u32(mapa_shared(smem_addr(&sm.tie_id), c), static_cast<uint32_t>(s.base + i));
            break;
          }
      }
    }
    cluster_sync();
    const u64 cut = entry_of(k_hi, sm.tie_id);
    __syncthreads();
    return {cut, 0};
  }
  for_slice(s, key_logit(k_lo), [&](float z, int id) {
    if (whole_list) {
      const float d = depth(z);
      if ((whole ? z == -INFINITY : !takes_part(z, id)) || d > p.deepest || bin_of(d) > bin) return;
    } else if (!in_bin(z, id)) {
      return;
    }
    const uint32_t i = atomicAdd(&sm.n_list, 1u);
    if (i < kList) sm.list[i] = entry_of(logit_key(z), static_cast<uint32_t>(id));
  });
  cluster_sync();
  const uint32_t n = pull_list(C, p.mass, mass, sm);   // into the histogram's place: nobody reads that any more
  if (whole_list) above = 0;
  for_pairs(n, sm, [&](u64 e, uint32_t i) { return sm.all.entry[i] < e ? sm.all.weight[i] : 0; },
            [&](uint32_t i, u64 e, u64 before) {
              before += above;
              if (before < f.need && f.need <= before + sm.all.weight[i]) sm.cut = e;
            });
  __syncthreads();
  const u64 cut = sm.cut;
  cluster_sync();             // the others have read this CTA's list
  return {cut, whole_list ? n : 0};
}

// The draw from the n entries of sm.all up to the cut.
__device__ void draw_from_list(const FilterArgs& a, int row, uint32_t n, u64 cut, Smem& sm) {
  const uint32_t tid = threadIdx.x;
  u64 v = 0;
  if (tid < n) {
    if (sm.all.entry[tid] > cut) sm.all.weight[tid] = 0;
    v = sm.all.weight[tid];
  }
  const u64 total = block_sum(v, sm.scan);
  const u64 target = __umul64hi(fraction64(a.u[row]), total);
  for_pairs(n, sm,
            [&](u64 e, uint32_t i) {
              return static_cast<uint32_t>(sm.all.entry[i]) < static_cast<uint32_t>(e) ? sm.all.weight[i] : 0;
            },
            [&](uint32_t i, u64 e, u64 before) {
              if (before <= target && target < before + sm.all.weight[i])
                a.out_tok[row] = static_cast<int>(static_cast<uint32_t>(e));
            });
}

template <bool kMask>
__global__ void __launch_bounds__(kThreads, 3) filter_kernel(const __grid_constant__ FilterArgs a, int C, int len) {
  extern __shared__ __align__(16) uint8_t raw[];
  Smem& sm = *reinterpret_cast<Smem*>(raw);
  Slice s;
  s.z = reinterpret_cast<float*>(raw + sizeof(Smem));
  s.len = len;
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  const int rank = static_cast<int>(cluster_ctarank()), row = blockIdx.x / C, V = a.vocab;
  for (int i = tid; i < kExpSteps; i += kThreads) sm.table[i] = exp_table()[i];
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
  const Rule r = rule_of(a, row);
  const bool by_k = r.top_k > 0 && r.top_k < V, by_p = r.top_p < 1.f;
  if (r.min_p > 0.f && tid == kThreads - 1) {   // 64-bit arithmetic: one thread's, beside the loads
    const double l = static_cast<double>(r.temperature) * log(static_cast<double>(fminf(r.min_p, 1.f)));
    const float hi = static_cast<float>(l);
    sm.log_min_p = make_float2(hi, static_cast<float>(l - static_cast<double>(hi)));
  }
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
  for (int i = q_hi + tid; i < len / 4; i += kThreads) load_quad(i);
  if (q_hi > q_lo) {
    // the copies may be waited for once the barrier is initialised and they are announced
    __syncthreads();
    if (!mbar_wait_bounded(&sm.loaded, 0, nullptr, nullptr))
      for (int i = q_lo + tid; i < q_hi; i += kThreads) load_quad(i);   // a thread takes what it loads
#pragma unroll 4
    for (int i = q_lo + tid; i < q_hi; i += kThreads) take(i, s4[i]);
  }
#pragma unroll
  for (int o = 1; o < kThreads / kGroups; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (tid % (kThreads / kGroups) == 0) sm.group[tid / (kThreads / kGroups)] = logit_key(m);
  __syncthreads();
  // the bound: the j-th largest group maximum, j = what this CTA owes to the top k (if that
  // is more than the groups can give, the bound is not used)
  const int owed = by_k ? (r.top_k + C - 1) / C : 1, j = min(owed, kMostAbove);
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
  const float bound = key_logit(max(__reduce_min_sync(0xffffffffu, least), logit_key(-kLargest)));
  // ------------------------------------------------ the cut
  const bool empty = m == -INFINITY;
  const WeightScale ws = weight_scale(m, r.temperature);
  auto mass = [&](float x) { return weight(x, ws, sm.table); };
  const u64 no_cut = entry_of(logit_key(-kLargest), ~0u);
  u64 cut = no_cut;
  if (r.min_p > 0.f && !empty) {
    // the least float z with z >= max + T log(min_p), the product in two floats
    const float2 l = sm.log_min_p;
    const float c = m + l.x, part = c - m;
    const float rest = ((m - (c - part)) + (l.x - part)) + l.y;    // what c lacks
    uint32_t key = c > -kLargest ? logit_key(c) : logit_key(-kLargest);
    if (c > -kLargest && rest > 0.f) ++key;
    cut = entry_of(min(key, logit_key(m)), ~0u);
  }
  const u64 fraction = fraction64(r.top_p);
  uint32_t n = 0;             // > 0: sm.all holds so many entries, all the kept ones among them
  bool search_k = by_k && !empty;
  if (search_k && owed <= kMostAbove) {
    for_slice(s, bound, [&](float x, int id) {
      if (x < bound) return;
      const uint32_t i = atomicAdd(&sm.n_list, 1u);
      if (i < kList) sm.list[i] = entry_of(logit_key(x), static_cast<uint32_t>(id));
    });
    cluster_sync();
    n = __reduce_add_sync(0xffffffffu, lane < C ? ld_cluster_u32(mapa_shared(smem_addr(&sm.n_list), lane)) : 0u);
    if (n <= kList) {
      search_k = false;
      if (!kMask && rank != 0) {           // the rest is the first CTA's
        cluster_sync();
        return;
      }
      pull_list(C, true, mass, sm);
      if (kMask)
        cluster_sync();                    // the others have read this CTA's list
      else
        cluster_arrive_release();          // they may leave; nobody reads this CTA's
      if (tid == 0) sm.cut = ~0ull;
      __syncthreads();
      for_pairs(n, sm, [&](u64 e, uint32_t i) { return static_cast<u64>(sm.all.entry[i] < e); },
                [&](uint32_t, u64 e, u64 before) {
                  if (before + 1 == static_cast<u64>(r.top_k)) sm.cut = e;
                });
      __syncthreads();
      const u64 cut_k = sm.cut;
      cut = min(cut, cut_k);
      if (by_p) {
        const u64 v = tid < n && sm.all.entry[tid] <= cut_k ? sm.all.weight[tid] : 0;
        const u64 total = block_sum(v, sm.scan);
        const u64 need = max(__umul64hi(fraction, total) + (fraction * total != 0 ? 1 : 0), 1ull);
        for_pairs(n, sm, [&](u64 e, uint32_t i) { return sm.all.entry[i] < e ? sm.all.weight[i] : 0; },
                  [&](uint32_t i, u64 e, u64 before) {
                    if (before < need && need <= before + sm.all.weight[i]) sm.cut = e;
                  });
        __syncthreads();
        cut = min(cut, sm.cut);
      }
      if (!kMask) {
        draw_from_list(a, row, n, cut, sm);
        cluster_wait_acquire();
        return;
      }
    } else {
      n = 0;
      cluster_sync();                      // the others have read this CTA's count
    }
  }
  u64 within = no_cut;
  if (search_k) {
    within = search(Part{false, static_cast<u64>(r.top_k), 1.f, m, INFINITY, ~0ull}, s, C, rank, mass, sm).cut;
    cut = min(cut, within);
  }
  if (by_p && !empty && n == 0) {
    // ids deeper than log2(2 V / (1 - p)) hold less than half of 1 - p of the mass together
    const float deepest = log2f(2.f * V / (1.f - fmaxf(r.top_p, 0.f))) + 0.01f;
    const Ended e = search(Part{true, fraction, ws.hi, m, deepest, min(within, no_cut) == no_cut ? ~0ull : within}, s, C,
                           rank, mass, sm);
    cut = min(cut, e.cut);
    if (!kMask && e.listed > 0) {
      if (rank == 0) draw_from_list(a, row, e.listed, cut, sm);
      return;
    }
  }
  const float cut_z = key_logit(~static_cast<uint32_t>(cut >> 32));
  const uint32_t cut_id = static_cast<uint32_t>(cut);
  auto kept = [&](float x, int id) { return x > cut_z || (x == cut_z && static_cast<uint32_t>(id) <= cut_id); };
  if constexpr (kMask) {
    float* out = a.out + row * a.out_ld;
    const bool aligned = ((reinterpret_cast<uintptr_t>(out) >> 2) & 3) == static_cast<uintptr_t>(shift);
    const bool inside = aligned && s.base >= 0 && s.base + len <= V;
    for (int i = tid; i < len / 4; i += kThreads) {
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
    wt[0] = kept(v.x, x) ? mass(v.x) : 0;
    wt[1] = kept(v.y, x + 1) ? mass(v.y) : 0;
    wt[2] = kept(v.z, x + 2) ? mass(v.z) : 0;
    wt[3] = kept(v.w, x + 3) ? mass(v.w) : 0;
    return true;
  };
  u64 mine = 0;
  if (!empty)
    for (int t = t_lo; t < t_hi; ++t) {
      u64 wt[4];
      if (tile_weights(t, wt)) mine += wt[0] + wt[1] + wt[2] + wt[3];
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
  // as many CTAs per row as its slices need, more while the launch is small
  constexpr int kMaxSlice = 16388;           // floats: three CTAs per SM
  int C = 1;
  while (C < kMaxCluster &&
         ((a.vocab + 3 + C - 1) / C > kMaxSlice - 3 || (a.rows * C * 2 <= 304 && a.vocab >= 2 * C * 2048)))
    C *= 2;
  const int len = ((a.vocab + 3 + C - 1) / C + 3) / 4 * 4;
  static std::atomic<bool> set[2][64];
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.rows) * C);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = sizeof(Smem) + static_cast<size_t>(len) * 4;
  cfg.stream = s;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  const bool mask = a.out != nullptr;
  if (e == cudaSuccess && (dev >= 64 || !set[mask][dev].load(std::memory_order_relaxed))) {
    const int most = static_cast<int>(sizeof(Smem) + kMaxSlice * 4);
    e = mask ? cudaFuncSetAttribute(filter_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, most)
             : cudaFuncSetAttribute(filter_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    if (e == cudaSuccess && dev < 64) set[mask][dev].store(true, std::memory_order_relaxed);
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
  return mask ? cudaLaunchKernelEx(&cfg, filter_kernel<true>, a, C, len)
              : cudaLaunchKernelEx(&cfg, filter_kernel<false>, a, C, len);
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
  else if (ld < vocab || ld > INT64_C(1) << 40)
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
  if (out_ld < vocab || out_ld > INT64_C(1) << 40 || (out == logits && out_ld != ld)) {
    memspec::set_op_error("out's row stride must be at least vocab, and in place the logits' own");
    return MEMSPEC_ERR_INVALID_ARG;
  }
  a.out = out;
  a.out_ld = out_ld;
  return memspec::filter_launch(a, stream);
}

}  // extern "C"
