// filter.cu - sampling rules per row: top-k, top-p and min-p on softmax(z / T)
// (memspec_op_sample_filtered, memspec_op_filter_logits).
//
// Order a row's ids by descending logit, equal logits by ascending id.  Each rule keeps a
// prefix of that order and all of them together the shortest: top-k the first k; top-p the
// shortest whose weights (expfix.cuh) hold p of the sum over the first k; min-p the ids
// with weight >= min_p of the largest.  So a rule's result is a cut (key, id): an id is
// kept if its logit's key is larger, or equal and its id not above the cut's.
//
// One CTA per row: the cut's key by a radix search, 8 bits a pass, over counts (top-k) or
// over sums of weights (top-p); the sums are integers, so their comparisons are exact
// whatever the order in which the atomics add.
#include <cuda_runtime.h>

#include <math.h>

#include <string>

#include "../../include/memspec_ops.h"
#include "expfix.cuh"
#include "internal.h"
#include "ptx.cuh"

namespace memspec {
namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxVocab = 131072;
constexpr float kLargest = 3.402823466e38f;

typedef unsigned long long u64;

// NaN as -inf, +inf as the largest finite number.
__device__ __forceinline__ float sane(float z) { return z == z ? fminf(z, kLargest) : -INFINITY; }

struct Smem {
  u64 table[kExpSteps];
  u64 hist[256];
  u64 scan[kWarps];
  float wmax[kWarps];
  u64 found_before;
  int found;
  int pick;
};

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
  }
  return r;
}

// Exclusive scan of one u64 per thread; *total gets the sum.
__device__ u64 block_scan(u64 v, u64* scratch, u64* total) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  u64 incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 n = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += n;
  }
  __syncthreads();
  if (lane == 31) scratch[w] = incl;
  __syncthreads();
  u64 before = 0, all = 0;
  for (int i = 0; i < kWarps; ++i) {
    if (i < w) before += scratch[i];
    all += scratch[i];
  }
  *total = all;
  return before + incl - v;
}

// The smallest prefix of the row's order whose sum of val(z) reaches `need` (1 <= need <=
// the sum over the row): its last id's key, and in *before the sum over larger keys.
template <class Val>
__device__ uint32_t find_key(const float* z, int V, u64 need, Val val, Smem& sm, u64* before) {
  uint32_t prefix = 0;
  u64 above = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256; i += kThreads) sm.hist[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < V; i += kThreads) {
      const float x = sane(z[i]);
      const uint32_t key = logit_key(x);
      if (shift < 24 && (key >> (shift + 8)) != prefix) continue;
      const u64 v = x == -INFINITY ? 0 : val(x);
      if (v != 0) atomicAdd(&sm.hist[(key >> shift) & 255], v);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      u64 sum = above;
      int d = 255;
      while (d > 0 && sum + sm.hist[d] < need) sum += sm.hist[d--];
      sm.found = d;
      sm.found_before = sum;
    }
    __syncthreads();
    prefix = (prefix << 8) | static_cast<uint32_t>(sm.found);
    above = sm.found_before;
    __syncthreads();
  }
  *before = above;
  return prefix;
}

template <bool kMask>
__global__ void __launch_bounds__(kThreads) filter_kernel(const __grid_constant__ FilterArgs a) {
  __shared__ Smem sm;
  const int row = blockIdx.x, tid = threadIdx.x, V = a.vocab;
  pdl_wait();
  pdl_launch_dependents();
  const float* z = a.logits + row * a.ld;
  const Rule r = rule_of(a, row);
  for (int i = tid; i < kExpSteps; i += kThreads) sm.table[i] = exp_table()[i];
  float m = -INFINITY;
  for (int i = tid; i < V; i += kThreads) m = fmaxf(m, sane(z[i]));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if ((tid & 31) == 0) sm.wmax[tid >> 5] = m;
  __syncthreads();
  for (int i = 0; i < kWarps; ++i) m = fmaxf(m, sm.wmax[i]);
  const bool empty = m == -INFINITY;
  const WeightScale ws = weight_scale(m, r.temperature);
  auto mass = [&](float x) { return weight(x, ws, sm.table); };
  // the cut: keys above `key`, and the first `ties` ids of it
  uint32_t key = logit_key(-kLargest);
  u64 ties = ~0ull;
  if (!empty) {
    if (r.top_k > 0 && r.top_k < V) {
      u64 live = 0, n, before;
      for (int i = tid; i < V; i += kThreads) live += sane(z[i]) > -INFINITY;
      block_scan(live, sm.scan, &n);
      if (static_cast<u64>(r.top_k) < n) {
        key = find_key(z, V, r.top_k, [](float) { return 1ull; }, sm, &before);
        ties = r.top_k - before;
      }
    }
    if (r.top_p < 1.f) {
      u64 mine = 0, at = 0, sum, n_at;
      for (int i = tid; i < V; i += kThreads) {
        const float x = sane(z[i]);
        const uint32_t k = logit_key(x);
        if (x > -INFINITY && k > key) mine += mass(x);
        at += k == key;
      }
      block_scan(mine, sm.scan, &sum);
      block_scan(at, sm.scan, &n_at);
      const u64 one = mass(key_logit(key));
      sum += (ties < n_at ? ties : n_at) * one;
      const u64 f = fraction64(r.top_p);
      u64 need = __umul64hi(f, sum) + (f * sum != 0 ? 1 : 0);
      if (need == 0) need = 1;
      u64 before;
      const uint32_t kp = find_key(z, V, need, mass, sm, &before);
      const u64 w = mass(key_logit(kp)), t = (need - before + w - 1) / w;
      if (kp > key || (kp == key && t < ties)) {
        key = kp;
        ties = t;
      }
    }
    if (r.min_p > 0.f) {
      // the least float z with (z - max) / T >= log(min_p)
      const double c = static_cast<double>(m) +
                       static_cast<double>(r.temperature) * log(static_cast<double>(fminf(r.min_p, 1.f)));
      float cf = static_cast<float>(c);
      if (static_cast<double>(cf) < c) cf = nextafterf(cf, INFINITY);
      const uint32_t km = logit_key(fmaxf(fminf(cf, m), -kLargest));
      if (km > key) {
        key = km;
        ties = ~0ull;
      }
    }
  }
  // the ids in order: which ties are kept, the running sum of kept weights
  const int per = (V + kThreads - 1) / kThreads;
  const int lo = min(tid * per, V), hi = min(lo + per, V);
  u64 at = 0, n_at;
  for (int i = lo; i < hi; ++i) at += logit_key(sane(z[i])) == key;
  u64 seen = block_scan(at, sm.scan, &n_at);
  auto kept = [&](float x, u64& seen) {
    if (x == -INFINITY) return false;
    const uint32_t k = logit_key(x);
    return k > key || (k == key && seen++ < ties);
  };
  if (kMask) {
    float* out = a.out + row * a.out_ld;
    for (int i = lo; i < hi; ++i) {
      const float x = sane(z[i]);
      out[i] = kept(x, seen) ? x : -INFINITY;
    }
    return;
  }
  u64 mine = 0, total, s2 = seen;
  for (int i = lo; i < hi; ++i) {
    const float x = sane(z[i]);
    if (kept(x, s2)) mine += mass(x);
  }
  const u64 before = block_scan(mine, sm.scan, &total);
  const u64 target = __umul64hi(fraction64(a.u[row]), total);
  if (empty) {
    if (tid == 0) a.out_tok[row] = -1;
  } else if (before <= target && target < before + mine) {
    u64 sum = before;
    for (int i = lo; i < hi; ++i) {
      const float x = sane(z[i]);
      if (kept(x, seen)) sum += mass(x);
      if (sum > target) {
        a.out_tok[row] = i;
        break;
      }
    }
  }
}

}  // namespace

cudaError_t launch_filter(const FilterArgs& a, cudaStream_t s, bool pdl) {
  if (a.vocab > kMaxVocab) return cudaErrorInvalidValue;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.rows));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl ? 1 : 0;
  return a.out != nullptr ? cudaLaunchKernelEx(&cfg, filter_kernel<true>, a)
                          : cudaLaunchKernelEx(&cfg, filter_kernel<false>, a);
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
