// kv_append.cu - a projection's rows made into queries, keys and values and put into a cache
// (memspec_op_kv_append), the cache's rows read back (memspec_op_kv_read) and the rotation's
// table (memspec_op_rope_table).
//
// Per head's vector x of a row: x' = x / sqrt(mean(x^2) + eps) * gain, the pairs (i, i + hd/2)
// turned by the position's angle, then bf16, or for a cache of codes rint(x' / s) with
// s = max(max|x'|, 127 * 2^-64) / 127.  Every value is read once and written once, all of it
// elementwise but two sums over a vector: the bound is memory, or at few rows the latency of
// two dependent loads (which sequence, then the angles).  A warp takes whole vectors, so sums
// are shuffles, and a lane holds both values of a pair, so a turn needs no exchange.
#include <algorithm>
#include <string>

#include "kv.cuh"
#include "ptx.cuh"

namespace memspec {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kHeadsPerWarp = 4;   // vectors of a warp, loaded together
constexpr int kHeadsPerCta = kWarps * kHeadsPerWarp;

struct AppendArgs {
  KvView kv;
  const int *starts, *lens;
  int n_seq, rows;
  const void* x;
  long long ldx;             // elements
  const float* rope;         // [2][positions][hd/2] or nullptr
  int positions;
  const int* offsets;        // [rows] or nullptr: the row's place
  long long prefix;
  const bf16 *q_gain, *k_gain;   // [hd] or nullptr
  float eps;
  bf16* q;                   // [rows][n_heads][hd]
  int n_heads;
};

struct ReadArgs {
  KvView kv;
  const int *starts, *lens;
  int n_seq, rows;
  bf16 *k, *v;               // [rows][kv heads][hd]
};

// The row's sequence and its place in it: sequence -1 behind the last one.  All threads call it.
struct RowAt {
  int seq, j, n, len;
};
__device__ __forceinline__ RowAt find_row(const int* starts, const int* lens, int n_seq, int rows, int row, int* shared) {
  const int b = find_sequence(starts, lens, n_seq, rows, row, shared);
  if (b < 0) return {-1, 0, 0, 0};
  const SeqRows s = seq_rows(starts, lens, b, rows);
  return {b, row - s.row0, s.n, s.len};
}

template <int E>
struct Vec {
  float lo[E], hi[E];   // elements E * lane .. and those half a vector further on
};

template <int HD, class T>
__device__ __forceinline__ Vec<HD / 64> load_vec(const T* p, int lane) {
  constexpr int E = HD / 64;
  Vec<E> r;
  if constexpr (sizeof(T) == 4) {
    if constexpr (E == 2) {
      const float2 a = __ldcs(reinterpret_cast<const float2*>(p) + lane);
      const float2 b = __ldcs(reinterpret_cast<const float2*>(p + HD / 2) + lane);
      r.lo[0] = a.x, r.lo[1] = a.y, r.hi[0] = b.x, r.hi[1] = b.y;
    } else {
      r.lo[0] = __ldcs(p + lane);
      r.hi[0] = __ldcs(p + HD / 2 + lane);
    }
  } else {
    if constexpr (E == 2) {
      const uint32_t a = __ldcs(reinterpret_cast<const uint32_t*>(p) + lane);
      const uint32_t b = __ldcs(reinterpret_cast<const uint32_t*>(p + HD / 2) + lane);
      r.lo[0] = __uint_as_float(a << 16), r.lo[1] = __uint_as_float(a & 0xffff0000u);
      r.hi[0] = __uint_as_float(b << 16), r.hi[1] = __uint_as_float(b & 0xffff0000u);
    } else {
      r.lo[0] = __bfloat162float(p[lane]);
      r.hi[0] = __bfloat162float(p[HD / 2 + lane]);
    }
  }
  return r;
}

template <int HD>
__device__ __forceinline__ void store_bf16(bf16* p, const Vec<HD / 64>& v, int lane) {
  if constexpr (HD == 128) {
    reinterpret_cast<__nv_bfloat162*>(p)[lane] = __floats2bfloat162_rn(v.lo[0], v.lo[1]);
    reinterpret_cast<__nv_bfloat162*>(p + HD / 2)[lane] = __floats2bfloat162_rn(v.hi[0], v.hi[1]);
  } else {
    p[lane] = __float2bfloat16_rn(v.lo[0]);
    p[HD / 2 + lane] = __float2bfloat16_rn(v.hi[0]);
  }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  return v;
}
// The largest; a NaN among them is the result, so that a vector with one is known by its scale.
__device__ __forceinline__ float max_nan(float a, float b) { return a > b || isnan(a) ? a : b; }
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = max_nan(v, __shfl_xor_sync(~0u, v, o));
  return v;
}

// Codes of a vector and its scale.  The division is as the definition has it: x / s is rounded
// once, then to a whole number.
template <int HD>
__device__ __forceinline__ void store_codes(char* p, float* scale, const Vec<HD / 64>& v, int lane) {
  constexpr int E = HD / 64;
  float top = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) top = max_nan(max_nan(top, fabsf(v.lo[e])), fabsf(v.hi[e]));
  top = warp_max(top);
  const float s = (top < 127.f * kSmallestScale ? 127.f * kSmallestScale : top) / 127.f;   // a NaN stays
  int8_t lo[E], hi[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    lo[e] = static_cast<int8_t>(__float2int_rn(fminf(fmaxf(v.lo[e] / s, -127.f), 127.f)));
    hi[e] = static_cast<int8_t>(__float2int_rn(fminf(fmaxf(v.hi[e] / s, -127.f), 127.f)));
  }
  if constexpr (E == 2) {
    reinterpret_cast<char2*>(p)[lane] = make_char2(lo[0], lo[1]);
    reinterpret_cast<char2*>(p + HD / 2)[lane] = make_char2(hi[0], hi[1]);
  } else {
    p[lane] = lo[0];
    p[HD / 2 + lane] = hi[0];
  }
  if (lane == 0) *scale = s;
}

template <int HD, class T>
__global__ void __launch_bounds__(kThreads) append_kernel(const __grid_constant__ AppendArgs a) {
  constexpr int E = HD / 64;
  __shared__ int shared;
  const int row = blockIdx.x, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int heads = a.n_heads + 2 * a.kv.n_heads;
  const int h0 = blockIdx.y * kHeadsPerCta + warp * kHeadsPerWarp;
  pdl_wait();
  pdl_launch_dependents();
  Vec<E> v[kHeadsPerWarp];
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
#pragma unroll
  for (int i = 0; i < kHeadsPerWarp; ++i)
    if (h0 + i < heads) v[i] = load_vec<HD>(x + (h0 + i) * HD, lane);
  float gq[2 * E], gk[2 * E];
  if (a.q_gain != nullptr) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      gq[e] = __bfloat162float(a.q_gain[lane * E + e]);
      gq[E + e] = __bfloat162float(a.q_gain[HD / 2 + lane * E + e]);
      gk[e] = __bfloat162float(a.k_gain[lane * E + e]);
      gk[E + e] = __bfloat162float(a.k_gain[HD / 2 + lane * E + e]);
    }
  }
  const RowAt at = find_row(a.starts, a.lens, a.n_seq, a.rows, row, &shared);
  if (at.seq < 0) return;
  const long long first = static_cast<long long>(at.len) - at.n, slot = first + at.j;
  const long long pos = a.prefix + first + (a.offsets != nullptr ? a.offsets[row] : at.j);
  const bool fits = slot >= 0 && slot < a.kv.max_pos && (a.rope == nullptr || (pos >= 0 && pos < a.positions));
  float c[E], s[E];
  if (fits && a.rope != nullptr) {
    const float* cos_t = a.rope + pos * (HD / 2);
    const float* sin_t = cos_t + static_cast<long long>(a.positions) * (HD / 2);
#pragma unroll
    for (int e = 0; e < E; ++e) c[e] = cos_t[lane * E + e], s[e] = sin_t[lane * E + e];
  }
#pragma unroll
  for (int i = 0; i < kHeadsPerWarp; ++i) {
    const int h = h0 + i;
    if (h >= heads) return;
    const bool is_q = h < a.n_heads, is_k = !is_q && h < a.n_heads + a.kv.n_heads;
    if (!fits) {   // nothing is kept of the row
      if (is_q) store_bf16<HD>(a.q + (static_cast<long long>(row) * a.n_heads + h) * HD, Vec<E>{}, lane);
      continue;
    }
    if (is_q || is_k) {
      if (a.q_gain != nullptr) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) sum += v[i].lo[e] * v[i].lo[e] + v[i].hi[e] * v[i].hi[e];
        const float r = rsqrtf(warp_sum(sum) * (1.f / HD) + a.eps);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          v[i].lo[e] = v[i].lo[e] * r * (is_q ? gq[e] : gk[e]);
          v[i].hi[e] = v[i].hi[e] * r * (is_q ? gq[E + e] : gk[E + e]);
        }
      }
      if (a.rope != nullptr) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float lo = v[i].lo[e], hi = v[i].hi[e];
          v[i].lo[e] = lo * c[e] - hi * s[e];
          v[i].hi[e] = lo * s[e] + hi * c[e];
        }
      }
    }
    if (is_q) {
      store_bf16<HD>(a.q + (static_cast<long long>(row) * a.n_heads + h) * HD, v[i], lane);
      continue;
    }
    const int kh = h - a.n_heads - (is_k ? 0 : a.kv.n_heads);
    char* p = (is_k ? a.kv.k : a.kv.v) + at.seq * a.kv.seq + kh * a.kv.head + slot * a.kv.pos;
    if (a.kv.k_scale == nullptr)
      store_bf16<HD>(reinterpret_cast<bf16*>(p), v[i], lane);
    else
      store_codes<HD>(p, (is_k ? a.kv.k_scale : a.kv.v_scale) + at.seq * a.kv.s_seq + kh * a.kv.s_head +
                             slot * a.kv.s_pos, v[i], lane);
  }
}

template <int HD>
__global__ void __launch_bounds__(kThreads) read_kernel(const __grid_constant__ ReadArgs a) {
  constexpr int E = HD / 64;
  __shared__ int shared;
  const int row = blockIdx.x, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  pdl_wait();
  pdl_launch_dependents();
  const RowAt at = find_row(a.starts, a.lens, a.n_seq, a.rows, row, &shared);
  if (at.seq < 0) return;
  const long long slot = static_cast<long long>(at.len) - at.n + at.j;
  const bool fits = slot >= 0 && slot < a.kv.max_pos;
  for (int i = blockIdx.y * kWarps + warp; i < 2 * a.kv.n_heads; i += gridDim.y * kWarps) {
    const bool is_k = i < a.kv.n_heads;
    const int h = is_k ? i : i - a.kv.n_heads;
    Vec<E> v{};
    if (fits) {
      const char* p = (is_k ? a.kv.k : a.kv.v) + at.seq * a.kv.seq + h * a.kv.head + slot * a.kv.pos;
      if (a.kv.k_scale == nullptr) {
        v = load_vec<HD>(reinterpret_cast<const bf16*>(p), lane);
      } else {
        const float s = (is_k ? a.kv.k_scale : a.kv.v_scale)[at.seq * a.kv.s_seq + h * a.kv.s_head + slot * a.kv.s_pos];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          v.lo[e] = s * static_cast<signed char>(p[lane * E + e]);
          v.hi[e] = s * static_cast<signed char>(p[HD / 2 + lane * E + e]);
        }
      }
    }
    store_bf16<HD>((is_k ? a.k : a.v) + (static_cast<long long>(row) * a.kv.n_heads + h) * HD, v, lane);
  }
}

template <class Kernel, class Args>
cudaError_t launch(Kernel* kernel, const Args& a, dim3 grid, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

bool misaligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// Whether n[i] places at strides st[i] (of any order) of `unit` values each never overlap.
bool apart(int64_t unit, const int32_t* n, const int64_t* st) {
  int order[3] = {0, 1, 2};
  std::sort(order, order + 3, [&](int x, int y) { return st[x] < st[y]; });
  int64_t extent = unit;
  for (int i : order) {
    if (n[i] == 1) continue;
    if (st[i] < extent) return false;
    extent += st[i] * (n[i] - 1);
  }
  return true;
}

memspec_status refuse(const char* why) {
  set_op_error(why);
  return MEMSPEC_ERR_INVALID_ARG;
}
memspec_status launched(const char* what, cudaError_t e) {
  if (e == cudaSuccess) return MEMSPEC_OK;
  set_op_error(std::string(what) + " launch: " + cudaGetErrorString(e));
  return MEMSPEC_ERR_CUDA;
}

}  // namespace

const char* kv_problem(const memspec_kv* kv, bool write) {
  if (kv == nullptr || kv->k_dev == nullptr || kv->v_dev == nullptr) return "the cache's k or v is null";
  if ((kv->k_scale_dev == nullptr) != (kv->v_scale_dev == nullptr)) return "scales of both k and v, or of none";
  if (kv->head_dim != 64 && kv->head_dim != 128) return "head_dim must be 64 or 128";
  if (kv->n_seq < 1 || kv->n_heads < 1 || kv->n_heads > 1024 || kv->max_pos < 1 || kv->max_pos > 1 << 30)
    return "the cache needs at least one sequence, 1 to 2^30 positions and 1 to 1024 heads";
  const bool codes = kv->k_scale_dev != nullptr;
  const int32_t n[3] = {kv->n_seq, kv->n_heads, kv->max_pos};
  const int64_t st[3] = {kv->seq_stride, kv->head_stride, kv->pos_stride};
  const int64_t ss[3] = {kv->scale_seq_stride, kv->scale_head_stride, kv->scale_pos_stride};
  for (int i = 0; i < 3; ++i) {
    if (n[i] == 1) continue;
    if (st[i] < (i == 2 ? kv->head_dim : 0) || st[i] > INT64_C(1) << 38 || st[i] % (codes ? 16 : 8) != 0)
      return "the cache's strides must be multiples of 16 bytes, up to 2^38 elements, positions a vector apart";
    if (codes && (ss[i] < 0 || ss[i] > INT64_C(1) << 40)) return "the scales' strides must be 0 to 2^40";
  }
  if (misaligned(kv->k_dev, 16) || misaligned(kv->v_dev, 16) || misaligned(kv->k_scale_dev, 4) ||
      misaligned(kv->v_scale_dev, 4))
    return "k and v must be 16-byte aligned, scales 4-byte";
  if (write && (!apart(kv->head_dim, n, st) || (codes && !apart(1, n, ss)) || kv->k_dev == kv->v_dev ||
                (codes && kv->k_scale_dev == kv->v_scale_dev)))
    return "the cache's vectors overlap";
  return nullptr;
}

KvView kv_view(const memspec_kv* kv) {
  const int size = kv->k_scale_dev != nullptr ? 1 : 2;
  KvView v{};
  v.k = static_cast<char*>(kv->k_dev);
  v.v = static_cast<char*>(kv->v_dev);
  v.k_scale = kv->k_scale_dev;
  v.v_scale = kv->v_scale_dev;
  // of a dimension of one place the stride is not read
  v.seq = kv->n_seq == 1 ? 0 : kv->seq_stride * size;
  v.head = kv->n_heads == 1 ? 0 : kv->head_stride * size;
  v.pos = kv->max_pos == 1 ? 0 : kv->pos_stride * size;
  v.s_seq = kv->n_seq == 1 ? 0 : kv->scale_seq_stride;
  v.s_head = kv->n_heads == 1 ? 0 : kv->scale_head_stride;
  v.s_pos = kv->max_pos == 1 ? 0 : kv->scale_pos_stride;
  v.n_seq = kv->n_seq;
  v.n_heads = kv->n_heads;
  v.max_pos = kv->max_pos;
  return v;
}

const char* batch_problem(const memspec_batch* b, const memspec_kv* kv) {
  if (b == nullptr || b->starts_dev == nullptr || b->lens_dev == nullptr) return "starts or lens is null";
  if (misaligned(b->starts_dev, 4) || misaligned(b->lens_dev, 4)) return "starts and lens must be 4-byte aligned";
  if (b->n_seq < 1 || b->n_seq > kMaxSeqs || b->n_seq > kv->n_seq)
    return "sequences: 1 to 1024, and at most the cache's";
  if (b->rows < 1 || b->rows > kMaxCallRows) return "rows must be in 1..65535";
  return nullptr;
}

}  // namespace memspec

extern "C" {

memspec_status memspec_op_rope_table(int32_t positions, int32_t head_dim, float base, float* table, void* stream) {
  using namespace memspec;
  if (table == nullptr || misaligned(table, 4)) return refuse("the table is null or misaligned");
  if (head_dim < 2 || head_dim % 2 != 0 || head_dim > 1024 || positions < 1 ||
      static_cast<int64_t>(positions) * (head_dim / 2) >= (INT64_C(1) << 31) - 256)
    return refuse("head_dim must be even in 2..1024, positions at least 1, positions * head_dim / 2 below 2^31 - 256");
  if (!(base > 0.f) || base > 3e38f) return refuse("base must be positive and finite");
  const int half = head_dim / 2;
  return launched("rope table", launch_rope_table(table, table + static_cast<int64_t>(positions) * half, positions,
                                                  half, base, static_cast<cudaStream_t>(stream)));
}

memspec_status memspec_op_kv_append(const memspec_batch* batch, const memspec_kv* kv, const memspec_append* p,
                                    void* stream) {
  using namespace memspec;
  if (const char* why = kv_problem(kv, true)) return refuse(why);
  if (const char* why = batch_problem(batch, kv)) return refuse(why);
  if (p == nullptr || p->qkv_dev == nullptr || p->q_dev == nullptr) return refuse("qkv or q is null");
  if (p->qkv_type != MEMSPEC_F32 && p->qkv_type != MEMSPEC_BF16) return refuse("qkv must be fp32 or bf16");
  const int hd = kv->head_dim, size = p->qkv_type == MEMSPEC_F32 ? 4 : 2;
  if (p->n_heads < 1 || p->n_heads > 1024) return refuse("n_heads must be in 1..1024");
  if (batch->rows > 1 && (p->ld < static_cast<int64_t>(p->n_heads + 2 * kv->n_heads) * hd || p->ld % 2 != 0 ||
                          p->ld > INT64_C(1) << 40))
    return refuse("qkv's row stride must be even, cover a row and be at most 2^40");
  if (misaligned(p->qkv_dev, 2 * size) || misaligned(p->q_dev, 4) || misaligned(p->rope_dev, 4) ||
      misaligned(p->offsets_dev, 4) || misaligned(p->q_gain_dev, 2) || misaligned(p->k_gain_dev, 2))
    return refuse("qkv must be aligned to two elements, q, the table and offsets to 4 bytes, gains to 2");
  if (p->rope_dev != nullptr && p->rope_positions < 1) return refuse("the table has no positions");
  if (p->prefix_len < 0) return refuse("prefix_len must not be negative");
  if ((p->q_gain_dev == nullptr) != (p->k_gain_dev == nullptr)) return refuse("gains of both q and k, or of none");
  if (!(p->eps >= 0.f) || p->eps > 3e38f) return refuse("eps must be at least 0 and finite");
  AppendArgs a{};
  a.kv = kv_view(kv);
  a.starts = batch->starts_dev;
  a.lens = batch->lens_dev;
  a.n_seq = batch->n_seq;
  a.rows = batch->rows;
  a.x = p->qkv_dev;
  a.ldx = batch->rows > 1 ? p->ld : 0;
  a.rope = p->rope_dev;
  a.positions = p->rope_positions;
  a.offsets = p->offsets_dev;
  a.prefix = p->prefix_len;
  a.q_gain = static_cast<const bf16*>(p->q_gain_dev);
  a.k_gain = static_cast<const bf16*>(p->k_gain_dev);
  a.eps = p->eps;
  a.q = static_cast<bf16*>(p->q_dev);
  a.n_heads = p->n_heads;
  const dim3 grid(batch->rows, (p->n_heads + 2 * kv->n_heads + kHeadsPerCta - 1) / kHeadsPerCta);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  return launched("kv append", size == 4 ? (hd == 64 ? launch(append_kernel<64, float>, a, grid, s)
                                                     : launch(append_kernel<128, float>, a, grid, s))
                                         : (hd == 64 ? launch(append_kernel<64, bf16>, a, grid, s)
                                                     : launch(append_kernel<128, bf16>, a, grid, s)));
}

memspec_status memspec_op_kv_read(const memspec_batch* batch, const memspec_kv* kv, void* k, void* v, void* stream) {
  using namespace memspec;
  if (const char* why = kv_problem(kv, false)) return refuse(why);
  if (const char* why = batch_problem(batch, kv)) return refuse(why);
  if (k == nullptr || v == nullptr || misaligned(k, 4) || misaligned(v, 4))
    return refuse("k and v must be 4-byte aligned and not null");
  ReadArgs a{};
  a.kv = kv_view(kv);
  a.starts = batch->starts_dev;
  a.lens = batch->lens_dev;
  a.n_seq = batch->n_seq;
  a.rows = batch->rows;
  a.k = static_cast<bf16*>(k);
  a.v = static_cast<bf16*>(v);
  const dim3 grid(batch->rows, (2 * kv->n_heads + 2 * kWarps - 1) / (2 * kWarps));
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  return launched("kv read", kv->head_dim == 64 ? launch(read_kernel<64>, a, grid, s)
                                                : launch(read_kernel<128>, a, grid, s));
}

}  // extern "C"
