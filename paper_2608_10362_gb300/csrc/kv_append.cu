// kv_append.cu - a projection's rows made into queries, keys and values and put into a cache
// (memspec_op_kv_append), the cache's rows read back (memspec_op_kv_read) and the rotation's
// table (memspec_op_rope_table).
//
// Per head's vector x of a row: x' = x / sqrt(mean(x^2) + eps) * gain, the pairs (i, i + hd/2)
// turned by the position's angle, then bf16, or for a cache of codes rint(x' / s) with
// s = max(max|x'|, 127 * 2^-64) / 127.  Every value is read once and written once, all of it
// elementwise but two sums over a vector: the bound is memory, or at few rows the latency of
// two dependent loads (which sequence, then the angles).  hd / 8 lanes take a vector, four
// elements of each half a lane: a pair is in one lane, so that a turn needs no exchange, two or
// four vectors share a warp's sums and every access is 8 or 16 bytes.  2047 rows of 96 heads of
// bf16: 24 us, 4.3 TB/s, in eight waves of short CTAs (a vector per warp, 4 bytes a lane: 33, bound
// by issue; fewer CTAs that take rows in turn 31; arithmetic in pairs no less).  One row: 2.0 us.
#include <algorithm>
#include <string>

#include "kv.cuh"
#include "ptx.cuh"

namespace memspec {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kSets = 2;           // vectors of a lane, loaded together (2047 rows: 1 28.4 us, 2 24.4, 4 30.6)

template <int HD>
struct Lanes {
  static constexpr int kLanes = HD / 8, kVectors = 32 / kLanes;   // of a vector; vectors at a time
  static constexpr int kHeads = kVectors * kSets * kWarps;        // of a CTA
};

struct AppendArgs {
  KvView kv;
  const int *starts, *lens;
  int n_seq, rows;
  const void* x;
  long long ldx;             // elements
  bool wide;                 // x and its rows are aligned to four elements
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
  const int b = n_seq == 1 ? 0 : find_sequence(starts, lens, n_seq, rows, row, shared);
  if (b < 0) return {-1, 0, 0, 0};
  const SeqRows s = seq_rows(starts, lens, b, rows);
  if (row < s.row0 || row >= s.row0 + s.n) return {-1, 0, 0, 0};
  return {b, row - s.row0, s.n, s.len};
}

__device__ __forceinline__ float2 bf16_pair(uint32_t v) {
  return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
__device__ __forceinline__ float4 two_pairs(uint32_t a, uint32_t b) {
  const float2 x = bf16_pair(a), y = bf16_pair(b);
  return make_float4(x.x, x.y, y.x, y.y);
}
// Four elements; p is aligned to four of them, or (wide: false) to two.
template <class T>
__device__ __forceinline__ float4 load4(const T* p, bool wide) {
  if constexpr (sizeof(T) == 4) {
    if (wide) return __ldcs(reinterpret_cast<const float4*>(p));
    const float2 a = __ldcs(reinterpret_cast<const float2*>(p)), b = __ldcs(reinterpret_cast<const float2*>(p) + 1);
    return make_float4(a.x, a.y, b.x, b.y);
  } else {
    if (wide) {
      const uint2 v = __ldcs(reinterpret_cast<const uint2*>(p));
      return two_pairs(v.x, v.y);
    }
    return two_pairs(__ldcs(reinterpret_cast<const uint32_t*>(p)), __ldcs(reinterpret_cast<const uint32_t*>(p) + 1));
  }
}
__device__ __forceinline__ float4 gain4(const bf16* p) {
  const uint2 v = *reinterpret_cast<const uint2*>(p);
  return two_pairs(v.x, v.y);
}
__device__ __forceinline__ void store4(bf16* p, const float4& v) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
__device__ __forceinline__ float4 mul(const float4& a, const float4& b) {
  return make_float4(a.x * b.x, a.y * b.y, a.z * b.z, a.w * b.w);
}
__device__ __forceinline__ float4 mul(const float4& a, float b) { return make_float4(a.x * b, a.y * b, a.z * b, a.w * b); }
__device__ __forceinline__ float dot(const float4& a) { return a.x * a.x + a.y * a.y + a.z * a.z + a.w * a.w; }

// The larger; a NaN is the result, so that a vector with one is known by its scale.
__device__ __forceinline__ float max_nan(float a, float b) { return a > b || isnan(a) ? a : b; }
__device__ __forceinline__ float top4(const float4& a) {
  return max_nan(max_nan(fabsf(a.x), fabsf(a.y)), max_nan(fabsf(a.z), fabsf(a.w)));
}
// Codes as the definition has them: x / s is rounded once, then to a whole number.
__device__ __forceinline__ void store_codes4(char* p, const float4& v, float s) {
  auto code = [s](float x) { return __float2int_rn(fminf(fmaxf(x / s, -127.f), 127.f)) & 255; };
  *reinterpret_cast<int*>(p) = code(v.x) | code(v.y) << 8 | code(v.z) << 16 | code(v.w) << 24;
}

template <int HD, class T>
__global__ void __launch_bounds__(kThreads) append_kernel(const __grid_constant__ AppendArgs a) {
  typedef Lanes<HD> L;
  __shared__ int shared;
  const int row = blockIdx.x, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int e = lane % L::kLanes * 4;    // the lane's elements: e .. e + 3 of each half
  const int heads = a.n_heads + 2 * a.kv.n_heads;
  const int h0 = blockIdx.y * L::kHeads + warp * L::kVectors * kSets + lane / L::kLanes;
  pdl_wait();
  pdl_launch_dependents();
  float4 lo[kSets], hi[kSets];
  const T* x = static_cast<const T*>(a.x) + row * a.ldx + e;
#pragma unroll
  for (int i = 0; i < kSets; ++i) {
    const int h = min(h0 + i * L::kVectors, heads - 1);
    lo[i] = load4(x + h * HD, a.wide);
    hi[i] = load4(x + h * HD + HD / 2, a.wide);
  }
  const RowAt at = find_row(a.starts, a.lens, a.n_seq, a.rows, row, &shared);
  if (at.seq < 0) return;
  const long long first = static_cast<long long>(at.len) - at.n, slot = first + at.j;
  const long long pos = a.prefix + first + (a.offsets != nullptr ? a.offsets[row] : at.j);
  const bool fits = slot >= 0 && slot < a.kv.max_pos && (a.rope == nullptr || (pos >= 0 && pos < a.positions));
  float4 c = make_float4(1.f, 1.f, 1.f, 1.f), s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (fits && a.rope != nullptr) {
    const float* cos_t = a.rope + pos * (HD / 2) + e;
    c = *reinterpret_cast<const float4*>(cos_t);
    s = *reinterpret_cast<const float4*>(cos_t + static_cast<long long>(a.positions) * (HD / 2));
  }
#pragma unroll
  for (int i = 0; i < kSets; ++i) {   // every lane goes through the sums, whatever its vector is
    const int h = h0 + i * L::kVectors;
    const bool is_q = h < a.n_heads, is_k = !is_q && h < a.n_heads + a.kv.n_heads;
    if (a.q_gain != nullptr) {
      float sum = dot(lo[i]) + dot(hi[i]);
#pragma unroll
      for (int o = L::kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
      if (is_q || is_k) {
        const bf16* g = (is_q ? a.q_gain : a.k_gain) + e;
        const float r = rsqrtf(sum * (1.f / HD) + a.eps);
        lo[i] = mul(mul(lo[i], r), gain4(g));
        hi[i] = mul(mul(hi[i], r), gain4(g + HD / 2));
      }
    }
    if (a.rope != nullptr && (is_q || is_k)) {
      const float4 l = lo[i], u = hi[i];
      lo[i] = make_float4(l.x * c.x - u.x * s.x, l.y * c.y - u.y * s.y, l.z * c.z - u.z * s.z, l.w * c.w - u.w * s.w);
      hi[i] = make_float4(l.x * s.x + u.x * c.x, l.y * s.y + u.y * c.y, l.z * s.z + u.z * c.z, l.w * s.w + u.w * c.w);
    }
    float scale = 0.f;
    if (a.kv.k_scale != nullptr) {
      float top = max_nan(top4(lo[i]), top4(hi[i]));
#pragma unroll
      for (int o = L::kLanes / 2; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(~0u, top, o));
      scale = (top < 127.f * kSmallestScale ? 127.f * kSmallestScale : top) / 127.f;   // a NaN stays
    }
    if (h >= heads) continue;
    const int kh = h - a.n_heads - (is_k ? 0 : a.kv.n_heads);
    char* p = (is_k ? a.kv.k : a.kv.v) + at.seq * a.kv.seq + kh * a.kv.head + slot * a.kv.pos;
    if (is_q || a.kv.k_scale == nullptr) {
      bf16* to = is_q ? a.q + (static_cast<long long>(row) * a.n_heads + h) * HD : reinterpret_cast<bf16*>(p);
      if (!fits) {   // nothing is kept of the row
        if (!is_q) continue;
        lo[i] = hi[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
      store4(to + e, lo[i]);
      store4(to + e + HD / 2, hi[i]);
    } else if (fits) {
      store_codes4(p + e, lo[i], scale);
      store_codes4(p + e + HD / 2, hi[i], scale);
      if (e == 0)
        (is_k ? a.kv.k_scale : a.kv.v_scale)[at.seq * a.kv.s_seq + kh * a.kv.s_head + slot * a.kv.s_pos] = scale;
    }
  }
}

template <int HD>
__global__ void __launch_bounds__(kThreads) read_kernel(const __grid_constant__ ReadArgs a) {
  typedef Lanes<HD> L;
  __shared__ int shared;
  const int row = blockIdx.x, warp = threadIdx.x / 32, lane = threadIdx.x % 32, e = lane % L::kLanes * 4;
  pdl_wait();
  pdl_launch_dependents();
  const RowAt at = find_row(a.starts, a.lens, a.n_seq, a.rows, row, &shared);
  if (at.seq < 0) return;
  const long long slot = static_cast<long long>(at.len) - at.n + at.j;
  const bool fits = slot >= 0 && slot < a.kv.max_pos;
#pragma unroll
  for (int i = 0; i < kSets; ++i) {
    const int at_h = blockIdx.y * L::kHeads + (warp * kSets + i) * L::kVectors + lane / L::kLanes;
    if (at_h >= 2 * a.kv.n_heads) return;
    const bool is_k = at_h < a.kv.n_heads;
    const int h = is_k ? at_h : at_h - a.kv.n_heads;
    float4 lo = make_float4(0.f, 0.f, 0.f, 0.f), hi = lo;
    if (fits) {
      const char* p = (is_k ? a.kv.k : a.kv.v) + at.seq * a.kv.seq + h * a.kv.head + slot * a.kv.pos;
      if (a.kv.k_scale == nullptr) {
        lo = load4(reinterpret_cast<const bf16*>(p) + e, true);
        hi = load4(reinterpret_cast<const bf16*>(p) + e + HD / 2, true);
      } else {
        float s = (is_k ? a.kv.k_scale : a.kv.v_scale)[at.seq * a.kv.s_seq + h * a.kv.s_head + slot * a.kv.s_pos];
        if (s < kSmallestScale) s = kSmallestScale;   // a NaN stays
        const char4 l = *reinterpret_cast<const char4*>(p + e), u = *reinterpret_cast<const char4*>(p + e + HD / 2);
        auto value = [s](const char4& v) {
          return make_float4(s * static_cast<signed char>(v.x), s * static_cast<signed char>(v.y),
                             s * static_cast<signed char>(v.z), s * static_cast<signed char>(v.w));
        };
        lo = value(l), hi = value(u);
      }
    }
    bf16* to = (is_k ? a.k : a.v) + (static_cast<long long>(row) * a.kv.n_heads + h) * HD + e;
    store4(to, lo);
    store4(to + HD / 2, hi);
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
  if (misaligned(p->qkv_dev, 2 * size) || misaligned(p->q_dev, 8) || misaligned(p->rope_dev, 16) ||
      misaligned(p->offsets_dev, 4) || misaligned(p->q_gain_dev, 8) || misaligned(p->k_gain_dev, 8))
    return refuse("qkv must be aligned to two elements, the table to 16 bytes, q and gains to 8, offsets to 4");
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
  a.wide = a.ldx % 4 == 0 && !misaligned(p->qkv_dev, 4 * size);
  a.rope = p->rope_dev;
  a.positions = p->rope_positions;
  a.offsets = p->offsets_dev;
  a.prefix = p->prefix_len;
  a.q_gain = static_cast<const bf16*>(p->q_gain_dev);
  a.k_gain = static_cast<const bf16*>(p->k_gain_dev);
  a.eps = p->eps;
  a.q = static_cast<bf16*>(p->q_dev);
  a.n_heads = p->n_heads;
  const int at_once = hd == 64 ? Lanes<64>::kHeads : Lanes<128>::kHeads;
  const dim3 grid(batch->rows, (p->n_heads + 2 * kv->n_heads + at_once - 1) / at_once);
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
  if (k == nullptr || v == nullptr || misaligned(k, 8) || misaligned(v, 8))
    return refuse("k and v must be 8-byte aligned and not null");
  ReadArgs a{};
  a.kv = kv_view(kv);
  a.starts = batch->starts_dev;
  a.lens = batch->lens_dev;
  a.n_seq = batch->n_seq;
  a.rows = batch->rows;
  a.k = static_cast<bf16*>(k);
  a.v = static_cast<bf16*>(v);
  const int at_once = kv->head_dim == 64 ? Lanes<64>::kHeads : Lanes<128>::kHeads;
  const dim3 grid(batch->rows, (2 * kv->n_heads + at_once - 1) / at_once);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  return launched("kv read", kv->head_dim == 64 ? launch(read_kernel<64>, a, grid, s)
                                                : launch(read_kernel<128>, a, grid, s));
}

}  // extern "C"
