// attn_join.cu - memspec_op_attention: which kernels a call's parts run, and the launch that joins
// the records of units whose keys several CTAs had (attn_plan.cuh).
//
// A record is HD sums of weights times values, the maximum the weights were taken against and their
// sum; records of one vector add up after each is scaled to the largest maximum, in the order of
// the line.  Two launches do it, for the two ways in which the kernels leave them.
#include <algorithm>
#include <string>

#include "attn_plan.cuh"
#include "ptx.cuh"

namespace memspec {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kTilesUnit = TileUnits::kUnit;
// Up to so many vectors per head of k and v: attn_rows.cu, in units of 8 or 16; more: attn_tiles.cu.  bf16 and codes, caches
// cold, attn_rows.cu / attn_tiles.cu, us:
//                                           8 vectors                16                       24
//   16 sequences of 2048, 8 heads of 128    28.0 / 33.3, 21.4 / 39.2  29.3 / 33.2, 33.9 / 39.0  44.8 / 34.4, 50.6 / 39.6
//   64 of 512, 8 heads of 128               32.8 / 36.0, 24.6 / 42.2  38.4 / 40.2, 39.0 / 46.9  54.8 / 44.0, 61.2 / 52.2
//   one of 16384, 8 heads of 128            21.2 / 30.5, 18.5 / 32.5  23.0 / 27.7, 25.6 / 31.0  24.4 / 31.0, 31.9 / 33.9
//   16 of 2048, 4 heads of 64               13.5 / 19.3, 12.6 / 21.2  14.7 / 18.5, 14.1 / 20.9  18.7 / 19.3, 18.9 / 21.7
// At 24 it is the keys that decide (two units read them twice), which the host does not know; attn_tiles.cu loses
// the least there.  Units of 16 for 4 vectors: 64 sequences of 16384 codes 590 us for 315 (what 8 vectors more cost is all lost).
constexpr int kRowsVectors = 16;

// Where a vector's records of a part are.
struct Records {
  int n;               // 0: the result is written already
  const float *sums, *md;   // of the first one: 4 of its sums, its maximum and sum of weights
  long long chunk;     // floats from 4 sums of it to the next 4
  int copies;          // of each CTA, one after another
  int copy, md_copy;   // floats from a CTA's copy to the next
  int record;          // floats of a unit's; the first CTA's is its second one, the others' their first
  __device__ int at(int c) const { return c == 0 ? 0 : (2 * c - 1) * record; }
};
template <int HD>
__device__ __forceinline__ Records records_of(const JoinArgs& a, const JoinPart& part, int seq, const SeqRows& found, int row,
                                              int h, int kv_head) {
  const bool own = part.at < 0;
  const int b = own ? seq : part.at, heads = a.group * a.kv_heads;
  const uint32_t base = part.bases[b], total = part.bases[part.list];
  const uint32_t vecs = (own ? found.n : a.rows) * a.group, vec = (row - (own ? found.row0 : 0)) * a.group + h - kv_head * a.group;
  const uint32_t tiles = tiles_of(own ? min(max(found.len, 0), a.max_pos) : part.keys);
  const uint32_t unit = vec / part.unit, in_unit = vec - unit * part.unit;
  int c0, c1;   // who has the first tile, and the last one: all between them have some
  bool pair;
  auto find = [&](auto cut, uint32_t per_head, uint32_t per_unit) {
    typedef decltype(cut) CUT;
    const uint32_t t0 = base + kv_head * per_head + unit * per_unit;
    const Pieces pieces(part.ctas, total, CUT::kGrain);
    pair = CUT::pair(vecs, unit);
    c0 = pieces.owner(t0 + CUT::place_of(0, pair));
    c1 = pieces.owner(t0 + CUT::place_of(tiles - 1, pair));
  };
  if (part.pairs)
    find(TileUnits{}, TileUnits::per_head(vecs, tiles), TileUnits::per_unit(tiles));
  else if (part.unit == 8)
    find(RowUnits<8>{}, RowUnits<8>::per_head(vecs, tiles), RowUnits<8>::per_unit(tiles));
  else
    find(RowUnits<16>{}, RowUnits<16>::per_head(vecs, tiles), RowUnits<16>::per_unit(tiles));
  // attn_rows.cu's records are one after another, one of a CTA; attn_tiles.cu's side by side, of its smaller units two
  const bool whole = c0 == c1;
  const long long all = static_cast<long long>(a.rows) * heads, i = whole ? static_cast<long long>(row) * heads + h : in_unit;
  const long long side = whole ? 2 * all : part.unit;
  const int record = part.unit * kRecord<HD>;
  Records r;
  r.copies = part.pairs && !pair ? 2 : 1;
  r.n = whole && part.full == nullptr ? 0 : (c1 - c0 + 1) * r.copies;
  const float* first = whole ? part.full : part.slots + (2ll * c0 + 1) * record;   // (of that CTA's two the one that begins a unit)
  r.sums = first + i * (part.pairs ? 4 : kRecord<HD>);
  r.md = part.pairs ? first + HD * side + 2 * i : r.sums + HD;
  r.chunk = part.pairs ? 4 * side : 4;
  r.copy = static_cast<int>(whole ? all : 128) * 4;
  r.md_copy = r.copy / 2;
  r.record = record;
  return r;
}

// Records of attn_rows.cu alone, of one vector up to one per CTA (one row of 32 / 8 heads over 8192 codes: 38): a warp
// to a row's head, kAtOnce of its records under way, its lanes the elements of a record, which are one after another.
constexpr int kAtOnce = 8;   // (that case 14.2 us; 4: 17.7, 16: 13.5, and calls with few records 0.5 more than with 4)
template <int HD>
__global__ void __launch_bounds__(kThreads) join_rows_kernel(const __grid_constant__ JoinArgs a) {
  constexpr int E = HD / 32;
  __shared__ int shared;
  const int row = blockIdx.x, warp = threadIdx.x / 32, lane = threadIdx.x % 32, heads = a.group * a.kv_heads;
  // (starts and lens were complete before the launch before this one began)
  const int seq = find_sequence(a.starts, a.lens, a.n_seq, a.rows, row, &shared);
  const SeqRows found = seq < 0 ? SeqRows{} : seq_rows(a.starts, a.lens, seq, a.rows);
  pdl_wait();
  pdl_launch_dependents();
  const int h = blockIdx.y * kWarps + warp;
  if (seq < 0 || h >= heads) return;
  float top = kStart, den = 0.f, sum[E] = {};
  bool any = false;
#pragma unroll 1
  for (int p = 0; p < a.parts; ++p) {
    const Records rec = records_of<HD>(a, a.part[p], seq, found, row, h, h / a.group);
    any |= rec.n > 0;
#pragma unroll 1
    for (int i0 = 0; i0 < rec.n; i0 += 32) {   // a lane has a record's maximum and sum of weights
      const int here = min(rec.n - i0, 32);
      float2 md = make_float2(kStart, 0.f);
      if (lane < here) md = *reinterpret_cast<const float2*>(rec.md + rec.at(i0 + lane));
      float now = fmaxf(top, md.x);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) now = fmaxf(now, __shfl_xor_sync(~0u, now, o));
      const float was = ex2(top - now), by = lane < here ? ex2(md.x - now) : 0.f;
      float d = by * md.y;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(~0u, d, o);
      den = fmaf(den, was, d);
#pragma unroll
      for (int e = 0; e < E; ++e) sum[e] *= was;
#pragma unroll 1
      for (int r0 = 0; r0 < here; r0 += kAtOnce) {   // (past the last one: that one, times 0)
        float2 x[kAtOnce][E / 2];
#pragma unroll
        for (int r = 0; r < kAtOnce; ++r) {
          const float* at = rec.sums + rec.at(i0 + min(r0 + r, here - 1)) + lane * E;
          if constexpr (E == 4) {
            const float4 y = *reinterpret_cast<const float4*>(at);
            x[r][0] = make_float2(y.x, y.y), x[r][E / 2 - 1] = make_float2(y.z, y.w);
          } else {
            x[r][0] = *reinterpret_cast<const float2*>(at);
          }
        }
#pragma unroll
        for (int r = 0; r < kAtOnce; ++r) {
          const float f = __shfl_sync(~0u, by, r0 + r);
#pragma unroll
          for (int e = 0; e < E; e += 2)
            sum[e] = fmaf(x[r][e / 2].x, f, sum[e]), sum[e + 1] = fmaf(x[r][e / 2].y, f, sum[e + 1]);
        }
      }
      top = now;
    }
  }
  if (!any) return;
  const float by = den == 0.f ? 0.f : 1.f / den;
  uint32_t* out = reinterpret_cast<uint32_t*>(a.out + row * a.ldo + h * HD + lane * E);
#pragma unroll
  for (int e = 0; e < E; e += 2) out[e / 2] = pack_bf16(sum[e] * by, sum[e + 1] * by);
}

// Where attn_tiles.cu's are among them: a lane to a vector, a warp to four elements of 32 vectors, so that its loads
// are 512 bytes in a row (a warp to a row's head, 16 bytes each from 32 places: 64 rows over 8192 positions 11 us more).
template <int HD>
__global__ void __launch_bounds__(kThreads) join_tiles_kernel(const __grid_constant__ JoinArgs a) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, kv_head = blockIdx.y;
  const uint32_t vec = blockIdx.x * 32 + lane;
  const int row = min(a.group_magic == 0 ? vec : __umulhi(vec, a.group_magic), a.rows - 1u);
  const int h = kv_head * a.group + vec - row * a.group, chunk = blockIdx.z * kWarps + warp;
  int seq = 0;   // (starts and lens were complete before the launch before this one began)
#pragma unroll 1
  for (int end = a.n_seq; end - seq > 1;) {   // the last one that begins at or before the row
    const int mid = (seq + end) / 2;
    if (a.starts[mid] <= row)
      seq = mid;
    else
      end = mid;
  }
  const SeqRows found = seq_rows(a.starts, a.lens, seq, a.rows);
  pdl_wait();
  pdl_launch_dependents();
  if (row < found.row0 || row >= found.row0 + found.n || vec >= static_cast<uint32_t>(a.rows) * a.group || chunk >= HD / 4) return;
  float top = kStart, den = 0.f, sum[4] = {};
#pragma unroll 1
  for (int p = 0; p < a.parts; ++p) {
    const Records rec = records_of<HD>(a, a.part[p], seq, found, row, h, kv_head);
    const float* const sums = rec.sums + chunk * rec.chunk;
    const int twice = rec.copies - 1;
#pragma unroll 4
    for (int r = 0; r < rec.n; ++r) {
      const int at = rec.at(r >> twice), copy = r & twice;
      const float2 md = *reinterpret_cast<const float2*>(rec.md + at + copy * rec.md_copy);
      const float now = fmaxf(top, md.x), was = ex2(top - now), by = ex2(md.x - now);
      top = now;
      den = fmaf(den, was, by * md.y);
      const float4 x = *reinterpret_cast<const float4*>(sums + at + copy * rec.copy);
      sum[0] = fmaf(x.x, by, sum[0] * was), sum[1] = fmaf(x.y, by, sum[1] * was);
      sum[2] = fmaf(x.z, by, sum[2] * was), sum[3] = fmaf(x.w, by, sum[3] * was);
    }
  }
  // weights of codes carry V's scale, so that their sum is down to 2^-129: its reciprocal may be past fp32, the result is not
  const float lift = den < 0x1p-60f ? 0x1p30f : 1.f, by = den == 0.f ? 0.f : 1.f / (den * lift);
#pragma unroll
  for (int e = 0; e < 4; ++e) sum[e] = sum[e] * lift * by;
  *reinterpret_cast<uint2*>(a.out + row * a.ldo + h * HD + chunk * 4) =
      make_uint2(pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3]));
}

// ---------------------------------------------------------------- host
// A launch of one of the two kernels over the batch's own keys, the prefix's, or both.
struct Launch {
  bool tiles, own, prefix, codes;
  int nt;                       // attn_rows.cu: units of 8 nt vectors
  size_t bases, slots;          // in the scratch
  int ctas() const { return tiles ? kTilesCtas : rows_ctas(codes); }
  int unit() const { return tiles ? kTilesUnit : 8 * nt; }
};
struct Layout {
  Launch launch[2];
  int n;
  size_t full[2], total;        // records of the cache's, of the prefix's units
};

Layout lay_out(const memspec_batch* b, const memspec_kv* kv, const memspec_attention* p) {
  Layout l{};
  const int group = p->n_heads / kv->n_heads;
  const bool two = p->prefix != nullptr && p->prefix_len > 0;
  auto launch = [&](const memspec_kv* part, long long vecs) {
    Launch x{};
    x.codes = part->k_scale_dev != nullptr;
    x.tiles = vecs > kRowsVectors;
    x.nt = vecs > 8 ? 2 : 1;
    return x;
  };
  l.launch[0] = launch(kv, static_cast<long long>(p->max_rows) * group);
  l.launch[0].own = true;
  l.n = 1;
  if (two) {
    Launch x = launch(p->prefix, static_cast<long long>(b->rows) * group);
    x.prefix = true;
    if (x.tiles && l.launch[0].tiles && x.codes == l.launch[0].codes) {
      // one launch of attn_tiles.cu for both (16 x 9 rows behind 8192 positions, 300 of their own: 40.0 us, two launches
      // 44.8).  Few own vectors stay attn_rows.cu's, and the prefix's launch does not wait for theirs (64 rows behind
      // 32768 codes, up to 1024 of their own: 73.1, waiting 75.2, all in one launch 83.7)
      x.own = true;
      l.launch[0] = x;
    } else {
      l.launch[l.n++] = x;
    }
  }
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t was = at;
    at += (bytes + 255) & ~size_t{255};
    return was;
  };
  const size_t record = (kv->head_dim + 4) * sizeof(float);
  const size_t all = static_cast<size_t>(b->rows) * p->n_heads * record;
  for (int i = 0; i < l.n; ++i) {
    Launch& x = l.launch[i];
    x.bases = take((static_cast<size_t>(b->n_seq) + 2) * sizeof(uint32_t));
    x.slots = take(size_t{2} * x.ctas() * x.unit() * record);
    // (attn_tiles.cu leaves two records of a vector, and never writes the result itself)
    if (x.own && (two || x.tiles)) l.full[0] = take(all * (x.tiles ? 2 : 1));
    if (x.prefix) l.full[1] = take(all * (x.tiles ? 2 : 1));
  }
  l.total = at;
  return l;
}

bool misaligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

const char* attention_problem(const memspec_batch* b, const memspec_kv* kv, const memspec_attention* p) {
  if (const char* why = kv_problem(kv, false)) return why;
  if (const char* why = batch_problem(b, kv)) return why;
  if (p == nullptr) return "null pointer";
  if (p->n_heads < 1 || p->n_heads % kv->n_heads != 0 || p->n_heads / kv->n_heads > 64)
    return "n_heads must be a multiple of the cache's heads, up to 64 times as many";
  if (p->max_rows < 1 || p->max_rows > b->rows) return "max_rows must be in 1..rows";
  if (!(fabsf(p->scale) <= 2e38f)) return "scale must be at most 2e38";   // (times log2(e) finite)
  if (p->prefix != nullptr) {
    if (const char* why = kv_problem(p->prefix, false)) return why;
    if (p->prefix->n_heads != kv->n_heads || p->prefix->head_dim != kv->head_dim)
      return "the prefix must have the cache's heads and head_dim";
    if (p->prefix_len < 0 || p->prefix_len > p->prefix->max_pos) return "prefix_len must be in 0..the prefix's max_pos";
  }
  // the line is counted in 32 bits: a unit per 8 vectors, each of all tiles, is more than there can be
  const double units = static_cast<double>(b->rows) * (p->n_heads / kv->n_heads) / 8 + TileUnits::kGrain * (b->n_seq + 1);
  const double keys = std::max(kv->max_pos, p->prefix != nullptr ? p->prefix_len : 0);
  if (units * kv->n_heads * (keys / kTile + 16) >= 3.5e9) return "too many rows for so many positions: split the call";
  return nullptr;
}

}  // namespace
}  // namespace memspec

extern "C" {

memspec_status memspec_op_attention_scratch_bytes(const memspec_batch* batch, const memspec_kv* kv,
                                                  const memspec_attention* p, size_t* bytes) {
  using namespace memspec;
  const char* why = bytes == nullptr ? "null pointer" : attention_problem(batch, kv, p);
  if (why != nullptr) {
    set_op_error(why);
    return MEMSPEC_ERR_INVALID_ARG;
  }
  *bytes = lay_out(batch, kv, p).total;
  return MEMSPEC_OK;
}

memspec_status memspec_op_attention(const memspec_batch* batch, const memspec_kv* kv, const memspec_attention* p,
                                    void* scratch, size_t scratch_bytes, void* stream) {
  using namespace memspec;
  const char* why = attention_problem(batch, kv, p);
  Layout l{};
  if (why == nullptr) {
    const int64_t row = static_cast<int64_t>(p->n_heads) * kv->head_dim;
    l = lay_out(batch, kv, p);
    if (p->q_dev == nullptr || p->out_dev == nullptr || scratch == nullptr) {
      why = "null pointer";
    } else if (misaligned(p->q_dev, 16) || misaligned(p->out_dev, 16) || misaligned(scratch, 16) ||
               misaligned(p->tree_dev, 4)) {
      why = "q, out and scratch must be 16-byte aligned, tree 4-byte";
    } else if (batch->rows > 1 && (p->ldq < row || p->ldo < row || p->ldq % 8 != 0 || p->ldo % 8 != 0 ||
                                   std::max(p->ldq, p->ldo) > INT64_C(1) << 40)) {
      why = "row strides must be multiples of 8 that cover a row, at most 2^40";
    } else if (p->q_dev == p->out_dev) {
      why = "out must not be q";
    } else if (scratch_bytes < l.total) {
      why = "scratch too small";
    }
  }
  if (why != nullptr) {
    set_op_error(why);
    return MEMSPEC_ERR_INVALID_ARG;
  }
  char* const mem = static_cast<char*>(scratch);
  const bool two = p->prefix != nullptr && p->prefix_len > 0;
  ListArgs a{};
  a.kv[0] = kv_view(kv);
  if (two) a.kv[1] = kv_view(p->prefix);
  a.starts = batch->starts_dev;
  a.lens = batch->lens_dev;
  a.rows = batch->rows;
  a.q = static_cast<const bf16*>(p->q_dev);
  a.ldq = batch->rows > 1 ? p->ldq : 0;
  a.scale = p->scale * 1.4426950408889634f;
  a.group = p->n_heads / kv->n_heads;
  a.kv_heads = kv->n_heads;
  a.group_magic = a.group == 1 ? 0u : static_cast<uint32_t>(((uint64_t{1} << 32) + a.group - 1) / a.group);
  a.ldo = batch->rows > 1 ? p->ldo : 0;
  JoinArgs j{};
  j.starts = batch->starts_dev;
  j.lens = batch->lens_dev;
  j.n_seq = batch->n_seq;
  j.rows = batch->rows;
  j.max_pos = kv->max_pos;
  j.group = a.group;
  j.group_magic = a.group_magic;
  j.kv_heads = kv->n_heads;
  j.out = static_cast<bf16*>(p->out_dev);
  j.ldo = a.ldo;
  cudaLaunchConfig_t cfg = {};
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cudaError_t e = cudaSuccess;
  for (int i = 0; i < l.n && e == cudaSuccess; ++i) {
    const Launch& x = l.launch[i];
    a.n_own = x.own ? batch->n_seq : 0;
    a.beside = i > 0;
    a.prefix_len = x.prefix ? p->prefix_len : 0;
    a.tree = x.own ? p->tree_dev : nullptr;
    const bool direct = !two && !x.tiles;
    a.out = direct ? j.out : nullptr;
    for (int k = 0; k < 2; ++k) a.full[k] = direct ? nullptr : reinterpret_cast<float*>(mem + l.full[k]);
    a.slots = reinterpret_cast<float*>(mem + x.slots);
    a.bases = reinterpret_cast<uint32_t*>(mem + x.bases);
    for (int k = 0; k < 2; ++k)
      if (k == 0 ? x.own : x.prefix)
        j.part[j.parts++] = {a.bases, a.slots, a.full[k], x.ctas(), a.n_own + (x.prefix ? 1 : 0), k == 0 ? -1 : a.n_own,
                             p->prefix_len, x.unit(), x.tiles ? 1 : 0};
    e = x.tiles ? launch_attn_tiles(kv->head_dim, x.codes, a, cfg)
                : launch_attn_rows(kv->head_dim, x.codes, x.nt, a, cfg);
  }
  if (e == cudaSuccess) {
    cfg.blockDim = dim3(kThreads);
    if (l.launch[0].tiles || l.launch[l.n - 1].tiles) {
      constexpr int at_once = 4 * kWarps;   // elements
      cfg.gridDim = dim3((batch->rows * a.group + 31) / 32, kv->n_heads, (kv->head_dim + at_once - 1) / at_once);
      e = kv->head_dim == 64 ? cudaLaunchKernelEx(&cfg, join_tiles_kernel<64>, j)
                             : cudaLaunchKernelEx(&cfg, join_tiles_kernel<128>, j);
    } else {
      cfg.gridDim = dim3(batch->rows, (p->n_heads + kWarps - 1) / kWarps);
      e = kv->head_dim == 64 ? cudaLaunchKernelEx(&cfg, join_rows_kernel<64>, j)
                             : cudaLaunchKernelEx(&cfg, join_rows_kernel<128>, j);
    }
  }
  if (e != cudaSuccess) {
    set_op_error(std::string("attention launch: ") + cudaGetErrorString(e));
    return MEMSPEC_ERR_CUDA;
  }
  return MEMSPEC_OK;
}

}  // extern "C"
