// attn_plan.cuh - what the attention kernels over a caller's cache (attn_rows.cu, attn_tiles.cu)
// and the launch that joins their sums (attn_join.cu) share: how a call's work is cut up.
//
// The list of a launch: the batch's sequences, then the prefix as one more, whose rows are the
// call's.  A unit is up to kUnit query vectors (rows x heads of a group) of one head of k and v;
// its keys are tiles of kTile.  All tiles of all units, by sequence, head, unit and key, stand on
// one line, each as long as it costs, and the CTAs take equal pieces of the line: what a piece
// holds follows from the lengths alone, which the device has and the host has not.  Units that end
// up in several CTAs leave a record of sums per CTA.
#pragma once
#include <cuda_fp16.h>

#include <cfloat>

#include "kv.cuh"

namespace memspec {

constexpr int kTile = 128;             // keys
constexpr float kStart = -FLT_MAX;     // the maximum of nothing
// Scores are kept in units of log2.  The maximum that weights are taken against is set kBelow under the largest score,
// and again only when a score passes it by more than kAbove, so that sums are rarely rescaled.  Codes: weights are fp16,
// which 2^6 keeps clear of the type's small end (it holds up to 2^15).  bf16: at most 2^-14, so that 2^14 of them
// times the largest values of bf16 stay within fp32.
template <bool CODES>
struct Weights {
  static constexpr float kAbove = CODES ? 14.f : -14.f, kBelow = CODES ? 6.f : -28.f;
};

struct ListArgs {
  KvView kv[2];              // the cache, the prefix
  const int *starts, *lens;
  int n_own;                 // sequences in the list (0: the prefix alone)
  int rows, prefix_len;      // (0: no prefix in the list)
  const bf16* q;
  long long ldq;
  const int* tree;
  float scale;               // log2(e) * the call's
  int group, kv_heads;
  uint32_t group_magic;      // ceil(2^32 / group), 0 for 1
  bf16* out;                 // where the sums of a unit within one CTA go, or nullptr: to `full`
  long long ldo;
  float* full[2];            // records of the cache's and of the prefix's units: [rows][heads], of attn_tiles.cu two such
  float* slots;              // [ctas][2] units' records
  uint32_t* bases;           // [list + 1]: where each sequence's tiles begin on the line
  int beside;                // the launch before this one is the same call's: what that one waited for is complete
};

// A record: HD sums, the maximum, the sum of weights (and two floats that align the next one).
template <int HD>
constexpr int kRecord = HD + 4;

__device__ __forceinline__ int list_len(const ListArgs& a) { return a.n_own + (a.prefix_len > 0 ? 1 : 0); }
__device__ __forceinline__ SeqRows list_rows(const ListArgs& a, int b) {
  if (b < a.n_own) return seq_rows(a.starts, a.lens, b, a.rows);
  return {0, a.rows, a.prefix_len};
}
__device__ __forceinline__ int list_keys(const ListArgs& a, int b, const SeqRows& s) {
  return b < a.n_own ? min(max(s.len, 0), a.kv[0].max_pos) : a.prefix_len;
}
// At least one, so that every row of a sequence is written.
__host__ __device__ constexpr uint32_t tiles_of(int keys) { return keys == 0 ? 1 : (keys + kTile - 1u) / kTile; }

// What a unit of up to UNIT vectors takes of the line: START to begin with, then TILE a tile; START2 and TILE2 (if not 0)
// where it has more than 128 vectors.  A tile is whose its beginning is; a CTA whose piece ends within a start has
// nothing of that unit, and who goes on in it does so as with its first: no CTA has more than its piece.
template <int UNIT, int TILE, int START, int TILE2, int START2>
struct Cut {
  static constexpr int kUnit = UNIT, kGrain = TILE2 > TILE ? TILE2 : TILE;
  __host__ __device__ static bool pair(uint32_t vecs, uint32_t unit) { return TILE2 > 0 && vecs - unit * UNIT > 128; }
  __host__ __device__ static uint32_t place_of(uint32_t t, bool pair) { return pair ? START2 + t * TILE2 : START + t * TILE; }
  __host__ __device__ static uint32_t per_unit(uint32_t tiles) { return place_of(tiles, TILE2 > 0); }
  // all units of a head together: one of them, but for the last one
  __host__ __device__ static uint32_t per_head(uint32_t vecs, uint32_t tiles) {
    const uint32_t units = (vecs + UNIT - 1) / UNIT;
    return units == 0 ? 0 : (units - 1) * per_unit(tiles) + place_of(tiles, pair(vecs, units - 1));
  }
  // the first tile at or after place `at`
  __device__ static uint32_t tile_from(uint32_t at, bool pair) {
    const uint32_t start = pair ? START2 : START, in = at < start ? 0 : at - start;
    return pair ? (in + TILE2 - 1) / (TILE2 > 0 ? TILE2 : 1) : (in + TILE - 1) / TILE;
  }
};

// Equal pieces of the line: the first total % ctas are one longer.  None is shorter than a tile: what lies within a
// unit, past its start, has one of it.
struct Pieces {
  uint32_t ctas, each, longer;
  __device__ Pieces(uint32_t ctas_, uint32_t total, int grain) {
    ctas = max(min(ctas_, total / grain), 1u);
    each = total / ctas;
    longer = total - each * ctas;
  }
  __device__ uint32_t begin(uint32_t c) const {
    c = min(c, ctas);
    return c * each + min(c, longer);
  }
  __device__ uint32_t owner(uint32_t x) const {
    const uint32_t at = longer * (each + 1);
    return min(x < at ? x / (each + 1) : longer + (x - at) / max(each, 1u), ctas - 1);
  }
};

// The list in shared memory: where each sequence begins on the line, and for the first ones their rows.
constexpr int kCached = 64;
struct alignas(128) Plan {   // what lies behind it stays on 128-byte lines (else 335 us for 275 at 64 long sequences)
  uint32_t bases[kMaxSeqs + 2];
  uint64_t sums[20];
  SeqRows rows[kCached];
};

// Made by all THREADS threads.  Sequences whose rows overlap (starts that do not ascend) can make the line longer
// than 32 bits count: it ends there, the rest is not worked on.
constexpr uint64_t kLineEnd = 0xf0000000u;
template <class CUT, int THREADS>
__device__ __forceinline__ void make_plan(const ListArgs& a, Plan& plan) {
  static_assert(THREADS <= 640, "a word of sums per warp");
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32, n = list_len(a);
  uint64_t before = 0;
#pragma unroll 1
  for (int b0 = 0; b0 < n; b0 += THREADS) {
    const int b = b0 + tid;
    uint64_t mine = 0;
    if (b < n) {
      const SeqRows s = list_rows(a, b);
      if (b < kCached) plan.rows[b] = s;
      mine = CUT::per_head(static_cast<uint32_t>(s.n) * a.group, tiles_of(list_keys(a, b, s))) * a.kv_heads;
    }
    uint64_t incl = mine;
#pragma unroll 1
    for (int o = 1; o < 32; o *= 2) {
      const uint64_t up = __shfl_up_sync(~0u, incl, o);
      if (lane >= o) incl += up;
    }
    if (lane == 31) plan.sums[warp] = incl;
    __syncthreads();
    uint64_t sum = before;
    const int warps = (min(n - b0, THREADS) + 31) / 32;   // those with a sequence
#pragma unroll 1
    for (int w = 0; w < warps; ++w) {
      if (w < warp) sum += plan.sums[w];
      before += plan.sums[w];
    }
    if (b < n) plan.bases[b] = static_cast<uint32_t>(min(sum + incl - mine, kLineEnd));
    if (b == n - 1) plan.bases[n] = static_cast<uint32_t>(min(sum + incl, kLineEnd));
    __syncthreads();
  }
}

// A CTA's stretch of one unit.
struct alignas(16) Stretch {
  int b, head, unit, t0, t1;   // key tiles [t0, t1)
  int tiles, row0, vecs;       // of the unit; vecs: of the sequence and head
  int keys;                    // that the unit sees
  long long first;             // the slot of the sequence's first row; the prefix's: past its end
  int own;                     // not the prefix
  __device__ bool whole() const { return t0 == 0 && t1 == tiles; }
  __device__ int end() const { return min(static_cast<long long>(keys), static_cast<long long>(t1) * kTile); }
};
// The stretches of this CTA, one after another.
template <class CUT>
struct Walk {
  const ListArgs& a;
  const Plan& plan;
  uint32_t x, x1;
  int b;
  __device__ Walk(const ListArgs& a_, const Plan& plan_) : a(a_), plan(plan_) {
    const int n = list_len(a);
    const Pieces pieces(gridDim.x, plan.bases[n], CUT::kGrain);
    x = pieces.begin(blockIdx.x);
    x1 = pieces.begin(blockIdx.x + 1);
    int lo = 0, hi = n;   // the last one that begins at or before x
#pragma unroll 1
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (plan.bases[mid] <= x)
        lo = mid;
      else
        hi = mid;
    }
    b = lo;
  }
  __device__ bool next(Stretch& u) {
    bool found = false;
#pragma unroll 1
    while (!found && x < x1) {
#pragma unroll 1
      while (plan.bases[b + 1] <= x) ++b;
      const SeqRows s = b < kCached ? plan.rows[b] : list_rows(a, b);
      u.b = b;
      u.own = b < a.n_own;
      u.row0 = s.row0;
      u.vecs = s.n * a.group;
      u.keys = list_keys(a, b, s);
      u.first = u.own ? static_cast<long long>(s.len) - s.n : u.keys;
      u.tiles = tiles_of(u.keys);
      const uint32_t per_head = CUT::per_head(u.vecs, u.tiles), in = x - plan.bases[b], per_unit = CUT::per_unit(u.tiles);
      u.head = in / per_head;
      const uint32_t in_head = in - u.head * per_head;
      u.unit = in_head / per_unit;
      const bool pair = CUT::pair(u.vecs, u.unit);
      const uint32_t at = in_head - u.unit * per_unit, end = min(CUT::place_of(u.tiles, pair), at + (x1 - x));
      u.t0 = min(CUT::tile_from(at, pair), static_cast<uint32_t>(u.tiles));
      u.t1 = min(CUT::tile_from(end, pair), static_cast<uint32_t>(u.tiles));
      x += end - at;
      found = u.t0 < u.t1;   // (pieces that lie within a unit's start, or a tile, have nothing of it)
    }
    return found;
  }
};

// The row and the head, of the group, of a sequence's vector.
__device__ __forceinline__ int vector_row(const ListArgs& a, int vec) {
  return a.group_magic == 0 ? vec : static_cast<int>(__umulhi(vec, a.group_magic));
}

// What a vector sees of its sequence's slots.
struct Sight {
  int limit;        // those up to this one
  uint32_t bits;    // and of the rows' own, bit by bit
};
__device__ __forceinline__ Sight sight_of(const ListArgs& a, const Stretch& u, int vec) {
  Sight s{0x7fffffff, 0u};
  if (u.own && vec < u.vecs) {
    const int j = vector_row(a, vec);
    s.limit = static_cast<int>(max(u.first + (a.tree != nullptr ? -1 : j), -1ll));
    if (a.tree != nullptr) s.bits = static_cast<uint32_t>(a.tree[u.row0 + j]);
  }
  return s;
}
__device__ __forceinline__ bool sees(const Sight& s, long long first, int key) {
  if (key <= s.limit) return true;
  const long long d = key - first;
  return d >= 0 && d < 32 && (s.bits >> d & 1);
}

// The launch that joins records: one part for the sequences' own keys, one for the prefix's.
struct JoinPart {
  const uint32_t* bases;
  const float *slots, *full;   // full == nullptr: units within one CTA are written already
  int ctas, list, at;          // the launch's; `at`: the prefix's place in its list, or -1: the row's sequence
  int keys;                    // of the prefix
  int unit;                    // vectors of a unit
  int pairs;                   // attn_tiles.cu's records
};
struct JoinArgs {
  JoinPart part[2];
  int parts;
  const int *starts, *lens;
  int n_seq, rows, max_pos, group, kv_heads;
  uint32_t group_magic;
  bf16* out;
  long long ldo;
};

// Small loads, copies and conversions that both kernels use.
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Two codes (bytes i and j of w, as code + 128) as fp16: 0x64 in front makes 1024 + 128 + code
template <int SEL>
__device__ __forceinline__ uint32_t codes_f16(uint32_t w) {
  const uint32_t u = __byte_perm(w, 0x64646464u, SEL);
  const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&u), __half2half2(__ushort_as_half(0x6480)));
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Query vectors as fp16, for the products with codes: each times the power of two that brings its largest value
// near 2^10, where fp16 holds all bits of bf16 (what falls off is below 2^-34 of the vector's largest; of one below 2^-110,
// which is left smaller, below 2^-144).
// Here of the vector of which each of LANES neighbours has eight values; the whole warp calls it.
template <int LANES>
__device__ __forceinline__ int exponent_of_lanes(const uint4& x) {
  auto of = [](uint32_t pair) {
    pair &= 0x7fff7fffu;
    return *reinterpret_cast<const __nv_bfloat162*>(&pair);
  };
  __nv_bfloat162 top = __hmax2(__hmax2(of(x.x), of(x.y)), __hmax2(of(x.z), of(x.w)));
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) top = __hmax2(top, __shfl_xor_sync(~0u, top, o));
  const uint32_t bits = *reinterpret_cast<const uint32_t*>(&top);
  return max(static_cast<int>(max(bits & 0xffffu, bits >> 16) >> 7) - 127, -110) - 10;
}
__device__ __forceinline__ float power(int e) { return __int_as_float((e + 127) << 23); }
__device__ __forceinline__ uint32_t scaled_f16(uint32_t pair, float by) {
  return pack_f16(__uint_as_float(pair << 16) * by, __uint_as_float(pair & 0xffff0000u) * by);
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool on) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src, bool on) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(on ? 4 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Launches (attn_rows.cu, attn_tiles.cu): `slots` holds two units' records for each CTA, of the unit's 8 nt or 256 vectors
// (attn_tiles.cu's smaller units: two copies of 128) by HD + 4 floats.
int rows_ctas(bool codes);
cudaError_t launch_attn_rows(int hd, bool codes, int nt, const ListArgs& a, cudaLaunchConfig_t cfg);
constexpr int kTilesCtas = 152;
cudaError_t launch_attn_tiles(int hd, bool codes, const ListArgs& a, cudaLaunchConfig_t cfg);   // InvalidValue: no tensor map
// In attn_tiles.cu a tile of up to 128 vectors takes 1.1 us (codes 1.5), of more 1.9 (2.4); a further stretch in a CTA 2.6
// us, where it is cut as well 5 (2.4, 4.2), of more vectors 5.3 (7.5).  One set of weights serves both types: 256 rows over
// 4355 positions, 16 x 9 rows behind 8192, 16 x 9 rows over codes, caches cold, 35.0, 40.0, 41.9 us; tiles of 1 and 2 with starts of
// 3 and 5: 36.1, 40.1, 41.7; starts of 2 and 4: 36.4, 44.1, 41.5.  In attn_rows.cu a tile takes 0.5 us; with a start of 2 of
// them one row of 32 heads over 2048 takes 12.9 us (0: 14.1, 4: 12.8), 5 rows over codes 13.4 (15.0, 13.1), 16 rows over codes 20.9
// (21.5, 21.9).
typedef Cut<256, 3, 8, 5, 16> TileUnits;
template <int VT>
using RowUnits = Cut<VT, 1, 2, 0, 0>;

}  // namespace memspec
