// lora.cu - low-rank adapters of many requests beside a shared projection
// (memspec_op_lora): y[r] = base[r] + scale[a] * B[a] (A[a] x[r]), a = ids[r].
//
// Rows of one adapter are taken together: a chunk is up to 16 MT rows of one adapter (or
// of none) in row order; every CTA finds its chunk from the ids itself, so no launch and no
// host knowledge of the ids is needed for that.  Both products run on mma.sync
// (m16n8k16, bf16 in, fp32 out) with a chunk's rows as M: the work is bounded by reading A
// and B and by reading and writing y, one or a few rows at a time fill no tcgen05 tile, and
// fragments come straight from memory (the contraction index is permuted so that a thread's
// fragments of two steps are 16 consecutive bytes).
// Two launches, or for short calls one that does the work of both (fused_kernel):
//   1. shrink: t = A x.  A cluster of 8 CTAs splits k, the 8 warps of a CTA split its part;
//      the sums are added warp by warp, then pushed into the CTA of the cluster that owns
//      the element and added rank by rank: one order, one t.
//   2. expand: y = base + scale B t.  t enters as three bf16 planes, which hold all its 24
//      bits.  The columns of n = 8 tiles are dealt so that a thread's results are float4s of a
//      row.  B, the base and the ids are read while the shrink
//      launch still runs (everything before it has completed when this one starts).
//
// Measured (us in a graph, inputs from memory; floor: every operand moved once at 6780 GB/s):
// 1 row, 4096 x 4096, rank 16: 4.8 (floor 0.04; a call is 12 to 16, the host's); 16 rows of 16
// adapters: 5.9 (0.54); 144 rows of 16 adapters, n 28672, k 4096, ranks up to 64: 26.2 (9.95;
// 20.6 with the operands in L2): 8 us until t is there, then 18 for 77 MB, the first CTAs done
// after 9; 256 rows of one adapter, n 4096, k 14336, rank 128: 18.4 (3.0), two to
// find the chunk, five for 58 MB through L2 in groups of 32 ranks and rows, two for the sums'
// exchange, four to five in the expansion, the rest launches; 21 rows, n 32003: 10.6
// (1.95), a base and a y without alignment moved 4 bytes at a time.
//
// Products are exact and every sum is fp32, but the tensor cores' additions may truncate, where
// separate ones round: over long k and many ranks the result is up to some twice as far from 64 bits
// as sums in 32 bits are (256 rows, k 14336, rank 128: 4.7e-7 of its norm, 2.9e-7; 144 rows, k 4096,
// rank 64: 0.9e-7, 2.0e-7; one row, rank 16: 0.5e-7, 0.6e-7).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <string>

#include "../../include/memspec_ops.h"
#include "internal.h"
#include "ptx.cuh"

namespace memspec {
namespace {

constexpr int kMaxLoraRows = 256;
constexpr int kMaxRank = 128;
constexpr int kThreads = 256;       // one per row where the ids are searched
constexpr int kWarps = kThreads / 32;
constexpr int kSplits = 8;          // CTAs over k: a portable cluster

struct LoraArgs {
  const bf16* x;
  long long ldx;
  const bf16* a;            // [n_adapters][rank][k]
  const bf16* b;            // [n_adapters][n][rank]
  const float* scales;      // [n_adapters] or nullptr (1)
  const int* ranks;         // [n_adapters] or nullptr (rank)
  const int* ids;           // [rows]
  const float* base;        // [rows] at ld_base, or nullptr (0)
  long long ld_base;
  float* y;
  long long ldy;
  int rows, n, k, n_adapters, rank;
  float* t;                 // [rows][rank]
  int vec;                  // 1: base and y take 16-byte accesses at every fourth column
};

// D += A B, 16 x 8 x 16.
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The call's chunks: up to CH rows of one adapter each, numbered by their first row.
template <int CH>
struct Chunks {
  int2 table[kWarps][32];   // a warp's distinct ids (-1: none) and how many rows have each
  int distinct[kWarps];
  int leaders[kWarps];
  int row[CH];              // the selected chunk's rows, ascending; -1 past the last
  int id, first, rank;      // rank 0: no adapter, or an empty one
  float scale;
};
// What a thread knows of row threadIdx.x.
struct RowPlace {
  int id;                   // -1: no adapter
  int rank;                 // of its adapter (0: none), and its scale: loaded while rows are counted
  float scale;
  int pos;                  // rows of the same adapter before it
  int chunk;                // the chunk that it leads, or -1
};
// All threads; returns the number of chunks.  Rows of one adapter mostly stand together, so
// a warp's 32 rows have few distinct ids and the counts of earlier warps are a short list
// (comparing each row with all earlier ones took 1 us more of a launch over 144 rows).
template <int CH>
__device__ int find_chunks(const LoraArgs& a, Chunks<CH>& s, RowPlace& p) {
  const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31;
  const unsigned below = (1u << lane) - 1;
  p.id = -2;
  if (tid < a.rows) {
    p.id = __ldcg(a.ids + tid);
    if (p.id < 0 || p.id >= a.n_adapters) p.id = -1;
  }
  p.pos = 0;
  if (w * 32 < a.rows) {
    const unsigned same = __match_any_sync(0xffffffffu, p.id);
    p.pos = __popc(same & below);
    const unsigned firsts = __ballot_sync(0xffffffffu, p.pos == 0);
    if (p.pos == 0) s.table[w][__popc(firsts & below)] = make_int2(p.id, __popc(same));
    if (lane == 0) s.distinct[w] = __popc(firsts);
  }
  __syncthreads();
  bool leads = false;
  if (w * 32 < a.rows) {
    for (int v = 0; v < w; ++v)
      for (int e = 0, n = s.distinct[v]; e < n; ++e) {
        const int2 q = s.table[v][e];
        p.pos += q.x == p.id ? q.y : 0;
      }
    leads = tid < a.rows && p.pos % CH == 0;
  }
  if (leads) {
    p.rank = p.id < 0 ? 0 : a.ranks == nullptr ? a.rank : __ldcg(a.ranks + p.id);
    p.scale = p.id < 0 || a.scales == nullptr ? 1.f : __ldcg(a.scales + p.id);
  }
  const unsigned mask = __ballot_sync(0xffffffffu, leads);
  if (lane == 0) s.leaders[w] = __popc(mask);
  __syncthreads();
  int before = __popc(mask & below), all = 0;
#pragma unroll
  for (int v = 0; v < kWarps; ++v) {
    if (v < w) before += s.leaders[v];
    all += s.leaders[v];
  }
  p.chunk = leads ? before : -1;
  return all;
}
// All threads: chunk c's id and rows.
template <int CH>
__device__ void select_chunk(const LoraArgs& a, const RowPlace& p, int c, Chunks<CH>& s) {
  const int tid = threadIdx.x;
  __syncthreads();
  if (tid < CH) s.row[tid] = -1;
  if (p.chunk == c) {
    s.id = p.id;
    s.first = p.pos;
    s.rank = max(0, min(p.rank, a.rank));
    s.scale = p.scale;
  }
  __syncthreads();
  if (tid < a.rows && p.id == s.id && p.pos >= s.first && p.pos < s.first + CH) s.row[p.pos - s.first] = tid;
  __syncthreads();
}

// ------------------------------------------------ t = A x
__device__ __forceinline__ void add4(float4& s, const float4& v) {
  s.x += v.x;
  s.y += v.y;
  s.z += v.z;
  s.w += v.w;
}
// This warp's sums over its part of CTA `split`'s columns: ranks j0 .. j0 + 8 NT - 1 (below
// `rank`) of adapter id and up to 16 MT rows (row[]: -1 for none), `tiles` 16-row tiles of them.
template <int MT, int NT>
__device__ __forceinline__ void shrink_sums(const LoraArgs& a, const int* row, int id, int rank, int j0, int split,
                                            int tiles, float (&acc)[MT][NT][4]) {
  const int w = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const bf16* xr[MT][2];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = row[m * 16 + h * 8 + g];
      xr[m][h] = r < 0 ? nullptr : a.x + r * a.ldx + 8 * t;
    }
  const bf16* ar[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int j = j0 + n * 8 + g;
    ar[n] = j < rank ? a.a + (static_cast<long long>(id) * a.rank + j) * a.k + 8 * t : nullptr;
  }
  const int blocks = (a.k + 31) / 32;         // of 32 columns
  const int end = static_cast<int>(static_cast<long long>(split + 1) * blocks / kSplits);
  const uint4 zero = make_uint4(0, 0, 0, 0);
  constexpr int kAhead = MT * 2 + NT <= 4 ? 4 : MT * 2 + NT <= 8 ? 2 : 1;   // blocks loaded together
  for (int b0 = static_cast<int>(static_cast<long long>(split) * blocks / kSplits) + w; b0 < end;
       b0 += kWarps * kAhead) {
    uint4 xv[kAhead][MT][2], av[kAhead][NT];
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      const int k0 = (b0 + q * kWarps) * 32;
      const bool in = b0 + q * kWarps < end && k0 + 8 * t < a.k;
#pragma unroll
      for (int n = 0; n < NT; ++n)
        av[q][n] = in && ar[n] != nullptr ? __ldcg(reinterpret_cast<const uint4*>(ar[n] + k0)) : zero;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          xv[q][m][h] =
              in && xr[m][h] != nullptr ? __ldcg(reinterpret_cast<const uint4*>(xr[m][h] + k0)) : zero;
    }
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        if (m >= tiles) break;
        const uint32_t a0[4] = {xv[q][m][0].x, xv[q][m][1].x, xv[q][m][0].y, xv[q][m][1].y};
        const uint32_t a1[4] = {xv[q][m][0].z, xv[q][m][1].z, xv[q][m][0].w, xv[q][m][1].w};
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          mma(acc[m][n], a0, av[q][n].x, av[q][n].y);
          mma(acc[m][n], a1, av[q][n].z, av[q][n].w);
        }
      }
    }
  }
}
// The warps' sums added up and pushed to the CTA of the cluster that owns the element: from
// there split[c] (`own` lanes' sums) of every CTA c are complete after the next cluster
// barrier.  All threads; the cluster's first barrier has been arrived at.
template <int MT, int NT>
__device__ __forceinline__ void share_sums(const float (&acc)[MT][NT][4], int tiles, int split, int own,
                                           float4 (*warp)[MT * NT * 32], float4 (*to)[MT * NT * 32 / kSplits]) {
  const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31;
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    if (m >= tiles) break;
#pragma unroll
    for (int n = 0; n < NT; ++n)
      warp[w][(m * NT + n) * 32 + lane] = make_float4(acc[m][n][0], acc[m][n][1], acc[m][n][2], acc[m][n][3]);
  }
  __syncthreads();
  cluster_wait_acquire();
  for (int f = tid; f < own * kSplits; f += kThreads) {
    float4 s = warp[0][f];
#pragma unroll
    for (int i = 1; i < kWarps; ++i) add4(s, warp[i][f]);
    const int owner = f / own;
    st_cluster_f4(mapa_shared(smem_addr(&to[split][f - owner * own]), owner), s);
  }
}

// t[row][j] for a chunk of up to 16 MT rows and 8 NT of the adapter's ranks.  Grid (cluster
// of kSplits over k, groups of 8 NT ranks, chunks): CTAs past the last chunk, which the host does
// not know, come last.
template <int MT, int NT>
struct ShrinkSmem {
  static constexpr int kFrags = MT * NT * 32;   // a lane's four sums of a 16 x 8 tile
  Chunks<MT * 16> chunk;
  float4 warp[kWarps][kFrags];                  // a warp's sums
  float4 split[kSplits][kFrags / kSplits];      // this CTA's sums, from each CTA of the cluster
};

template <int MT, int NT>
__global__ void __launch_bounds__(kThreads, 2) shrink_kernel(const __grid_constant__ LoraArgs a) {
  extern __shared__ __align__(16) uint8_t raw[];
  typedef ShrinkSmem<MT, NT> S;
  S& sm = *reinterpret_cast<S*>(raw);
  const int tid = threadIdx.x, split = blockIdx.x, j0 = blockIdx.y * NT * 8;
  cluster_arrive_release();   // waited for before the first push into a peer
  pdl_wait();
  pdl_launch_dependents();
  // the CTAs of a cluster have one chunk and one rank group: they leave together
  RowPlace place;
  const bool found = static_cast<int>(blockIdx.z) < find_chunks(a, sm.chunk, place);
  if (found) select_chunk(a, place, blockIdx.z, sm.chunk);
  const int rank = found ? sm.chunk.rank : 0;
  if (j0 >= rank) {
    cluster_wait_acquire();
    return;
  }
  int tiles = 0;              // 16-row tiles with rows
#pragma unroll
  for (int m = 0; m < MT; ++m) tiles += sm.chunk.row[m * 16] >= 0;
  float acc[MT][NT][4] = {};
  shrink_sums<MT, NT>(a, sm.chunk.row, sm.chunk.id, rank, j0, split, tiles, acc);
  const int own = tiles * NT * 32 / kSplits;
  share_sums<MT, NT>(acc, tiles, split, own, sm.warp, sm.split);
  cluster_arrive_release();
  cluster_wait_acquire();
  for (int i = tid; i < own; i += kThreads) {
    float4 s = sm.split[0][i];
#pragma unroll
    for (int c = 1; c < kSplits; ++c) add4(s, sm.split[c][i]);
    const int f = split * own + i, l = f & 31, n = (f >> 5) % NT, m = (f >> 5) / NT;
    const int j = j0 + n * 8 + 2 * (l & 3);
    const int r0 = sm.chunk.row[m * 16 + (l >> 2)], r1 = sm.chunk.row[m * 16 + 8 + (l >> 2)];
    if (j >= a.rank) continue;
    if (r0 >= 0) *reinterpret_cast<float2*>(a.t + r0 * a.rank + j) = make_float2(s.x, s.y);
    if (r1 >= 0) *reinterpret_cast<float2*>(a.t + r1 * a.rank + j) = make_float2(s.z, s.w);
  }
}

// ------------------------------------------------ y = base + scale B t

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float bf16_part(float x) { return __bfloat162float(__float2bfloat16_rn(x)); }
// A pair of bf16 at ranks r, r + 1 without what lies past the adapter's rank (which may be
// anything).
__device__ __forceinline__ uint32_t within(uint32_t pair, int r, int rank) {
  return r + 1 < rank ? pair : (r < rank ? pair & 0xffffu : 0u);
}
__device__ __forceinline__ void copy16_async(void* dst, const void* src, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_addr(dst)), "l"(src), "r"(in ? 16 : 0)
               : "memory");
}

// KT: steps of 16 ranks.  B's columns arrive by cp.async kStages items ahead (loads into
// registers as they were needed left a warp waiting half the time: gate/up of 144 rows 30 us).
template <int KT>
struct Ring {
  // of an item, what a warp takes at a time; 16 leave room for CTAs of the launch before (256
  // rows, n 4096, k 14336, rank 128: 18.4 us, 21.4 with 32 columns and one CTA per SM)
  static constexpr int kCols = KT <= 4 ? 32 : 16;
  static constexpr int kPieces = KT * 2;           // of 8 ranks, per column
  static constexpr int kStages = KT <= 2 ? 4 : KT == 4 ? 3 : 2;
  uint4 b[kStages][kCols * kPieces];
};
typedef float4 Turn[16][8 + 1];     // a warp's tile where rows are not 16-byte aligned
// The fragments of t's three planes of up to MT 16-row tiles, a uint4 per lane.
template <int KT, int MT>
struct Planes {
  uint4 v[MT][KT][3][32];
};

// One warp's items lo + w, lo + w + 8, ... below hi of a chunk.
template <int KT, int MT>
struct ExpandWarp {
  static constexpr int kCols = Ring<KT>::kCols, kTiles = kCols / 8, kQuads = kCols / 16;
  static constexpr int kRows = kCols / 2;   // of a tile, that a lane has where rows fit no 16-byte access
  static constexpr int kPieces = Ring<KT>::kPieces, kStages = Ring<KT>::kStages;
  const LoraArgs& a;
  Ring<KT>& ring;
  Turn& turn;
  const int* row;
  int rank, tiles, lo, mine;
  float scale;
  const bf16* bp;
  // of what is stored next: rows g, g + 8 of kQuads float4s, or a column of kRows rows (loaded as they
  // were stored, four rows at a time, 81 us for 40 at 144 x 32003)
  float base[kRows];

  template <int CH>
  __device__ ExpandWarp(const LoraArgs& args, Ring<KT>& r, Turn& t, const Chunks<CH>& c, int from, int to)
      : a(args), ring(r), turn(t), row(c.row), rank(c.rank), tiles(0), scale(c.scale) {
    static_assert(CH == MT * 16, "the chunk's rows");
    const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
    for (int m = 0; m < MT; ++m) tiles += row[m * 16] >= 0;
    lo = from + w;
    mine = to > lo ? (to - lo + kWarps - 1) / kWarps : 0;
    bp = a.b + (static_cast<long long>(max(c.id, 0)) * a.n + lane / kPieces) * a.rank + lane % kPieces * 8;
  }
  // a thread's 8 ranks of 32 (KT = 1: 4 of 16) are split over two steps
  __device__ int steps() const { return KT == 1 ? (rank + 15) / 16 : (rank + 31) / 32 * 2; }
  __device__ int column(int item) const { return (lo + item * kWarps) * kCols; }

  // lane's piece of kPieces columns of an item: piece lane % kPieces, swapped by fours in odd
  // columns so that two columns' pieces lie in different banks
  __device__ void load_b(int item) {
    const int c0 = column(item), lane = threadIdx.x & 31, piece = lane % kPieces;
#pragma unroll
    for (int i = 0; i < kCols * kPieces / 32; ++i) {
      const int col = lane / kPieces + i * (32 / kPieces);
      const bool in = c0 + col < a.n && piece * 8 < rank;
      copy16_async(&ring.b[item % kStages][col * kPieces + (KT >= 4 ? piece ^ ((col & 1) << 2) : piece)],
                   in ? bp + static_cast<long long>(c0 + i * (32 / kPieces)) * a.rank : a.b, in);
    }
  }
  __device__ void load_base(int m, int c0) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    if (a.vec) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = row[m * 16 + h * 8 + g];
#pragma unroll
        for (int q = 0; q < kQuads; ++q) {
          const int x = c0 + 16 * q + 4 * t;
          const float4 v = r >= 0 && x < a.n && a.base != nullptr
                               ? __ldcg(reinterpret_cast<const float4*>(a.base + r * a.ld_base + x))
                               : make_float4(0.f, 0.f, 0.f, 0.f);
          float* const b = base + (h * kQuads + q) * 4;
          b[0] = v.x;
          b[1] = v.y;
          b[2] = v.z;
          b[3] = v.w;
        }
      }
    } else {
      const int x = c0 + lane % kCols;
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const int r = row[m * 16 + lane / kCols * kRows + i];
        base[i] = r >= 0 && a.base != nullptr && x < a.n ? __ldcg(a.base + r * a.ld_base + x) : 0.f;
      }
    }
  }
  // The first loads: they do not depend on t.
  __device__ void start() {
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) {
      if (i < mine && rank > 0) load_b(i);
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
    if (mine > 0) load_base(0, column(0));
  }
  __device__ void run(const Planes<KT, MT>& planes) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    // column of MMA column g of tile j: 16 (j / 2) + 4 (g / 2) + 2 (j % 2) + g % 2, so that a
    // thread's results of two tiles (their columns 2 t, 2 t + 1) are columns 4 t .. 4 t + 3 of
    // 16: four threads write 64 bytes of a row at once
    const int bcol = 4 * (g >> 1) + (g & 1), n_steps = steps();
    for (int i = 0; i < mine; ++i) {
      const int c0 = column(i);
      if (i + kStages - 1 < mine && rank > 0) load_b(i + kStages - 1);
      asm volatile("cp.async.commit_group;" ::: "memory");
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
      __syncwarp();
      for (int m = 0; m < tiles; ++m) {
        float acc[kTiles][4] = {};
#pragma unroll
        for (int s2 = 0; s2 < (KT + 1) / 2; ++s2) {
          if (2 * s2 >= n_steps) break;
          uint4 bv[kTiles];
#pragma unroll
          for (int j = 0; j < kTiles; ++j) {
            const int col = bcol + 16 * (j >> 1) + 2 * (j & 1);
            const uint4* p = &ring.b[i % kStages][col * kPieces];
            if (KT == 1) {
              const uint2 u = reinterpret_cast<const uint2*>(p)[t];
              bv[j] = make_uint4(u.x, u.y, 0u, 0u);
            } else {
              bv[j] = p[KT >= 4 ? (s2 * 4 + t) ^ ((col & 1) << 2) : s2 * 4 + t];
            }
            if (rank & 7) {
              const int r = KT == 1 ? 4 * t : (s2 * 4 + t) * 8;
              bv[j].x = within(bv[j].x, r, rank);
              bv[j].y = within(bv[j].y, r + 2, rank);
              bv[j].z = within(bv[j].z, r + 4, rank);
              bv[j].w = within(bv[j].w, r + 6, rank);
            }
          }
#pragma unroll
          for (int o = 0; o < (KT == 1 ? 1 : 2); ++o) {
#pragma unroll
            for (int p = 0; p < 3; ++p) {
              const uint4 f = planes.v[m][2 * s2 + o][p][lane];
              const uint32_t fa[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
              for (int j = 0; j < kTiles; ++j) mma(acc[j], fa, o ? bv[j].z : bv[j].x, o ? bv[j].w : bv[j].y);
            }
          }
        }
        if (a.vec)
          store(m, c0, acc);
        else
          store_turned(m, c0, acc);
        // the base of what this warp does next
        if (m + 1 < tiles)
          load_base(m + 1, c0);
        else if (i + 1 < mine)
          load_base(0, column(i + 1));
      }
      __syncwarp();   // the stage is read before it is filled again
    }
  }
  __device__ void store(int m, int c0, const float (&acc)[kTiles][4]) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = row[m * 16 + h * 8 + g];
#pragma unroll
      for (int q = 0; q < kQuads; ++q) {
        const int x = c0 + 16 * q + 4 * t;
        if (r < 0 || x >= a.n) continue;
        const float* const b = base + (h * kQuads + q) * 4;
        float4 o = make_float4(b[0], b[1], b[2], b[3]);
        if (rank > 0) {   // else the base's own bits
          o.x = fmaf(scale, acc[2 * q][2 * h], o.x);
          o.y = fmaf(scale, acc[2 * q][2 * h + 1], o.y);
          o.z = fmaf(scale, acc[2 * q + 1][2 * h], o.z);
          o.w = fmaf(scale, acc[2 * q + 1][2 * h + 1], o.w);
        }
        *reinterpret_cast<float4*>(a.y + r * a.ldy + x) = o;
      }
    }
  }
  // Through shared memory: a lane per column, 128 bytes of a row at once or 64 of two.
  __device__ void store_turned(int m, int c0, const float (&acc)[kTiles][4]) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    __syncwarp();
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int q = 0; q < kQuads; ++q)
        turn[h * 8 + g][4 * q + t] =
            make_float4(acc[2 * q][2 * h], acc[2 * q][2 * h + 1], acc[2 * q + 1][2 * h], acc[2 * q + 1][2 * h + 1]);
    __syncwarp();
    const int x = c0 + lane % kCols, i0 = lane / kCols * kRows;
    if (x >= a.n) return;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int r = row[m * 16 + i0 + i];
      if (r < 0) break;
      float o = base[i];
      if (rank > 0) o = fmaf(scale, reinterpret_cast<const float*>(&turn[i0 + i][0])[lane % kCols], o);
      a.y[r * a.ldy + x] = o;
    }
  }
};

// The second of two launches, as many CTAs as are resident at once.  Each has a part of one
// chunk's (up to 32 rows') items; where there are more chunks than CTAs, an even part of all
// (chunk, item) pairs in that order.  (Such parts for all calls: the CTAs with the end of one
// chunk and the start of the next finish last, 11.5 us for 10.8 at 21 x 32003.  Cut by their
// bytes: no faster, and a microsecond more to find a CTA's part.)
constexpr int kExpandTiles = 2;
template <int KT>
struct ExpandSmem {
  Ring<KT> ring[kWarps];
  Planes<KT, kExpandTiles> planes;
  Chunks<kExpandTiles * 16> chunk;
  Turn turn[kWarps];          // not there where rows are 16-byte aligned
  static constexpr size_t bytes(bool vec) { return vec ? sizeof(ExpandSmem) - sizeof(turn) : sizeof(ExpandSmem); }
  static constexpr int per_sm(bool vec) { return 2 * (bytes(vec) + 1024) <= 228 * 1024 ? 2 : 1; }
};

template <int KT>
__global__ void __launch_bounds__(kThreads, 2) expand_kernel(const __grid_constant__ LoraArgs a) {
  typedef ExpandSmem<KT> S;
  extern __shared__ __align__(16) uint8_t raw[];
  S& sm = *reinterpret_cast<S*>(raw);
  const int tid = threadIdx.x, w = tid >> 5;
  // the ids, B, base and scales may be read now: the launch before this one (shrink) lets
  // it start only after its own wait, so all that came earlier has completed
  RowPlace place;
  const int chunks = find_chunks(a, sm.chunk, place);
  const int cols = (a.n + Ring<KT>::kCols - 1) / Ring<KT>::kCols;
  const long long items = static_cast<long long>(chunks) * cols;
  const int ctas = gridDim.x, cta = blockIdx.x;
  long long at, end;
  if (chunks <= ctas) {       // CTAs [c ctas / chunks, (c + 1) ctas / chunks), rounded up, for chunk c
    const int c = cta * chunks / ctas, first = (c * ctas + chunks - 1) / chunks;
    const int of = ((c + 1) * ctas + chunks - 1) / chunks - first, part = cta - first;
    at = static_cast<long long>(c) * cols + static_cast<long long>(cols) * part / of;
    end = static_cast<long long>(c) * cols + static_cast<long long>(cols) * (part + 1) / of;
  } else {
    at = items * cta / ctas;
    end = items * (cta + 1) / ctas;
  }
  bool waited = false;
  while (at < end) {
    const int c = static_cast<int>(at / cols);
    const int lo = static_cast<int>(at - static_cast<long long>(c) * cols);
    const int hi = static_cast<int>(min(static_cast<long long>(cols), lo + (end - at)));
    at += hi - lo;
    select_chunk(a, place, c, sm.chunk);
    ExpandWarp<KT, kExpandTiles> e(a, sm.ring[w], sm.turn[w], sm.chunk, lo, hi);
    e.start();
    if (!waited) {
      pdl_wait();
      pdl_launch_dependents();
      waited = true;
    }
    const int steps = e.steps();
    for (int i = tid; i < e.tiles * steps * 32; i += kThreads) {
      const int l = i & 31, s = (i >> 5) % steps, m = (i >> 5) / steps;
      // the ranks of a lane's fragments of step s: as they lie in its pieces of B
      const int r = KT == 1 ? 4 * (l & 3) : (s >> 1) * 32 + 8 * (l & 3) + (s & 1) * 4;
      float v[2][4] = {};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int row = sm.chunk.row[m * 16 + h * 8 + (l >> 2)];
        if (row < 0 || r >= e.rank) continue;
        const float4 q = __ldcg(reinterpret_cast<const float4*>(a.t + row * a.rank + r));
        v[h][0] = q.x;
        v[h][1] = r + 1 < e.rank ? q.y : 0.f;
        v[h][2] = r + 2 < e.rank ? q.z : 0.f;
        v[h][3] = r + 3 < e.rank ? q.w : 0.f;
      }
#pragma unroll
      for (int p = 0; p < 3; ++p) {
        sm.planes.v[m][s][p][l] = make_uint4(pack_bf16(v[0][0], v[0][1]), pack_bf16(v[1][0], v[1][1]),
                                             pack_bf16(v[0][2], v[0][3]), pack_bf16(v[1][2], v[1][3]));
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int q = 0; q < 4; ++q) v[h][q] -= bf16_part(v[h][q]);
      }
    }
    __syncthreads();
    e.run(sm.planes);
  }
}

// ------------------------------------------------ both at once, for few rows
// A cluster of kSplits CTAs takes a chunk of up to 16 rows: they share the sums of t as the
// shrink launch does, each then sends its elements' planes to all, and takes an eighth of the
// columns - or, where n is long, of the grid's z-th part of them, for which t is computed again
// (A is in L2).  Its first columns of B and of the base are under way meanwhile.
template <int KT>
struct FusedSmem {
  static constexpr int NT = KT * 2, kFrags = NT * 32;
  Ring<KT> ring[kWarps];
  Planes<KT, 1> planes;
  float4 warp[kWarps][kFrags];
  float4 split[kSplits][kFrags / kSplits];
  Chunks<16> chunk;
  Turn turn[kWarps];
};

template <int KT>
__global__ void __launch_bounds__(kThreads, KT == 1 ? 2 : 1) fused_kernel(const __grid_constant__ LoraArgs a) {
  typedef FusedSmem<KT> S;
  constexpr int NT = S::NT;
  extern __shared__ __align__(16) uint8_t raw[];
  S& sm = *reinterpret_cast<S*>(raw);
  const int tid = threadIdx.x, w = tid >> 5, split = blockIdx.x;
  cluster_arrive_release();   // waited for before the first push into a peer
  pdl_wait();
  pdl_launch_dependents();
  // the CTAs of a cluster have one chunk: they leave together
  RowPlace place;
  if (static_cast<int>(blockIdx.y) >= find_chunks(a, sm.chunk, place)) {
    cluster_wait_acquire();
    return;
  }
  select_chunk(a, place, blockIdx.y, sm.chunk);
  const int cols = (a.n + Ring<KT>::kCols - 1) / Ring<KT>::kCols, part = blockIdx.z * kSplits + split, parts = gridDim.z * kSplits;
  ExpandWarp<KT, 1> e(a, sm.ring[w], sm.turn[w], sm.chunk, static_cast<int>(static_cast<long long>(cols) * part / parts),
                      static_cast<int>(static_cast<long long>(cols) * (part + 1) / parts));
  e.start();
  if (e.rank > 0) {
    constexpr int own = S::kFrags / kSplits;
    float acc[1][NT][4] = {};
    shrink_sums<1, NT>(a, sm.chunk.row, sm.chunk.id, e.rank, 0, split, 1, acc);
    share_sums<1, NT>(acc, 1, split, own, sm.warp, sm.split);
    cluster_arrive_release();
    cluster_wait_acquire();
    // an owned element to one CTA per thread: two rows' pairs of ranks, three planes
    for (int i = tid; i < own * kSplits; i += kThreads) {
      const int mine = i % own, to = i / own;
      float4 s = sm.split[0][mine];
#pragma unroll
      for (int c = 1; c < kSplits; ++c) add4(s, sm.split[c][mine]);
      const int f = split * own + mine, l = f & 31, j = (f >> 5) * 8 + 2 * (l & 3);
      // the lane and the word that hold ranks j, j + 1 (run()'s order), rows g and g + 8
      const int step = KT == 1 ? 0 : (j >> 5) * 2 + (j >> 2 & 1), t = KT == 1 ? j >> 2 : j >> 3 & 3;
      const int word = j & 2;
#pragma unroll
      for (int p = 0; p < 3; ++p) {
        const uint32_t at = mapa_shared(smem_addr(&sm.planes.v[0][step][p][(l & ~3) | t]) + word * 4, to);
        st_cluster_u32(at, pack_bf16(s.x, s.y));
        st_cluster_u32(at + 4, pack_bf16(s.z, s.w));
        s.x -= bf16_part(s.x);
        s.y -= bf16_part(s.y);
        s.z -= bf16_part(s.z);
        s.w -= bf16_part(s.w);
      }
    }
    cluster_arrive_release();
  }
  cluster_wait_acquire();
  e.run(sm.planes);
}

// Opt a kernel in to more than 48 KB of shared memory, once per device.
template <class Kernel>
cudaError_t allow_smem(Kernel* kernel, size_t bytes, std::atomic<bool> (&set)[64]) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev >= 64 || !set[dev].load(std::memory_order_relaxed))) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
    if (e == cudaSuccess && dev < 64) set[dev].store(true, std::memory_order_relaxed);
  }
  return e;
}

template <int MT, int NT>
cudaError_t launch_shrink(const LoraArgs& a, cudaLaunchConfig_t cfg) {
  static_assert(sizeof(ShrinkSmem<MT, NT>) <= 113 * 1024, "shared memory for two CTAs per SM");
  static std::atomic<bool> set[64];
  cfg.gridDim = dim3(kSplits, (a.rank + NT * 8 - 1) / (NT * 8), std::min(a.rows, a.n_adapters + 1 + a.rows / (MT * 16)));
  cfg.dynamicSmemBytes = sizeof(ShrinkSmem<MT, NT>);
  if (const cudaError_t e = allow_smem(shrink_kernel<MT, NT>, cfg.dynamicSmemBytes, set); e != cudaSuccess) return e;
  return cudaLaunchKernelEx(&cfg, shrink_kernel<MT, NT>, a);
}

template <int KT>
cudaError_t launch_expand(const LoraArgs& a, cudaLaunchConfig_t cfg) {
  typedef ExpandSmem<KT> S;
  static_assert(sizeof(S) <= 227 * 1024 && S::per_sm(true) == 2, "shared memory");
  static std::atomic<bool> set[64];
  // one item per warp, or as many CTAs as are resident at once
  const long long items = static_cast<long long>((a.n + Ring<KT>::kCols - 1) / Ring<KT>::kCols) *
                          std::min(a.rows, a.n_adapters + 1 + a.rows / (kExpandTiles * 16));
  cfg.gridDim = dim3(static_cast<unsigned>(std::min<long long>((items + kWarps - 1) / kWarps, 152 * S::per_sm(a.vec))));
  cfg.dynamicSmemBytes = S::bytes(a.vec);
  if (const cudaError_t e = allow_smem(expand_kernel<KT>, sizeof(S), set); e != cudaSuccess) return e;
  return cudaLaunchKernelEx(&cfg, expand_kernel<KT>, a);
}

// At most so many chunks of 16 rows, and parts of at most 4096 columns (512 a CTA).
int fused_chunks(const LoraArgs& a) { return std::min(a.rows, a.n_adapters + 1 + a.rows / 16); }
int fused_parts(const LoraArgs& a) { return (a.n + 4095) / 4096; }

template <int KT>
cudaError_t launch_fused(const LoraArgs& a, cudaLaunchConfig_t cfg) {
  static_assert(sizeof(FusedSmem<KT>) <= 227 * 1024, "shared memory");
  static std::atomic<bool> set[64];
  cfg.gridDim = dim3(kSplits, fused_chunks(a), fused_parts(a));
  cfg.dynamicSmemBytes = sizeof(FusedSmem<KT>);
  if (const cudaError_t e = allow_smem(fused_kernel<KT>, cfg.dynamicSmemBytes, set); e != cudaSuccess) return e;
  return cudaLaunchKernelEx(&cfg, fused_kernel<KT>, a);
}

cudaError_t launch_lora(const LoraArgs& a, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = kSplits;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  // One launch while its clusters fit at once, two CTAs per SM up to rank 16 and one up to 32: a
  // call is 2 to 2.5 us shorter on the host (16.9 -> 14.6 us at 1 x 4096 x 4096), and mostly on the
  // GPU (64 rows, n 1024: 4.4 us, two launches 6.1; 144 rows of 16 adapters, n 4096, rank 16: 7.4,
  // 8.1; 64 rows, k 14336, rank 32: 7.2, 9.1; but 1 x 4096 x 4096 4.9, 4.4).  In two waves it is
  // the longer one: 256 rows, n 11008, rank 16 15.8 us (11.5), 16 rows of 16 adapters, n 1024,
  // rank 32 8.3 (5.8).
  if (a.rank <= 32 && fused_chunks(a) * fused_parts(a) <= (a.rank <= 16 ? 34 : 14))
    return a.rank <= 16 ? launch_fused<1>(a, cfg) : launch_fused<2>(a, cfg);
  // The first product's tile: as small as fits the chip in one wave of clusters, 34 of two CTAs
  // per SM, or nearly.  Up to 32 rows 16 by 16 ranks (16 rows, k 14336, rank 128 6.4 us, by 32 7.4, by
  // 64 8.8), then by 32 (16 rows of 16 adapters of rank 64 8.4; 10.7, 9.7), then by 64; more rows 32
  // by 32 (256 rows of one adapter, rank 64 10.3, 16 by 64 11.3; 144 rows, n 28672 26.3, 29.0) and
  // with many adapters 16 by 64 (256 rows of 32, rank 128 25.7, 32 by 32 31.9; 64 rows of 64, rank 64
  // 27.0, 31.8).
  auto clusters = [&](int rows, int ranks) {
    return std::min(a.rows, a.n_adapters + 1 + a.rows / rows) * ((a.rank + ranks - 1) / ranks);
  };
  const cudaError_t e = a.rows <= 32 ? (clusters(16, 16) <= 34   ? launch_shrink<1, 2>(a, cfg)
                                        : clusters(16, 32) <= 64 ? launch_shrink<1, 4>(a, cfg)
                                                                 : launch_shrink<1, 8>(a, cfg))
                        : clusters(32, 32) <= 52 ? launch_shrink<2, 4>(a, cfg)
                                                 : launch_shrink<1, 8>(a, cfg);
  if (e != cudaSuccess) return e;
  cfg.numAttrs = 1;
  return a.rank <= 16   ? launch_expand<1>(a, cfg)
         : a.rank <= 32 ? launch_expand<2>(a, cfg)
         : a.rank <= 64 ? launch_expand<4>(a, cfg)
                        : launch_expand<8>(a, cfg);
}

size_t lora_scratch(int rows, int rank) { return static_cast<size_t>(rows) * rank * 4; }

bool misaligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

}  // namespace
}  // namespace memspec

extern "C" {

memspec_status memspec_op_lora_scratch_bytes(int32_t rows, int32_t n_out, int32_t k, int32_t rank,
                                             size_t* bytes) {
  using namespace memspec;
  if (bytes == nullptr || rows < 1 || rows > kMaxLoraRows || n_out < 1 || k < 8 || k % 8 != 0 || rank < 8 ||
      rank % 8 != 0 || rank > kMaxRank) {
    set_op_error("rows in 1..256, n_out >= 1, k a positive multiple of 8, rank a multiple of 8 in 8..128");
    return MEMSPEC_ERR_INVALID_ARG;
  }
  *bytes = lora_scratch(rows, rank);
  return MEMSPEC_OK;
}

memspec_status memspec_op_lora(const memspec_lora* adapters, const void* x, int64_t ldx, const int32_t* ids,
                               const float* base, int64_t ld_base, float* y, int64_t ldy, int32_t rows,
                               int32_t n_out, int32_t k, void* scratch, size_t scratch_bytes, void* stream) {
  using namespace memspec;
  const char* why = nullptr;
  size_t need = 0;
  if (adapters == nullptr || adapters->a_dev == nullptr || adapters->b_dev == nullptr || x == nullptr ||
      ids == nullptr || y == nullptr || scratch == nullptr) {
    why = "null pointer";
  } else if (memspec_op_lora_scratch_bytes(rows, n_out, k, adapters->rank, &need) != MEMSPEC_OK) {
    return MEMSPEC_ERR_INVALID_ARG;
  } else if (adapters->n_adapters < 1 || std::max({adapters->n_adapters, n_out, k}) > (1 << 24)) {
    why = "n_adapters must be at least 1, n_adapters, n_out and k at most 2^24";
  } else if (rows > 1 && (ldx < k || ldx % 8 != 0 || ldy < n_out || (base != nullptr && ld_base < n_out) ||
                          std::max({ldx, ldy, base != nullptr ? ld_base : 0}) > INT64_C(1) << 40)) {
    why = "row strides must cover a row and be at most 2^40, x's a multiple of 8";
  } else if (rows > 1 && base == y && ld_base != ldy) {
    why = "in place, base and y have one row stride";
  } else if (misaligned(x, 16) || misaligned(adapters->a_dev, 16) || misaligned(adapters->b_dev, 16) ||
             misaligned(scratch, 16) || misaligned(y, 4) || misaligned(base, 4) || misaligned(ids, 4) ||
             misaligned(adapters->scales_dev, 4) || misaligned(adapters->ranks_dev, 4)) {
    why = "x, A, B and scratch must be 16-byte aligned, the rest 4-byte";
  } else if (scratch_bytes < need) {
    why = "scratch too small";
  }
  if (why != nullptr) {
    set_op_error(why);
    return MEMSPEC_ERR_INVALID_ARG;
  }
  LoraArgs a{};
  a.x = static_cast<const bf16*>(x);
  a.ldx = ldx;
  a.a = static_cast<const bf16*>(adapters->a_dev);
  a.b = static_cast<const bf16*>(adapters->b_dev);
  a.scales = adapters->scales_dev;
  a.ranks = adapters->ranks_dev;
  a.ids = ids;
  a.base = base;
  a.ld_base = ld_base;
  a.y = y;
  a.ldy = ldy;
  a.rows = rows;
  a.n = n_out;
  a.k = k;
  a.n_adapters = adapters->n_adapters;
  a.rank = adapters->rank;
  a.t = static_cast<float*>(scratch);
  a.vec = n_out % 4 == 0 && (rows == 1 || ldy % 4 == 0) && !misaligned(y, 16) &&
          (base == nullptr || ((rows == 1 || ld_base % 4 == 0) && !misaligned(base, 16)));
  const cudaError_t e = launch_lora(a, static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) {
    set_op_error(std::string("lora launch: ") + cudaGetErrorString(e));
    return MEMSPEC_ERR_CUDA;
  }
  return MEMSPEC_OK;
}

}  // extern "C"
