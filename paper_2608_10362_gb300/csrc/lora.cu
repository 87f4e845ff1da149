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
//   1. shrink: t = A x.  A cluster of 8 CTAs splits k, the 8 warps of a CTA split its part;
//      the sums are added warp by warp, then pushed into the CTA of the cluster that owns
//      the element and added rank by rank: one order, one t.
//   2. expand: y = base + scale B t.  t enters as three bf16 planes, which hold all its 24
//      bits.  The columns of four n = 8 tiles are dealt so that a thread's results are 8
//      consecutive floats of a row.  B, the base and the ids are read while the shrink
//      launch still runs (everything before it has completed when this one starts).
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

__device__ __forceinline__ int rank_of(const LoraArgs& a, int id) {
  return a.ranks == nullptr ? a.rank : max(0, min(a.ranks[id], a.rank));
}

// D += A B, 16 x 8 x 16.
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Chunk c of the call: up to CH rows of one adapter.
template <int CH>
struct Chunk {
  int ids[kMaxLoraRows];    // -1: none
  int leaders[kThreads / 32];
  int row[CH];              // the chunk's rows, ascending; -1 past the last
  int id, first;
  bool found;
};
// Chunks are numbered by their first row.  All threads; false: there is no chunk c.
template <int CH>
__device__ bool find_chunk(const LoraArgs& a, int c, Chunk<CH>& s) {
  const int tid = threadIdx.x;
  int id = -2;
  if (tid < a.rows) {
    id = __ldcg(a.ids + tid);
    if (id < 0 || id >= a.n_adapters) id = -1;
  }
  s.ids[tid] = id;
  if (tid < CH) s.row[tid] = -1;
  if (tid == 0) s.found = false;
  __syncthreads();
  int pos = 0;              // rows of the same adapter before this one
  const int4* v = reinterpret_cast<const int4*>(s.ids);
  const int last = min(tid, a.rows) >> 2;
  for (int j = 0; j <= last && j < kMaxLoraRows / 4; ++j) {
    const int4 q = v[j];
    pos += (q.x == id && 4 * j < tid) + (q.y == id && 4 * j + 1 < tid) + (q.z == id && 4 * j + 2 < tid) +
           (q.w == id && 4 * j + 3 < tid);
  }
  const bool leads = tid < a.rows && pos % CH == 0;
  const unsigned mask = __ballot_sync(0xffffffffu, leads);
  if ((tid & 31) == 0) s.leaders[tid >> 5] = __popc(mask);
  __syncthreads();
  int before = __popc(mask & ((1u << (tid & 31)) - 1));
  for (int w = 0; w < (tid >> 5); ++w) before += s.leaders[w];
  if (leads && before == c) {
    s.id = id;
    s.first = pos;
    s.found = true;
  }
  __syncthreads();
  if (!s.found) return false;
  if (tid < a.rows && id == s.id && pos >= s.first && pos < s.first + CH) s.row[pos - s.first] = tid;
  __syncthreads();
  return true;
}

// t[row][j] for a chunk of up to 16 MT rows and 8 NT of the adapter's rows.  Grid (cluster
// of kSplits over k, chunks, groups of 8 NT ranks).
template <int MT, int NT>
struct ShrinkSmem {
  static constexpr int kElems = MT * 16 * NT * 8;
  Chunk<MT * 16> chunk;
  float warp[kWarps][kElems];                 // a warp's sums
  float split[kSplits][kElems / kSplits];     // this CTA's elements, from each CTA of the cluster
};

template <int MT, int NT>
__global__ void __launch_bounds__(kThreads) shrink_kernel(const __grid_constant__ LoraArgs a) {
  extern __shared__ __align__(16) uint8_t raw[];
  typedef ShrinkSmem<MT, NT> S;
  S& sm = *reinterpret_cast<S*>(raw);
  const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int split = blockIdx.x, j0 = blockIdx.z * NT * 8;
  cluster_arrive_release();   // waited for before the first push into a peer
  pdl_wait();
  pdl_launch_dependents();
  // the CTAs of a cluster have one chunk and one rank group: they leave together
  const bool found = find_chunk(a, blockIdx.y, sm.chunk) && sm.chunk.id >= 0;
  const int rank = found ? rank_of(a, sm.chunk.id) : 0;
  if (j0 >= rank) {
    cluster_wait_acquire();
    return;
  }
  const bf16* xr[MT][2];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = sm.chunk.row[m * 16 + h * 8 + g];
      xr[m][h] = r < 0 ? nullptr : a.x + r * a.ldx + 8 * t;
    }
  const bf16* ar[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int j = j0 + n * 8 + g;
    ar[n] = j < rank ? a.a + (static_cast<long long>(sm.chunk.id) * a.rank + j) * a.k + 8 * t : nullptr;
  }
  int tiles = 0;              // 16-row tiles with rows
#pragma unroll
  for (int m = 0; m < MT; ++m) tiles += sm.chunk.row[m * 16] >= 0;
  float acc[MT][NT][4] = {};
  const int blocks = (a.k + 31) / 32;         // of 32 columns
  const int end = static_cast<int>(static_cast<long long>(split + 1) * blocks / kSplits);
  const uint4 zero = make_uint4(0, 0, 0, 0);
  constexpr int kAhead = MT * 2 + NT <= 4 ? 4 : 2;    // blocks loaded together
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
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        sm.warp[w][(m * 16 + (q >> 1) * 8 + g) * (NT * 8) + n * 8 + 2 * t + (q & 1)] = acc[m][n][q];
  __syncthreads();
  cluster_wait_acquire();
  constexpr int kOwn = S::kElems / kSplits;
  for (int e = tid; e < S::kElems; e += kThreads) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) s += sm.warp[i][e];
    st_cluster_f(mapa_shared(smem_addr(&sm.split[split][e % kOwn]), e / kOwn), s);
  }
  cluster_arrive_release();
  cluster_wait_acquire();
  for (int i = tid; i < kOwn; i += kThreads) {
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < kSplits; ++c) s += sm.split[c][i];
    const int e = split * kOwn + i, j = j0 + e % (NT * 8), r = sm.chunk.row[e / (NT * 8)];
    if (r >= 0 && j < a.rank) a.t[r * a.rank + j] = s;
  }
}

// y for a chunk of up to 32 rows; a warp takes 32 columns at a time.  KT: steps of 16 ranks.
constexpr int kExpandTiles = 2;
constexpr int kColsPerWarp = 32;
template <int KT>
struct ExpandSmem {
  Chunk<kExpandTiles * 16> chunk;
  uint4 t[kExpandTiles][KT][3][32];   // fragments of t's planes, one per lane
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float bf16_part(float x) { return __bfloat162float(__float2bfloat16_rn(x)); }

template <int KT>
__global__ void __launch_bounds__(kThreads, KT <= 4 ? 2 : 1) expand_kernel(const __grid_constant__ LoraArgs a) {
  __shared__ ExpandSmem<KT> sm;
  const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  // the ids, B, base and scales may be read now: the launch before this one (shrink) lets
  // it start only after its own wait, so all that came earlier has completed
  if (!find_chunk(a, blockIdx.y, sm.chunk)) return;
  const int id = sm.chunk.id;
  const int rank = id < 0 ? 0 : rank_of(a, id);
  const float scale = id < 0 || a.scales == nullptr ? 1.f : a.scales[id];
  const int steps = (rank + 15) / 16;
  int tiles = 0;
#pragma unroll
  for (int m = 0; m < kExpandTiles; ++m) tiles += sm.chunk.row[m * 16] >= 0;
  // column of MMA column n of tile j: 8 consecutive ones per thread, or (rows that no
  // 16-byte access fits) pairs
  const int bcol = a.vec ? 8 * (g >> 1) + (g & 1) : g, bstep = a.vec ? 2 : 8;
  const bf16* bw = a.b + static_cast<long long>(max(id, 0)) * a.n * a.rank + 4 * t;
  uint2 bv[KT][4];
  auto load_b = [&](int c0) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int col = c0 + bcol + j * bstep;
      const bf16* p = bw + static_cast<long long>(col) * a.rank;
#pragma unroll
      for (int s = 0; s < KT; ++s) {
        const int r = s * 16 + 4 * t;
        bv[s][j] = make_uint2(0, 0);
        if (col < a.n && r < rank) {
          bv[s][j] = __ldcg(reinterpret_cast<const uint2*>(p + s * 16));
          if (r + 4 > rank) {     // entries past the adapter's rank may be anything
            if (r + 1 >= rank) bv[s][j].x &= 0xffffu;
            if (r + 2 >= rank) bv[s][j].y = 0;
            if (r + 3 >= rank) bv[s][j].y &= 0xffffu;
          }
        }
      }
    }
  };
  float base[2][8];
  auto load_base = [&](int m, int c0) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = sm.chunk.row[m * 16 + h * 8 + g];
      const float* p = a.base + r * a.ld_base + c0;
#pragma unroll
      for (int i = 0; i < 8; ++i) base[h][i] = 0.f;
      if (r < 0 || a.base == nullptr) continue;
      if (a.vec) {
#pragma unroll
        for (int q = 0; q < 2; ++q)
          if (c0 + 8 * t + 4 * q < a.n) {
            const float4 v = __ldcg(reinterpret_cast<const float4*>(p + 8 * t + 4 * q));
            base[h][4 * q] = v.x, base[h][4 * q + 1] = v.y, base[h][4 * q + 2] = v.z, base[h][4 * q + 3] = v.w;
          }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int c = (i >> 1) * 8 + 2 * t + (i & 1);
          if (c0 + c < a.n) base[h][i] = __ldcg(p + c);
        }
      }
    }
  };
  const int stride = gridDim.x * kWarps * kColsPerWarp;
  const int c_first = (blockIdx.x * kWarps + w) * kColsPerWarp;
  load_b(c_first);
  load_base(0, c_first);
  pdl_wait();
  pdl_launch_dependents();
  for (int i = tid; i < tiles * steps * 32; i += kThreads) {
    const int l = i & 31, s = (i >> 5) % steps, m = (i >> 5) / steps;
    const int r = s * 16 + 4 * (l & 3);
    float v[2][4] = {};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = sm.chunk.row[m * 16 + h * 8 + (l >> 2)];
      if (row < 0 || r >= rank) continue;
      const float4 q = __ldcg(reinterpret_cast<const float4*>(a.t + row * a.rank + r));
      v[h][0] = q.x;
      v[h][1] = r + 1 < rank ? q.y : 0.f;
      v[h][2] = r + 2 < rank ? q.z : 0.f;
      v[h][3] = r + 3 < rank ? q.w : 0.f;
    }
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      sm.t[m][s][p][l] = make_uint4(pack_bf16(v[0][0], v[0][1]), pack_bf16(v[1][0], v[1][1]),
                                    pack_bf16(v[0][2], v[0][3]), pack_bf16(v[1][2], v[1][3]));
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int q = 0; q < 4; ++q) v[h][q] -= bf16_part(v[h][q]);
    }
  }
  __syncthreads();
  for (int c0 = c_first; c0 < a.n; c0 += stride) {
    if (c0 != c_first) load_b(c0);
    for (int m = 0; m < tiles; ++m) {
      if (c0 != c_first || m > 0) load_base(m, c0);
      float acc[4][4] = {};
#pragma unroll
      for (int s = 0; s < KT; ++s) {
        if (s >= steps) break;
#pragma unroll
        for (int p = 0; p < 3; ++p) {
          const uint4 f = sm.t[m][s][p][lane];
          const uint32_t fa[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) mma(acc[j], fa, bv[s][j].x, bv[s][j].y);
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = sm.chunk.row[m * 16 + h * 8 + g];
        if (r < 0) continue;
        float* y = a.y + r * a.ldy + c0;
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = rank > 0 ? fmaf(scale, acc[i >> 1][h * 2 + (i & 1)], base[h][i]) : base[h][i];
        if (a.vec) {
#pragma unroll
          for (int q = 0; q < 2; ++q)
            if (c0 + 8 * t + 4 * q < a.n)
              *reinterpret_cast<float4*>(y + 8 * t + 4 * q) = make_float4(o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int c = (i >> 1) * 8 + 2 * t + (i & 1);
            if (c0 + c < a.n) y[c] = o[i];
          }
        }
      }
    }
  }
}

template <int MT, int NT>
cudaError_t launch_shrink(const LoraArgs& a, cudaLaunchConfig_t cfg) {
  static_assert(sizeof(ShrinkSmem<MT, NT>) <= 227 * 1024, "shared memory");
  cfg.gridDim = dim3(kSplits, std::min(a.rows, a.n_adapters + 1 + a.rows / (MT * 16)), (a.rank + NT * 8 - 1) / (NT * 8));
  cfg.dynamicSmemBytes = sizeof(ShrinkSmem<MT, NT>);
  if (sizeof(ShrinkSmem<MT, NT>) > 48 * 1024) {   // set once per device
    static std::atomic<bool> set[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && (dev >= 64 || !set[dev].load(std::memory_order_relaxed))) {
      e = cudaFuncSetAttribute(shrink_kernel<MT, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                               static_cast<int>(cfg.dynamicSmemBytes));
      if (e == cudaSuccess && dev < 64) set[dev].store(true, std::memory_order_relaxed);
    }
    if (e != cudaSuccess) return e;
  }
  return cudaLaunchKernelEx(&cfg, shrink_kernel<MT, NT>, a);
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
  const cudaError_t e = a.rows <= 32 ? launch_shrink<1, 2>(a, cfg) : launch_shrink<4, 4>(a, cfg);
  if (e != cudaSuccess) return e;
  cfg.numAttrs = 1;
  const int chunks = std::min(a.rows, a.n_adapters + 1 + a.rows / (kExpandTiles * 16));
  const int cols = (a.n + kWarps * kColsPerWarp - 1) / (kWarps * kColsPerWarp);
  cfg.gridDim = dim3(std::min(cols, std::max(1, 1216 / chunks)), chunks);
  return a.rank <= 16   ? cudaLaunchKernelEx(&cfg, expand_kernel<1>, a)
         : a.rank <= 32 ? cudaLaunchKernelEx(&cfg, expand_kernel<2>, a)
         : a.rank <= 64 ? cudaLaunchKernelEx(&cfg, expand_kernel<4>, a)
                        : cudaLaunchKernelEx(&cfg, expand_kernel<8>, a);
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
  } else if (adapters->n_adapters < 1 || n_out > (1 << 24) || k > (1 << 24)) {
    why = "n_adapters must be at least 1, n_out and k at most 2^24";
  } else if (ldx < k || ldx % 8 != 0 || ldy < n_out || (base != nullptr && ld_base < n_out)) {
    why = "row strides must cover a row, x's a multiple of 8";
  } else if (base == y && ld_base != ldy) {
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
  a.vec = n_out % 4 == 0 && ldy % 4 == 0 && !misaligned(y, 16) &&
          (base == nullptr || (ld_base % 4 == 0 && !misaligned(base, 16)));
  const cudaError_t e = launch_lora(a, static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) {
    set_op_error(std::string("lora launch: ") + cudaGetErrorString(e));
    return MEMSPEC_ERR_CUDA;
  }
  return MEMSPEC_OK;
}

}  // extern "C"
