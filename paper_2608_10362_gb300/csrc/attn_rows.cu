// attn_rows.cu - attention of a batch's rows over a layer's cache (memspec_op_attention).
//
// A unit is the query vectors (rows x heads of a group) of one sequence and one head of k and
// v, up to VT of them, against all keys: S^T = K Q^T, P = exp2(S^T - m), O^T += V^T P^T with
// mma.sync (m16n8k16, fp32 sums), keys and then the vectors' elements as M, query vectors as N.
// Few vectors per key: the bound is reading K and V once, so work is cut by keys: all units'
// tiles of 128 keys, one after another, are split evenly over the CTAs (whatever the lengths
// are; every CTA works its share out from the lengths itself), a warp takes 16 keys at a time
// through a cp.async ring of its own.  What a unit's CTAs found is joined by a second launch.
//
// Scores are kept in units of log2: z = log2(e) scale q.k.  The running maximum m of a vector is
// taken again only when a score passes it by more than 2^14, so that O is rarely rescaled; it
// is set 2^6 below the largest, so that weights in fp16 stay clear of its small end.
// Codes: exact in fp16 (1024 + 128 + code by one byte permutation, less 1152).  K's scale
// multiplies the score, V's is added to it as a logarithm: weights are w' = p * scale_v with a
// maximum of their own kind, and the sum of p is that of w' / scale_v; so no range of scales
// overflows fp16.
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>
#include <cfloat>
#include <string>

#include "kv.cuh"
#include "ptx.cuh"

namespace memspec {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kTile = 16 * kWarps;          // keys that a CTA's warps take in one turn
constexpr float kStart = -FLT_MAX;          // the maximum of nothing
constexpr float kAbove = 14.f, kBelow = 6.f;

// One part of a call's keys: the batch's own, or (starts == nullptr) the prefix of all rows.
struct RowsArgs {
  KvView kv;
  const int *starts, *lens;
  int n_seq, rows;
  int prefix_len;            // the prefix's keys
  const bf16* q;
  long long ldq;
  const int* tree;
  float scale;               // log2(e) * the call's
  int group;                 // heads of q per head of k and v
  int n_heads;
  bf16* out;                 // where units within one CTA go, or nullptr: to `full`
  long long ldo;
  float* full;               // [rows][n_heads] records
  float* slots;              // [2 CTAs][VT] records
  uint32_t* bases;           // [n_seq + 1]: tiles before each sequence's units
};

// A record: HD sums, the maximum, the sum of weights (and two floats that align the next one).
template <int HD>
constexpr int kRecord = HD + 4;

template <int HD_, bool CODES_, int NT_>
struct Shape {
  static constexpr int HD = HD_, NT = NT_, VT = 8 * NT_;
  static constexpr bool CODES = CODES_;
  static constexpr int kRowBytes = HD * (CODES ? 1 : 2);
  static constexpr int kStage = 2 * 16 * kRowBytes + (CODES ? 128 : 0);
  static constexpr int kQBytes = VT * HD * 2;
  static constexpr int kFixed = (kMaxSeqs + 8) * 4 + kQBytes + VT * 16 + 64;
  static constexpr int kPerSm = CODES && NT <= 2 ? 2 : 1;
  static constexpr int kBudget = (kPerSm == 2 ? 113 : 226) * 1024 - kFixed;
  static constexpr int kDepth = std::min(8, kBudget / (kWarps * kStage));
  static constexpr int kParts = HD / 32;                 // the reduction goes in parts of 32 elements
  static constexpr int kRing = std::max(kWarps * kDepth * kStage, kWarps * VT * 32 * 4 + kWarps * VT * 8);
  static constexpr int kSmem = kFixed + kRing;
  static_assert(kDepth >= 2 && kSmem <= 227 * 1024, "shared memory");
};

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
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(at)
               : "memory");
  return v;
}
__device__ __forceinline__ uint32_t movmatrix(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
template <bool F16>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (F16)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
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

// The plan: sequence b's units are tiles bases[b] .. bases[b + 1], ordered by head, vector tile
// and key tile.  A sequence with rows has at least one tile, so that every row is written.
struct Unit {
  int b, head, vt, t0, t1, tiles;   // key tiles [t0, t1) of `tiles`
  int row0, n, vecs;
  long long keys, first;            // keys that anyone sees; the first row's own slot
};
template <int VT>
__device__ __forceinline__ SeqRows part_rows(const RowsArgs& a, int b) {
  if (a.starts == nullptr) return {0, a.rows, a.prefix_len};
  return seq_rows(a.starts, a.lens, b, a.rows);
}
__device__ __forceinline__ int keys_of(const RowsArgs& a, const SeqRows& s) {
  return min(max(s.len, 0), a.starts == nullptr ? a.prefix_len : a.kv.max_pos);
}
__host__ __device__ constexpr uint32_t tiles_of(int keys) { return keys == 0 ? 1 : (keys + kTile - 1u) / kTile; }

// Exclusive sums of the sequences' tiles into bases[0 .. n_seq], by all threads.
template <int VT>
__device__ void make_plan(const RowsArgs& a, uint32_t* bases, uint32_t* warp_sums) {
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
  uint32_t before = 0;
  for (int b0 = 0; b0 < a.n_seq; b0 += kThreads) {
    const int b = b0 + tid;
    uint32_t mine = 0;
    if (b < a.n_seq) {
      const SeqRows s = part_rows<VT>(a, b);
      const uint32_t vts = (static_cast<uint32_t>(s.n) * a.group + VT - 1) / VT;
      mine = vts * a.kv.n_heads * tiles_of(keys_of(a, s));
    }
    uint32_t incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const uint32_t up = __shfl_up_sync(~0u, incl, o);
      if (lane >= o) incl += up;
    }
    if (lane == 31) warp_sums[warp] = incl;
    __syncthreads();
    uint32_t sum = before;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) sum += warp_sums[w];
      before += warp_sums[w];
    }
    if (b < a.n_seq) bases[b] = sum + incl - mine;
    __syncthreads();
  }
  if (tid == 0) bases[a.n_seq] = before;
  __syncthreads();
}

// Where CTA c's share of the tiles begins, and which CTA has tile x.  No CTA that shares has
// nothing: with fewer tiles than CTAs the first ones have one each.
__device__ __forceinline__ uint32_t share_begin(uint32_t c, uint32_t ctas, uint32_t total) {
  ctas = min(ctas, total);
  return c >= ctas ? total : static_cast<uint32_t>(static_cast<uint64_t>(c) * total / ctas);
}
__device__ __forceinline__ uint32_t share_owner(uint32_t x, uint32_t ctas, uint32_t total) {
  return static_cast<uint32_t>(((static_cast<uint64_t>(x) + 1) * min(ctas, total) - 1) / total);
}

// Which vector of the tile sees which of its sequence's slots.
struct Sight {
  int limit;        // slots up to this one
  uint32_t bits;    // and of those from the first row's own on, bit by bit
};
__device__ __forceinline__ bool sees(const Sight& s, long long first, int key) {
  if (key <= s.limit) return true;
  const long long d = key - first;
  return d >= 0 && d < 32 && (s.bits >> d & 1);
}

template <class S>
struct Smem {
  uint32_t* bases;
  uint32_t* sums;
  char* q;
  Sight* sight;     // [VT]
  float* q_scale;
  char* ring;
  __device__ explicit Smem(char* p) {
    bases = reinterpret_cast<uint32_t*>(p);
    sums = bases + kMaxSeqs + 1;   // 7 words with room for 8 warps behind
    q = p + (kMaxSeqs + 8) * 4 + 64;
    sight = reinterpret_cast<Sight*>(q + S::kQBytes);
    q_scale = reinterpret_cast<float*>(sight + S::VT);
    ring = q + S::kQBytes + S::VT * 16;
  }
};

// Keys kb .. kb + 15 (as far as there are `end`) of one head into a stage: rows in 16-byte
// chunks, permuted so that the fragments' reads meet no bank twice.
template <class S>
__device__ __forceinline__ int k_chunk(int row, int c) {
  if constexpr (S::CODES) return S::HD == 128 ? c ^ (row & 1) * 4 : c;
  return c ^ (row & 7);
}
template <class S>
__device__ __forceinline__ int v_chunk(int row, int c) {
  if constexpr (S::CODES && S::HD == 64) return c ^ (row >> 1 & 3);
  return c ^ (row & 7);
}
template <class S>
__device__ __forceinline__ void fill(const KvView& kv, const char* k, const char* v, const float* ks, const float* vs,
                                     uint32_t stage, long long kb, long long end, int lane) {
  constexpr int C = S::kRowBytes / 16;   // chunks of a row
#pragma unroll
  for (int i = 0; i < 16 * C / 32; ++i) {
    const int at = i * 32 + lane, row = at / C, c = at % C;
    const bool on = kb + row < end;
    const long long off = (on ? kb + row : 0) * kv.pos + c * 16;
    cp_async16(stage + row * S::kRowBytes + k_chunk<S>(row, c) * 16, k + off, on);
    cp_async16(stage + 16 * S::kRowBytes + row * S::kRowBytes + v_chunk<S>(row, c) * 16, v + off, on);
  }
  if constexpr (S::CODES) {
    const int row = lane & 15;
    const bool on = kb + row < end;
    cp_async4(stage + 32 * S::kRowBytes + lane * 4, (lane < 16 ? ks : vs) + (on ? kb + row : 0) * kv.s_pos, on);
  }
}

template <class S>
__global__ void __launch_bounds__(kThreads, S::kPerSm) rows_kernel(const __grid_constant__ RowsArgs a) {
  constexpr int HD = S::HD, NT = S::NT, VT = S::VT, KS = HD / 16, MT = HD / 16;
  constexpr bool CODES = S::CODES;
  extern __shared__ __align__(128) char smem_raw[];
  const Smem<S> sm(smem_raw);
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, g = lane >> 2, t = lane & 3;
  pdl_wait();
  pdl_launch_dependents();
  make_plan<VT>(a, sm.bases, sm.sums);
  if (blockIdx.x == 0)
    for (int b = tid; b <= a.n_seq; b += kThreads) a.bases[b] = sm.bases[b];
  const uint32_t total = sm.bases[a.n_seq];
  uint32_t x = share_begin(blockIdx.x, gridDim.x, total);
  const uint32_t x1 = share_begin(blockIdx.x + 1, gridDim.x, total);
  const uint32_t ring = smem_addr(sm.ring) + warp * S::kDepth * S::kStage, q_smem = smem_addr(sm.q);

  while (x < x1) {
    // ---- the unit that tile x belongs to
    Unit u;
    {
      int lo = 0, hi = a.n_seq;   // the last b with bases[b] <= x
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        (sm.bases[mid] <= x ? lo : hi) = mid;
      }
      u.b = lo;
    }
    {
      const SeqRows s = part_rows<VT>(a, u.b);
      u.row0 = s.row0;
      u.n = s.n;
      u.keys = keys_of(a, s);
      u.first = a.starts == nullptr ? u.keys : static_cast<long long>(s.len) - s.n;
      u.tiles = tiles_of(static_cast<int>(u.keys));
      u.vecs = s.n * a.group;
      const uint32_t vts = (u.vecs + VT - 1) / VT, in = x - sm.bases[u.b];
      u.t0 = in % u.tiles;
      u.vt = in / u.tiles % vts;
      u.head = in / u.tiles / vts;
      u.t1 = static_cast<int>(min(static_cast<uint32_t>(u.tiles), u.t0 + (x1 - x)));
    }
    const long long end = min(u.keys, static_cast<long long>(u.t1) * kTile);
    const int seq = a.starts == nullptr ? 0 : u.b;
    const char* k = a.kv.k + seq * a.kv.seq + u.head * a.kv.head;
    const char* v = a.kv.v + seq * a.kv.seq + u.head * a.kv.head;
    const float* ks = CODES ? a.kv.k_scale + seq * a.kv.s_seq + u.head * a.kv.s_head : nullptr;
    const float* vs = CODES ? a.kv.v_scale + seq * a.kv.s_seq + u.head * a.kv.s_head : nullptr;
    const long long kb0 = static_cast<long long>(u.t0) * kTile + warp * 16;
#pragma unroll
    for (int d = 0; d < S::kDepth - 1; ++d) {
      if (kb0 + d * kTile < end) fill<S>(a.kv, k, v, ks, vs, ring + d * S::kStage, kb0 + d * kTile, end, lane);
      cp_commit();
    }

    // ---- the unit's vectors
    {
      constexpr int C = HD / 8, N = (VT * C + kThreads - 1) / kThreads;
      uint4 in[N];
      float top = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int at = i * kThreads + tid, vec = u.vt * VT + at / C;
        in[i] = make_uint4(0, 0, 0, 0);
        if (at < VT * C && vec < u.vecs) {
          const int row = u.row0 + vec / a.group, head = u.head * a.group + vec % a.group;
          in[i] = *reinterpret_cast<const uint4*>(a.q + row * a.ldq + head * HD + at % C * 8);
        }
        if constexpr (CODES) {
          const uint32_t w[4] = {in[i].x, in[i].y, in[i].z, in[i].w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float e0 = fabsf(__uint_as_float(w[j] << 16)), e1 = fabsf(__uint_as_float(w[j] & 0xffff0000u));
            if (e0 <= FLT_MAX) top = fmaxf(top, e0);
            if (e1 <= FLT_MAX) top = fmaxf(top, e1);
          }
        }
      }
      float up = 1.f;
      if constexpr (CODES) {
        // fp16 holds what bf16 holds of values near 2^10: the tile's largest is brought there by a
        // power of two, which is exact; what falls off is below 2^-34 of the largest
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
        if (lane == 0) sm.q_scale[warp] = top;
        __syncthreads();
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sm.q_scale[w]);
        const int e = top > 0.f ? min(max(ilogbf(top), -110), 127) : 0;
        up = __int_as_float((min(10 - e, 120) + 127) << 23);
        __syncthreads();
        if (tid == 0) sm.q_scale[0] = 1.f / up;
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int at = i * kThreads + tid, vec = at / C, c = at % C;
        if (at >= VT * C) continue;
        if constexpr (CODES) {
          const uint32_t w[4] = {in[i].x, in[i].y, in[i].z, in[i].w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            // elements hd, hd + 1 go where the fragments' order wants them: a lane's word of four codes
            // is one step's pairs k = 2t, 2t + 1 and 2t + 8, 2t + 9
            const int hd = c * 8 + j * 2, to = hd / 64 * 64 + hd % 16 / 4 * 16 + hd % 64 / 16 * 2 + hd % 4 / 2 * 8;
            const int chunk = to / 8 ^ (vec & 7);
            *reinterpret_cast<uint32_t*>(sm.q + vec * HD * 2 + chunk * 16 + to % 8 * 2) =
                pack_f16(__uint_as_float(w[j] << 16) * up, __uint_as_float(w[j] & 0xffff0000u) * up);
          }
        } else {
          *reinterpret_cast<uint4*>(sm.q + vec * HD * 2 + (c ^ (vec & 7)) * 16) = in[i];
        }
      }
      if (tid < VT) {
        const int vec = u.vt * VT + tid, j = vec / a.group;
        Sight s{0x7fffffff, 0u};
        if (a.starts != nullptr && vec < u.vecs) {
          s.limit = static_cast<int>(max(u.first + (a.tree != nullptr ? -1 : j), -1ll));
          if (a.tree != nullptr) s.bits = static_cast<uint32_t>(a.tree[u.row0 + j]);
        }
        sm.sight[tid] = s;
      }
      __syncthreads();
    }
    const float scale = CODES ? a.scale * sm.q_scale[0] : a.scale;
    uint32_t qf[NT <= 2 ? NT : 1][KS][2];
    auto q_frags = [&](int nt, int ks, uint32_t (&r)[4]) {   // of steps ks and ks + 1
      ldsm4(r, q_smem + (nt * 8 + (lane & 7)) * HD * 2 + ((ks * 2 + (lane >> 3)) ^ (lane & 7)) * 16);
    };
    if constexpr (NT <= 2) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int ks = 0; ks < KS; ks += 2) {
          uint32_t r[4];
          q_frags(nt, ks, r);
          qf[nt][ks][0] = r[0], qf[nt][ks][1] = r[1], qf[nt][ks + 1][0] = r[2], qf[nt][ks + 1][1] = r[3];
        }
    }

    // ---- the keys
    float o[MT][NT][4] = {}, m[NT][2], l[NT][2] = {};
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) m[nt][0] = m[nt][1] = kStart;
    int slot = 0;
    for (long long kb = kb0; kb < end; kb += kTile) {
      {
        const long long ahead = kb + (S::kDepth - 1) * kTile;
        const int to = slot == 0 ? S::kDepth - 1 : slot - 1;
        if (ahead < end) fill<S>(a.kv, k, v, ks, vs, ring + to * S::kStage, ahead, end, lane);
        cp_commit();
      }
      cp_wait<S::kDepth - 1>();
      __syncwarp();
      const uint32_t kp = ring + slot * S::kStage, vp = kp + 16 * S::kRowBytes;
      slot = slot + 1 == S::kDepth ? 0 : slot + 1;
      float z[NT][4] = {};
      if constexpr (CODES) {
#pragma unroll
        for (int h = 0; h < HD / 64; ++h) {
          const uint4 r0 = lds128(kp + g * S::kRowBytes + k_chunk<S>(g, t + 4 * h) * 16);
          const uint4 r1 = lds128(kp + (g + 8) * S::kRowBytes + k_chunk<S>(g + 8, t + 4 * h) * 16);
          const uint32_t w0[4] = {r0.x, r0.y, r0.z, r0.w}, w1[4] = {r1.x, r1.y, r1.z, r1.w};
#pragma unroll
          for (int p = 0; p < 4; p += 2) {
            uint32_t f[2][4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const uint32_t y0 = w0[p + i] ^ 0x80808080u, y1 = w1[p + i] ^ 0x80808080u;
              f[i][0] = codes_f16<0x4140>(y0), f[i][1] = codes_f16<0x4140>(y1);
              f[i][2] = codes_f16<0x4342>(y0), f[i][3] = codes_f16<0x4342>(y1);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              if constexpr (NT <= 2) {
                mma<true>(z[nt], f[0], qf[nt][4 * h + p][0], qf[nt][4 * h + p][1]);
                mma<true>(z[nt], f[1], qf[nt][4 * h + p + 1][0], qf[nt][4 * h + p + 1][1]);
              } else {
                uint32_t r[4];
                q_frags(nt, 4 * h + p, r);
                mma<true>(z[nt], f[0], r[0], r[1]);
                mma<true>(z[nt], f[1], r[2], r[3]);
              }
            }
          }
        }
      } else {
#pragma unroll
        for (int ks = 0; ks < KS; ks += 2) {
          uint32_t f[2][4];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int row = lane & 15;
            ldsm4(f[i], kp + row * S::kRowBytes + k_chunk<S>(row, 2 * (ks + i) + (lane >> 4)) * 16);
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            if constexpr (NT <= 2) {
              mma<false>(z[nt], f[0], qf[nt][ks][0], qf[nt][ks][1]);
              mma<false>(z[nt], f[1], qf[nt][ks + 1][0], qf[nt][ks + 1][1]);
            } else {
              uint32_t r[4];
              q_frags(nt, ks, r);
              mma<false>(z[nt], f[0], r[0], r[1]);
              mma<false>(z[nt], f[1], r[2], r[3]);
            }
          }
        }
      }
      // scores; rows g and g + 8 of the 16 keys
      float rv[2] = {1.f, 1.f};
      if constexpr (CODES) {
        const float* sc = reinterpret_cast<const float*>(sm.ring + (kp - smem_addr(sm.ring)) + 32 * S::kRowBytes);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float k_s = sc[g + 8 * i], v_s = sc[16 + g + 8 * i];
          if (k_s < kSmallestScale) k_s = kSmallestScale;   // a NaN stays
          if (v_s < kSmallestScale) v_s = kSmallestScale;
          k_s *= scale;
          const float lv = __log2f(v_s);
          rv[i] = __frcp_rn(v_s);
          if (isnan(rv[i])) rv[i] = 0.f;   // the weight is a NaN already where it counts
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            z[nt][2 * i] = fmaf(z[nt][2 * i], k_s, lv);
            z[nt][2 * i + 1] = fmaf(z[nt][2 * i + 1], k_s, lv);
          }
        }
      } else {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 4; ++i) z[nt][i] *= scale;
      }
      const bool edge = kb + 16 > end || kb + 15 >= u.first;
      if (edge) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const long long key = kb + g + (i >> 1) * 8;
            const Sight s = sm.sight[nt * 8 + 2 * t + (i & 1)];
            if (key >= end || !sees(s, u.first, static_cast<int>(key))) z[nt][i] = -INFINITY;
          }
      }
      bool above = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 2; ++i) above |= fmaxf(z[nt][i], z[nt][2 + i]) - m[nt][i] > kAbove;
      if (__any_sync(~0u, above)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float top = fmaxf(z[nt][i], z[nt][2 + i]);
#pragma unroll
            for (int d = 4; d < 32; d *= 2) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
            const float now = top - m[nt][i] > kAbove ? top - kBelow : m[nt][i], by = ex2(m[nt][i] - now);
            m[nt][i] = now;
            l[nt][i] *= by;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) o[mt][nt][i] *= by, o[mt][nt][2 + i] *= by;
          }
      }
      uint32_t p[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w[i] = ex2(z[nt][i] - m[nt][i & 1]);
          l[nt][i & 1] = CODES ? fmaf(w[i], rv[i >> 1], l[nt][i & 1]) : l[nt][i & 1] + w[i];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
          p[nt][i] = movmatrix(CODES ? pack_f16(w[2 * i], w[2 * i + 1]) : pack_bf16(w[2 * i], w[2 * i + 1]));
      }
      if constexpr (CODES) {
#pragma unroll
        for (int c = 0; c < MT; c += 2) {
          uint32_t r[4];
          const int row = lane & 15;
          ldsm4_t(r, vp + row * S::kRowBytes + v_chunk<S>(row, c + (lane >> 4)) * 16);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t y0 = r[2 * i] ^ 0x80808080u, y1 = r[2 * i + 1] ^ 0x80808080u;
            const uint32_t f[4] = {codes_f16<0x4240>(y0), codes_f16<0x4341>(y0), codes_f16<0x4240>(y1),
                                   codes_f16<0x4341>(y1)};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma<true>(o[c + i][nt], f, p[nt][0], p[nt][1]);
          }
        }
      } else {
        auto v_frags = [&](int mt, uint32_t (&f)[4]) {
          const int row = (lane & 7) + (lane >> 4) * 8;
          ldsm4_t(f, vp + row * S::kRowBytes + v_chunk<S>(row, 2 * mt + (lane >> 3 & 1)) * 16);
        };
        bool odd = false;   // an infinity or a NaN among values that not every vector sees
        if (edge) {
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            uint32_t f[4];
            v_frags(mt, f);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              odd |= (f[i] & 0x7f80u) == 0x7f80u || (f[i] & 0x7f800000u) == 0x7f800000u;
          }
          odd = __any_sync(~0u, odd);
        }
        if (!odd) {
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            uint32_t f[4];
            v_frags(mt, f);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma<false>(o[mt][nt], f, p[nt][0], p[nt][1]);
          }
        } else {
          // vector by vector, with the values that it does not see taken as 0: a weight of 0 times
          // one of these is not 0
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll 1
            for (int col = 0; col < 8; ++col) {
              const Sight s = sm.sight[nt * 8 + col];
              uint32_t keep[2];
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const long long key = kb + 2 * t + 8 * i;
                keep[i] = (key < end && sees(s, u.first, static_cast<int>(key)) ? 0xffffu : 0u) |
                          (key + 1 < end && sees(s, u.first, static_cast<int>(key + 1)) ? 0xffff0000u : 0u);
              }
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) {
                uint32_t f[4];
                v_frags(mt, f);
                f[0] &= keep[0], f[1] &= keep[0], f[2] &= keep[1], f[3] &= keep[1];
                float d[4] = {};
                mma<false>(d, f, p[nt][0], p[nt][1]);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  if (2 * t + (i & 1) == col) o[mt][nt][i] += d[i];
              }
            }
        }
      }
      __syncwarp();   // the stage is read before it is filled again
    }

    // ---- the warps' sums into one, 32 elements of the vectors at a time
    cp_wait<0>();
    __syncthreads();
    float* part = reinterpret_cast<float*>(sm.ring);             // [warp][VT][32]
    float* ml = part + kWarps * VT * 32;                         // [warp][VT][2]
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int d = 4; d < 32; d *= 2) l[nt][i] += __shfl_xor_sync(~0u, l[nt][i], d);
        if (g == 0)
          *reinterpret_cast<float2*>(ml + (warp * VT + nt * 8 + 2 * t + i) * 2) = make_float2(m[nt][i], l[nt][i]);
      }
    const bool whole = u.t0 == 0 && u.t1 == u.tiles;
    float* to = whole ? nullptr
                      : a.slots + (2 * static_cast<long long>(blockIdx.x) + (u.t0 == 0)) * VT * kRecord<HD>;
    __syncthreads();
#pragma unroll
    for (int half = 0; half < S::kParts; ++half) {
      if (half > 0) __syncthreads();
#pragma unroll
      for (int mh = 0; mh < 2; ++mh)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int e = mh * 16 + (CODES ? 2 * g + (i >> 1) : g + (i >> 1) * 8);
            part[(warp * VT + nt * 8 + 2 * t + (i & 1)) * 32 + (e ^ (t & 3) * 8)] = o[half * 2 + mh][nt][i];
          }
      __syncthreads();
      for (int i = tid; i < VT * 32; i += kThreads) {
        const int vec = i / 32, e = i % 32;
        float top = kStart;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, ml[(w * VT + vec) * 2]);
        float sum = 0.f, den = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float by = ex2(ml[(w * VT + vec) * 2] - top);
          sum = fmaf(by, part[(w * VT + vec) * 32 + (e ^ (vec >> 1 & 3) * 8)], sum);
          den = fmaf(by, ml[(w * VT + vec) * 2 + 1], den);
        }
        const int id = u.vt * VT + vec;
        if (id >= u.vecs) continue;
        const int row = u.row0 + id / a.group, head = u.head * a.group + id % a.group;
        if (whole && a.out != nullptr) {
          a.out[row * a.ldo + head * HD + half * 32 + e] = __float2bfloat16_rn(den == 0.f ? 0.f : sum / den);
          continue;
        }
        float* rec = whole ? a.full + (static_cast<long long>(row) * a.n_heads + head) * kRecord<HD>
                           : to + vec * kRecord<HD>;
        rec[half * 32 + e] = sum;
        if (half == 0 && e == 0) rec[HD] = top, rec[HD + 1] = den;
      }
    }
    __syncthreads();
    x += u.t1 - u.t0;
  }
}

// ---------------------------------------------------------------- joining what CTAs found
struct JoinPart {
  const uint32_t* bases;
  const float *slots, *full;
  int ctas, vt;              // vectors of a tile
  int keys;                  // of the prefix; -1: of the sequence
};
struct JoinArgs {
  JoinPart part[2];
  int parts;
  const int *starts, *lens;
  int n_seq, rows, max_pos, group, kv_heads;
  bf16* out;
  long long ldo;
};

template <int HD>
__global__ void __launch_bounds__(kThreads) join_kernel(const __grid_constant__ JoinArgs a) {
  constexpr int E = HD / 32;
  __shared__ int found[4];
  const int row = blockIdx.x, warp = threadIdx.x / 32, lane = threadIdx.x % 32, n_heads = a.group * a.kv_heads;
  pdl_wait();
  pdl_launch_dependents();
  if (threadIdx.x == 0) found[0] = -1;
  __syncthreads();
  for (int b = threadIdx.x; b < a.n_seq; b += kThreads) {
    const SeqRows s = seq_rows(a.starts, a.lens, b, a.rows);
    if (row >= s.row0 && row < s.row0 + s.n) found[0] = b, found[1] = s.row0, found[2] = s.n, found[3] = s.len;
  }
  __syncthreads();
  if (found[0] < 0) return;
  for (int h = blockIdx.y * kWarps + warp; h < n_heads; h += gridDim.y * kWarps) {
    float top = kStart, den = 0.f, sum[E] = {};
    bool any = false;
    for (int p = 0; p < a.parts; ++p) {
      const JoinPart& part = a.part[p];
      const bool own = part.keys < 0;
      const int b = own ? found[0] : 0, n = own ? found[2] : a.rows;
      const int keys = own ? min(max(found[3], 0), a.max_pos) : part.keys;
      const uint32_t tiles = tiles_of(keys), vec = (row - (own ? found[1] : 0)) * a.group + h % a.group;
      const uint32_t vts = (static_cast<uint32_t>(n) * a.group + part.vt - 1) / part.vt;
      const uint32_t t0 = part.bases[b] + ((h / a.group) * vts + vec / part.vt) * tiles;
      const uint32_t total = part.bases[own ? a.n_seq : 1];
      const int c0 = share_owner(t0, part.ctas, total), c1 = share_owner(t0 + tiles - 1, part.ctas, total);
      if (c0 == c1 && part.full == nullptr) continue;   // written by that CTA
      any = true;
      for (int c = c0; c <= c1; ++c) {
        const float* rec = c0 == c1 ? part.full + (static_cast<long long>(row) * n_heads + h) * kRecord<HD>
                                    : part.slots + ((2 * static_cast<long long>(c) + (c == c0)) * part.vt + vec % part.vt) *
                                                       kRecord<HD>;
        const float m = rec[HD], now = fmaxf(top, m), was = ex2(top - now), by = ex2(m - now);
        den = fmaf(rec[HD + 1], by, den * was);
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] = fmaf(rec[e * 32 + lane], by, sum[e] * was);
        top = now;
      }
    }
    if (!any) continue;
    bf16* out = a.out + row * a.ldo + h * HD;
#pragma unroll
    for (int e = 0; e < E; ++e) out[e * 32 + lane] = __float2bfloat16_rn(den == 0.f ? 0.f : sum[e] / den);
  }
}

// ---------------------------------------------------------------- host
struct Layout {   // of a call's scratch, in bytes
  size_t bases[2], slots[2], full[2], total;
  int nt[2], ctas[2];
};

int vector_tiles(long long vecs) { return static_cast<int>(std::min<long long>((vecs + 7) / 8, 5)); }
int per_sm(bool codes, int nt) { return codes && nt <= 2 ? 2 : 1; }

Layout lay_out(const memspec_batch* b, const memspec_kv* kv, const memspec_attention* p) {
  Layout l{};
  const int group = p->n_heads / kv->n_heads;
  const bool two = p->prefix != nullptr && p->prefix_len > 0;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t was = at;
    at += (bytes + 255) & ~size_t{255};
    return was;
  };
  const size_t record = (kv->head_dim + 4) * sizeof(float);
  for (int i = 0; i < (two ? 2 : 1); ++i) {
    const memspec_kv* part = i == 0 ? kv : p->prefix;
    l.nt[i] = vector_tiles(static_cast<long long>(i == 0 ? p->max_rows : b->rows) * group);
    l.ctas[i] = 152 * per_sm(part->k_scale_dev != nullptr, l.nt[i]);
    l.bases[i] = take((i == 0 ? b->n_seq + 1 : 2) * sizeof(uint32_t));
    l.slots[i] = take(size_t{2} * l.ctas[i] * l.nt[i] * 8 * record);
    l.full[i] = two ? take(static_cast<size_t>(b->rows) * p->n_heads * record) : 0;
  }
  l.total = at;
  return l;
}

template <class S>
cudaError_t launch_rows(const RowsArgs& a, cudaLaunchConfig_t cfg) {
  static std::atomic<bool> set[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev >= 64 || !set[dev].load(std::memory_order_relaxed))) {
    e = cudaFuncSetAttribute(rows_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    if (e == cudaSuccess && dev < 64) set[dev].store(true, std::memory_order_relaxed);
  }
  if (e != cudaSuccess) return e;
  cfg.dynamicSmemBytes = S::kSmem;
  return cudaLaunchKernelEx(&cfg, rows_kernel<S>, a);
}
template <int HD, bool CODES>
cudaError_t launch_nt(int nt, const RowsArgs& a, const cudaLaunchConfig_t& cfg) {
  switch (nt) {
    case 1: return launch_rows<Shape<HD, CODES, 1>>(a, cfg);
    case 2: return launch_rows<Shape<HD, CODES, 2>>(a, cfg);
    case 3: return launch_rows<Shape<HD, CODES, 3>>(a, cfg);
    case 4: return launch_rows<Shape<HD, CODES, 4>>(a, cfg);
    default: return launch_rows<Shape<HD, CODES, 5>>(a, cfg);
  }
}

bool misaligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

const char* attention_problem(const memspec_batch* b, const memspec_kv* kv, const memspec_attention* p) {
  if (const char* why = kv_problem(kv, false)) return why;
  if (const char* why = batch_problem(b, kv)) return why;
  if (p == nullptr) return "null pointer";
  if (p->n_heads < 1 || p->n_heads % kv->n_heads != 0 || p->n_heads / kv->n_heads > 64)
    return "n_heads must be a multiple of the cache's heads, up to 64 times as many";
  if (p->max_rows < 1 || p->max_rows > b->rows) return "max_rows must be in 1..rows";
  if (!(p->scale >= -3e38f && p->scale <= 3e38f)) return "scale must be finite";
  if (p->prefix != nullptr) {
    if (const char* why = kv_problem(p->prefix, false)) return why;
    if (p->prefix->n_heads != kv->n_heads || p->prefix->head_dim != kv->head_dim)
      return "the prefix must have the cache's heads and head_dim";
    if (p->prefix_len < 0 || p->prefix_len > p->prefix->max_pos) return "prefix_len must be in 0..the prefix's max_pos";
  }
  // tiles are counted in 32 bits; every vector tile has at most this many
  const double vts = static_cast<double>(b->rows) * (p->n_heads / kv->n_heads) / 8 + b->n_seq;
  const double keys = std::max(kv->max_pos, p->prefix != nullptr ? p->prefix_len : 0);
  if (vts * kv->n_heads * (keys / kTile + 1) >= 4e9) return "too many rows for so many positions: split the call";
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
  RowsArgs a{};
  a.rows = batch->rows;
  a.q = static_cast<const bf16*>(p->q_dev);
  a.ldq = batch->rows > 1 ? p->ldq : 0;
  a.scale = p->scale * 1.4426950408889634f;
  a.n_heads = p->n_heads;
  a.group = p->n_heads / kv->n_heads;
  JoinArgs j{};
  j.parts = two ? 2 : 1;
  j.starts = batch->starts_dev;
  j.lens = batch->lens_dev;
  j.n_seq = batch->n_seq;
  j.rows = batch->rows;
  j.max_pos = kv->max_pos;
  j.group = a.group;
  j.kv_heads = kv->n_heads;
  j.out = static_cast<bf16*>(p->out_dev);
  j.ldo = batch->rows > 1 ? p->ldo : 0;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kThreads);
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cudaError_t e = cudaSuccess;
  for (int i = 0; i < j.parts && e == cudaSuccess; ++i) {
    a.kv = kv_view(i == 0 ? kv : p->prefix);
    a.starts = i == 0 ? batch->starts_dev : nullptr;
    a.lens = batch->lens_dev;
    a.n_seq = i == 0 ? batch->n_seq : 1;
    a.prefix_len = i == 0 ? 0 : p->prefix_len;
    a.tree = i == 0 ? p->tree_dev : nullptr;
    a.out = two ? nullptr : j.out;
    a.ldo = j.ldo;
    a.full = two ? reinterpret_cast<float*>(mem + l.full[i]) : nullptr;
    a.slots = reinterpret_cast<float*>(mem + l.slots[i]);
    a.bases = reinterpret_cast<uint32_t*>(mem + l.bases[i]);
    j.part[i] = {a.bases, a.slots, a.full, l.ctas[i], l.nt[i] * 8, i == 0 ? -1 : p->prefix_len};
    cfg.gridDim = dim3(l.ctas[i]);
    const bool codes = a.kv.k_scale != nullptr;
    e = kv->head_dim == 64 ? (codes ? launch_nt<64, true>(l.nt[i], a, cfg) : launch_nt<64, false>(l.nt[i], a, cfg))
                           : (codes ? launch_nt<128, true>(l.nt[i], a, cfg) : launch_nt<128, false>(l.nt[i], a, cfg));
  }
  if (e == cudaSuccess) {
    cfg.gridDim = dim3(batch->rows, (p->n_heads + 4 * kWarps - 1) / (4 * kWarps));
    e = kv->head_dim == 64 ? cudaLaunchKernelEx(&cfg, join_kernel<64>, j) : cudaLaunchKernelEx(&cfg, join_kernel<128>, j);
  }
  if (e != cudaSuccess) {
    set_op_error(std::string("attention launch: ") + cudaGetErrorString(e));
    return MEMSPEC_ERR_CUDA;
  }
  return MEMSPEC_OK;
}

}  // extern "C"
