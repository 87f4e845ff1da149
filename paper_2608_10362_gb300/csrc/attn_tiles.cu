// attn_tiles.cu - attention over a caller's cache for many query vectors per key: the verify
// rows of a batch, prompts, and a prefix that all rows share (memspec_op_attention).
//
// A unit (attn_plan.cuh) is up to 256 query vectors of one head of k and v.  The vectors are the
// rows of tcgen05 MMAs of M = 128, S = Q K^T and O += P V over tiles of 128 keys, S and O in
// tensor memory, P written over S.  Two softmax warpgroups, a thread per row:
//   units of more than 128 vectors: each has 128 of them and both halves of every tile, so that
//   a tile that was read once serves 256 vectors;
//   smaller ones: both have the same vectors, and a half of every tile each.
// A step is 64 keys of a warpgroup: its scores pass through registers once, and S has two buffers, so
// that the next step's MMAs run during this one's softmax.
// Every CTA takes an equal piece of the call's work whatever the lengths are, and leaves records
// of sums (two per vector for the smaller units) that attn_join.cu puts together.
//
// K and V pass through two slots each in shared memory, K-major and N-major alike [key][hd] with the
// 128-byte swizzle.  bf16 comes by TMA.  Codes are fetched by warps that write them as fp16, times their scale over
// a power of two near the tile's largest: a value is off by 2^-10 of itself (its factor and the product are
// rounded), or by 2^-15 of the largest scale of its tile (the product and what is taken from it round at fp16's smallest
// step, 2^-24, by half of it each, of what that scale makes 2^-9).  K's power multiplies the tile's scores, V's is added to
// them as a logarithm: weights are w' = p * power, against a maximum of their own kind, and the sum of p is that of
// w' / power; so no range of scales overflows fp16.  (Exact codes with a scale per key in the softmax, as attn_rows.cu
// has them, would be three numbers per key for every thread out of shared memory, at 128 bytes a clock 0.7 us of a
// step.)  A vector of Q is taken to fp16
// by a power of two of its own.
//
// What bounds it: a tile for 256 vectors takes 1.9 us of bf16, of which the MMAs' part is 1.3 (S in steps of 64 keys
// reads its operands from shared memory for 48 clocks per 32 of arithmetic), and 2.4 of codes, where converting and the
// softmax share the SM's issue.  64 rows of 32 heads, 8 of k and v, over 262144 positions: 219 us, 1.26 PFLOP/s, codes
// 256.  At ordinary lengths it is what comes before and after: 6 us to the first S, 2 to write the records, 4 to 6 for
// the join (the same rows over 8192 positions, caches cold, 26.5 us, of which 6.5 are tiles).  Registers are full: three of
// the four forms spill 12 to 32 bytes a thread.
//
// Roles (warps): 0-3, 4-7 softmax; copies, 4, or 8 of codes; two with the MMAs of a warpgroup each;
// one for Q; one for which units these are.  Every wait is bounded, those of a role's warps for one another too (see
// Stretches); after one that ran out the records of all the CTA's vectors are NaN, and so their results.
#include <algorithm>
#include <atomic>

#include "attn_plan.cuh"
#include "ptx.cuh"

namespace memspec {

namespace {

constexpr int kSoft = 256;              // threads of the softmax
constexpr int kSlots = 4;               // tiles in shared memory: K of two, V of two
constexpr int kRefs = 4;                // a tile's references are read until its P is written
constexpr int kListed = 8;              // stretches told of (as many again as are read behind one another at most)
constexpr int kStep = 64;               // keys of a warpgroup's step
// What a scale of 0 counts as: it meets -inf where a vector does not see a key, which 0 would make a NaN.  fp32's largest
// times it is 2^-21.
constexpr float kLeastScale = 0x1p-149f;
typedef TileUnits Units;
constexpr int kTilesUnit = Units::kUnit;

template <int HD_, bool CODES_>
struct Shape {
  static constexpr int HD = HD_;
  static constexpr bool CODES = CODES_;
  static constexpr int kCopy = CODES ? 128 : 64;       // threads for K, and as many for V
  static constexpr int kThreads = kSoft + 2 * kCopy + 128;
  static constexpr int kWidth = CODES ? 32 : 64;       // scores of a step in registers at a time (a thread has 96 and 128)
  static constexpr int kSlotBytes = kTile * HD * 2;
  static constexpr int kQBytes = 128 * HD * 2;         // of 128 vectors
  static constexpr int kSmem = 1024 + kSlots * kSlotBytes + 2 * kQBytes;
};

struct CodesSmem {   // of K's or V's threads, by the tile's parity: one barrier a tile
  float scale[2][kTile];
  float2 top[2][4];
};
struct Ctl {
  uint64_t full[kSlots], empty[kSlots];
  uint64_t raw[2];           // V of an edge tile has landed, but is still to be looked over
  uint64_t q_full;           // a stretch's vectors are there
  uint64_t q_free[2];        // its last S is complete: every second stretch, so that who waits is never a phase late
  uint64_t s_full[2][2];     // [warpgroup][buffer] S of a step is complete
  uint64_t p_full[2][2];     // ... its P is written (4 warps)
  uint64_t o_full[2][2];     // ... its P V is complete
  uint64_t drain[2];
  uint32_t tmem_base;
  int abort_flag;
  uint32_t bad[2][kTile / 32];        // keys of an edge tile whose values are not all finite
  float4 refs[kRefs];                 // codes: the exponents K's and V's scales are taken against, 1 / V's power of two
  CodesSmem codes[2];
  int q_exp[4][kTilesUnit];           // codes: the exponents that a stretch's vectors were taken down by; the next one's
                                      // may be there, and the one's after it begun, before this one's softmax reads its own
  Plan plan;
  uint64_t listed[kListed];           // a stretch's entry is there
  Stretch list[kListed];              // (none: t0 == t1)
};

// 32 TMEM lanes x 32 consecutive columns, a lane per thread: load (and wait) ...
__device__ __forceinline__ void tmem_ld_x32(uint32_t taddr, float* v) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
      "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
// ... 64 columns ...
__device__ __forceinline__ void tmem_ld_x64(uint32_t taddr, float* v) {
  uint32_t r[64];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
      "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, "
      "%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, "
      "%48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]),
        "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]),
        "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]),
        "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]),
        "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
      : "r"(taddr)
      : "memory");
#pragma unroll
  for (int i = 0; i < 64; ++i) v[i] = __uint_as_float(r[i]);
}
// ... and store (tmem_st_wait completes it).
__device__ __forceinline__ void tmem_st_x32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {"
      "%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st_x16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {"
      "%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Two floats at a time (half the issue slots, half the code).
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair_of(float a, float b) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void split(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// D[tmem] (+)= A[tmem] * B[smem], issued by one thread.
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                       uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Instruction descriptor: fp32 sums, A and B both bf16 or both fp16.
template <bool F16>
constexpr uint32_t idesc(int m, int n) {
  return make_idesc_bf16_f32(m, n) & ~(F16 ? (1u << 7) | (1u << 10) : 0u);
}

// ptx.cuh's mbar_wait_bounded, whose attempts may each sleep for 10 us.  A wait for a step or a tile is over when
// the others are slower than any they can be; one for a stretch lasts as long as the stretch has tiles.
constexpr long long kStretchBudgetCycles = 64 * kWaitBudgetCycles;
__device__ __forceinline__ bool wait_bounded(uint64_t* bar, uint32_t parity, volatile int* abort_flag,
                                             long long budget = kWaitBudgetCycles) {
  auto attempt = [&] {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_addr(bar)), "r"(parity), "r"(10000u)
        : "memory");
    return ok != 0;
  };
  if (attempt()) return true;
  const long long t0 = clock64();
#pragma unroll 1
  while (!attempt()) {
    if (abort_flag != nullptr && *abort_flag) return false;
    if (clock64() - t0 > budget) {
      if (abort_flag != nullptr) *abort_flag = 1;
      return false;
    }
  }
  return true;
}

// The slot of tile t (of the CTA) of K or V, and how often it has been used before.
__device__ __forceinline__ int slot_of(int t, int is_v) { return 2 * is_v + (t & 1); }
__device__ __forceinline__ int use_of(int t) { return t >> 1; }

struct TileMaps {   // of the caches of bf16
  CUtensorMap k[2], v[2];
};
// 5-D box: 64 columns, 128 positions, hd / 64 halves of one head and sequence
__device__ __forceinline__ void tma_load_5d(void* dst, const CUtensorMap* map, int pos, int head, int seq, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %2, %4, %5}], [%6];" ::"r"(smem_addr(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(pos), "r"(head), "r"(seq), "r"(smem_addr(bar))
      : "memory");
}

// Byte of element chunk c (16 bytes) of row r in an operand tile of 128 rows.
__device__ __forceinline__ int chunk_at(int r, int c) { return (c >> 3) * (128 * 128) + r * 128 + (((c ^ r) & 7) << 4); }

// The stretches of a CTA, as the roles go through them: one lane works them out (walk_role), and is
// never so far ahead that an entry is written again before all have read it.  All warps see the same ones: once a wait
// has run out that lane makes the next one the last.  So the warps of a role pass the same barriers whatever
// becomes of their waits: after one that ran out a warp goes on to the end of what is listed.  (That its results are lost is
// seen to at the end.  Leaving at each barrier by one decision: 16 x 9 rows over codes 38.9 us, at each stretch 38.0.)
struct Stretches {
  Ctl& ctl;
  int at = 0;
  __device__ explicit Stretches(Ctl& c) : ctl(c) {}
  __device__ __forceinline__ bool next(Stretch& u) {
    const int i = at % kListed;
    // (not given up for abort_flag: walk_role looks at that, and lists an end)
    if (!__all_sync(~0u, wait_bounded(&ctl.listed[i], static_cast<uint32_t>(at / kListed) & 1u, nullptr, 2 * kStretchBudgetCycles))) {
      ctl.abort_flag = 1;
      return false;
    }
    u = ctl.list[i];
    ++at;
    return u.t0 < u.t1;
  }
};
__device__ __forceinline__ void walk_role(const ListArgs& a, Ctl& ctl) {
  Walk<Units> walk(a, ctl.plan);
  Stretch u;
  bool more = true;
#pragma unroll 1
  for (int i = 0; more; ++i) {
    more = walk.next(u);
    // the last S of the stretch before last is complete: so are the roles' steps of the one two before that
    if (i >= 2 &&
        !wait_bounded(&ctl.q_free[i & 1], static_cast<uint32_t>(i - 2 >> 1) & 1u, &ctl.abort_flag, kStretchBudgetCycles))
      more = false;
    if (!more) u.t0 = u.t1 = 0;
    ctl.list[i % kListed] = u;
    mbar_arrive(&ctl.listed[i % kListed]);
  }
}
__device__ __forceinline__ bool is_pair(const Stretch& u) { return Units::pair(u.vecs, u.unit); }
// ---------------------------------------------------------------- copies
// A tile of V that not every vector sees all of: rows of the sequence's own, or rows past the keys' end.
__device__ __forceinline__ bool own_rows(const Stretch& u, int t) { return u.own && (t + 1) * kTile > u.first; }
__device__ __forceinline__ bool is_edge(const Stretch& u, int t) { return own_rows(u, t) || (t + 1) * kTile > u.end(); }

// bf16: one lane for K, one for V.
template <class S>
__device__ __forceinline__ void tma_role(const ListArgs& a, const TileMaps& maps, Ctl& ctl, int is_v, uint8_t* ring) {
  Stretches walk(ctl);
  volatile int* abort_flag = &ctl.abort_flag;
  int tile = 0;
  uint64_t* last[2] = {nullptr, nullptr};   // what the last loads of the two slots complete, and its phase
  uint32_t raws = 0, phase[2] = {0, 0};
  bool ok = true;
  Stretch u;
#pragma unroll 1
  while (ok && walk.next(u)) {
    const int part = u.own ? 0 : 1;
    const CUtensorMap* map = is_v ? &maps.v[part] : &maps.k[part];
    const int seq = u.own && a.kv[0].seq != 0 ? u.b : 0, head = a.kv[part].head != 0 ? u.head : 0;
#pragma unroll 1
    for (int t = u.t0; t < u.t1; ++t, ++tile) {
      const int s = slot_of(tile, is_v), i = s & 1;
      if (use_of(tile) > 0 &&
          !__all_sync(~0u, wait_bounded(&ctl.empty[s], static_cast<uint32_t>(use_of(tile) - 1) & 1u, abort_flag))) {
        ok = false;
        break;
      }
      const bool edge = is_v && is_edge(u, t);
      uint64_t* bar = edge ? &ctl.raw[i] : &ctl.full[s];
      if (threadIdx.x % 32 == 0) {
        mbar_arrive_expect_tx(bar, S::kSlotBytes);
        tma_load_5d(ring + s * S::kSlotBytes, map, t * kTile, head, seq, bar);
      }
      last[i] = bar;
      phase[i] = edge ? raws >> i & 1u : static_cast<uint32_t>(use_of(tile)) & 1u;
      if (edge) raws ^= 1u << i;
      __syncwarp();
    }
  }
  for (int i = 0; i < 2; ++i)   // no copy is in flight when the CTA leaves, whoever gave up
    if (last[i] != nullptr) mbar_wait_drain(last[i], phase[i]);
}

// bf16: the edge tiles of V, by kCopy threads: zeros where the keys have ended (a weight of 0 times
// what lies there need not be 0), and for infinities and NaN of the rows' own, whose keys are noted.
template <class S>
__device__ __forceinline__ void edge_role(Ctl& ctl, uint8_t* ring) {
  constexpr int C = S::HD / 8;
  constexpr int kCopy = S::kCopy;
  const int tid = threadIdx.x % kCopy;
  Stretches walk(ctl);
  bool ok = true;
  int tile = 0;
  uint32_t raws = 0;
  Stretch u;
#pragma unroll 1
  while (walk.next(u)) {
#pragma unroll 1
    for (int t = u.t0; t < u.t1; ++t, ++tile) {
      if (!is_edge(u, t)) continue;
      const int s = slot_of(tile, 1), i = s & 1, key0 = t * kTile;
      ok = ok && __all_sync(~0u, wait_bounded(&ctl.raw[i], raws >> i & 1u, &ctl.abort_flag, kStretchBudgetCycles));
      raws ^= 1u << i;
      if (tid < kTile / 32) ctl.bad[i][tid] = 0u;
      named_bar_sync(2, kCopy);
      const int live = min(u.end() - key0, kTile);
      const int from = own_rows(u, t) ? min(static_cast<int>(max(u.first - key0, 0ll)), live) : live;
      auto chunk = [&](int at) {
        return reinterpret_cast<uint4*>(ring + s * S::kSlotBytes + chunk_at(at / C, at % C));
      };
#pragma unroll 1
      for (int at = live * C + tid; at < kTile * C; at += kCopy) *chunk(at) = make_uint4(0u, 0u, 0u, 0u);
      constexpr int N = 8;   // under way
#pragma unroll 1
      for (int at = from * C + tid; at < live * C; at += N * kCopy) {
        uint32_t odd = 0u;
#pragma unroll
        for (int n = 0; n < N; ++n) {   // (past the last: that thread's first again)
          const uint4 x = *chunk(at + n * kCopy < live * C ? at + n * kCopy : at);
          // exponents of all ones carry into the sign's place
          auto high = [](uint32_t v) { return (v & 0x7fff7fffu) + 0x00800080u; };
          if ((high(x.x) | high(x.y) | high(x.z) | high(x.w)) & 0x80008000u) odd |= 1u << n;
        }
#pragma unroll 1
        for (; odd != 0u; odd &= odd - 1u) {
          const int n = __ffs(odd) - 1, one = at + n * kCopy < live * C ? at + n * kCopy : at;
          atomicOr(&ctl.bad[i][one / C / 32], 1u << one / C % 32);
          *chunk(one) = make_uint4(0u, 0u, 0u, 0u);
        }
      }
      fence_proxy_async_smem();
      named_bar_sync(2, kCopy);
      if (ok && tid == 0) mbar_arrive(&ctl.full[s]);
    }
  }
}

// Codes: kCopy threads for K and as many for V.  64 bytes of a row by four lanes: a thread's 16 codes are two
// chunks of fp16.  The next tile is on its way to registers while this one is written.
__device__ __forceinline__ float sane_scale(float s) { return s < kSmallestScale ? kSmallestScale : s; }   // a NaN stays
__device__ __forceinline__ float finite_or_0(float s) { return s <= FLT_MAX ? s : 0.f; }
// The exponent that a tile's scales are taken against (the largest finite one's), as a power of two and its inverse.
__device__ __forceinline__ int reference(float top) { return min((__float_as_int(fmaxf(top, kSmallestScale)) >> 23) - 127, 126); }

template <class S>
__device__ __forceinline__ void codes_role(const ListArgs& a, Ctl& ctl, int is_v, uint8_t* ring, CodesSmem& sm) {
  constexpr int kCopy = S::kCopy;
  static_assert(kCopy == kTile, "a thread per scale");
  constexpr int J = S::HD / 64, N = kTile * 4 / kCopy;   // parts of a row, rows
  const int tid = threadIdx.x % kCopy, r0 = tid / 4, c = tid % 4;
  Stretches walk(ctl);
  int tile = 0;
  Stretch u;
#pragma unroll 1
  while (walk.next(u)) {
    const KvView& kv = a.kv[u.own ? 0 : 1];
    const int seq = u.own ? u.b : 0, end = u.end();
    const char* base = (is_v ? kv.v : kv.k) + seq * kv.seq + u.head * kv.head;
    const float* ks = kv.k_scale + seq * kv.s_seq + u.head * kv.s_head;
    const float* vs = kv.v_scale + seq * kv.s_seq + u.head * kv.s_head;
    uint4 next[N * J];
    float sc[2] = {0.f, 0.f};   // of V; of K (K's threads alone)
    auto fetch = [&](int t) {
      int key = t * kTile + r0;
      const char* src = base + key * kv.pos + c * 16;
      const long long step = kv.pos * (kCopy / 4);
#pragma unroll
      for (int n = 0; n < N; ++n) {
#pragma unroll
        for (int j = 0; j < J; ++j)
          next[n * J + j] = key < end ? __ldcs(reinterpret_cast<const uint4*>(src + j * 64)) : make_uint4(0, 0, 0, 0);
        key += kCopy / 4;
        src += step;
      }
    };
    auto fetch_scales = [&](int t) {
      const int key = t * kTile + tid;
      const long long at = key * kv.s_pos;
      sc[0] = key < end ? vs[at] : 0.f;
      if (!is_v) sc[1] = key < end ? ks[at] : 0.f;
      if (key + 2 * kTile < end)   // a later tile's lines into L2
        asm volatile("prefetch.global.L2 [%0];" ::"l"(base + (key + 2 * kTile) * kv.pos));
    };
    fetch_scales(u.t0);
    fetch(u.t0);
#pragma unroll 1
    for (int t = u.t0; t < u.t1; ++t, ++tile) {
      const int s = slot_of(tile, is_v), buf = tile & 1;
      const float v_s = sane_scale(sc[0]), k_s = sane_scale(sc[1]);
      sm.scale[buf][tid] = is_v ? v_s : k_s;
      float2 top = make_float2(finite_or_0(v_s), finite_or_0(k_s));
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        top.x = fmaxf(top.x, __shfl_xor_sync(~0u, top.x, o));
        top.y = fmaxf(top.y, __shfl_xor_sync(~0u, top.y, o));
      }
      if (tid % 32 == 0) sm.top[buf][tid / 32] = top;
      named_bar_sync(3 + is_v, kCopy);
#pragma unroll
      for (int i = 0; i < kCopy / 32; ++i) top.x = fmaxf(top.x, sm.top[buf][i].x), top.y = fmaxf(top.y, sm.top[buf][i].y);
      const int ref_v = reference(top.x), ref_k = reference(top.y);
      // (where it runs out the tile is written and told of all the same: four arrivals a tile, whose barrier keeps them apart)
      if (use_of(tile) > 0) wait_bounded(&ctl.empty[s], static_cast<uint32_t>(use_of(tile) - 1) & 1u, &ctl.abort_flag);
      __syncwarp();
      // V of a key whose scale is not finite: 0 where some vector does not see it, those that do are told
      if (is_v) {
        const uint32_t bad = __ballot_sync(~0u, !(sc[0] <= FLT_MAX));
        if (tid % 32 == 0) ctl.bad[s & 1][tid / 32] = bad;
      } else if (tid == 0) {   // (S of two tiles before is complete, after the softmax of four before: its entry is free)
        ctl.refs[tile % kRefs] = make_float4(__int_as_float(ref_k + 9), ref_v + 9.f, power(-ref_v) / 512.f, 0.f);
      }
      uint4 in[N * J];
#pragma unroll
      for (int i = 0; i < N * J; ++i) in[i] = next[i];
      if (t + 1 < u.t1) {
        fetch_scales(t + 1);
        fetch(t + 1);
      }
      const float down = power(-(is_v ? ref_v : ref_k));
      const bool hide = is_v && own_rows(u, t);
      uint8_t* slot = ring + s * S::kSlotBytes;
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const int r = r0 + n * (kCopy / 4);
        float f = sm.scale[buf][r] * down;
        if (!(f <= FLT_MAX)) f = hide ? 0.f : NAN;
        // a byte u = code + 128 alone is the fp16 u 2^-24: times f 2^15, less f / 4, it is code f 2^-9, rounded once
        // (f is below 2; of the last step below it 65504 is within a rounding)
        const __half2 by = __float2half2_rn(f >= 1.999f ? 65504.f : f * 32768.f), less = __hmul2(by, __float2half2_rn(-0x1p-17f));
        auto pair = [&](uint32_t bytes) {
          const __half2 y = __hfma2(*reinterpret_cast<const __half2*>(&bytes), by, less);
          return *reinterpret_cast<const uint32_t*>(&y);
        };
        auto chunk = [&](uint32_t a, uint32_t b) {   // eight codes
          return make_uint4(pair(__byte_perm(a, 0u, 0x4140)), pair(__byte_perm(a, 0u, 0x4342)), pair(__byte_perm(b, 0u, 0x4140)),
                            pair(__byte_perm(b, 0u, 0x4342)));
        };
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const uint4 x = in[n * J + j];
          const int ch = j * 8 + c * 2;
          *reinterpret_cast<uint4*>(slot + chunk_at(r, ch)) = chunk(x.x ^ 0x80808080u, x.y ^ 0x80808080u);
          *reinterpret_cast<uint4*>(slot + chunk_at(r, ch + 1)) = chunk(x.z ^ 0x80808080u, x.w ^ 0x80808080u);
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (threadIdx.x % 32 == 0) mbar_arrive(&ctl.full[s]);
    }
  }
}

// ---------------------------------------------------------------- query vectors
// A stretch's vectors into shared memory by THREADS threads (`tid` of them; sync: their barrier), K-major; a
// negative scale turns their signs.  Codes: to fp16.  ok: no wait of the warp has run out.
template <class S, int THREADS, class Sync>
__device__ __forceinline__ void load_q(const ListArgs& a, Ctl& ctl, const Stretch& u, int stretch, int tid, uint8_t* q_smem, bool ok,
                                       Sync sync) {
  constexpr int HD = S::HD, C = HD / 8;
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
  const int vec0 = u.unit * kTilesUnit, chunks = min(u.vecs - vec0, kTilesUnit) * C;
  auto dst = [&](int at) { return q_smem + (at / C >> 7) * S::kQBytes + chunk_at(at / C & 127, at % C); };
  // as they are, all under way at once; then each thread goes over its own
#pragma unroll 1
  for (int at = tid; at < chunks; at += THREADS) {
    const int id = vec0 + at / C, row = vector_row(a, id);
    cp_async16(smem_addr(dst(at)), a.q + static_cast<long long>(u.row0 + row) * a.ldq +
                                       (u.head * a.group + id - row * a.group) * HD + at % C * 8, true);
  }
  cp_commit();
  cp_wait<0>();
  if constexpr (S::CODES) {
#pragma unroll 4
    for (int at = tid; at - tid % 32 < chunks; at += THREADS) {   // (by whole warps; a vector's chunks are of one)
      const bool on = at < chunks;
      uint4* p = reinterpret_cast<uint4*>(dst(on ? at : tid));
      const uint4 x = *p;
      const int e = exponent_of_lanes<C>(x);
      const float up = power(-e);
      if (!on) continue;
      *p = make_uint4(scaled_f16(x.x ^ flip, up), scaled_f16(x.y ^ flip, up), scaled_f16(x.z ^ flip, up),
                      scaled_f16(x.w ^ flip, up));
      if (at % C == 0) ctl.q_exp[stretch & 3][at / C] = e;
    }
  } else if (flip != 0u) {
#pragma unroll 1
    for (int at = tid; at < chunks; at += THREADS) {
      uint4* p = reinterpret_cast<uint4*>(dst(at));
      const uint4 x = *p;
      *p = make_uint4(x.x ^ flip, x.y ^ flip, x.z ^ flip, x.w ^ flip);
    }
  }
  fence_proxy_async_smem();
  sync();
  if (ok && tid == 0) mbar_arrive(&ctl.q_full);
}

// The smaller units' vectors, ahead of their stretch.  Those of a pair are many, and the first stretch's are waited
// for by all: the softmax warps load them.
__device__ __forceinline__ bool softmax_loads(const Stretch& u, int stretch) { return stretch == 0 || is_pair(u); }
template <class S>
__device__ __forceinline__ void q_role(const ListArgs& a, Ctl& ctl, uint8_t* q_smem) {
  Stretches walk(ctl);
  int stretch = 0;
  Stretch u;
#pragma unroll 1
  for (; walk.next(u); ++stretch) {
    if (softmax_loads(u, stretch)) continue;
    if (stretch > 0 &&
        !__all_sync(~0u, wait_bounded(&ctl.q_free[(stretch - 1) & 1], static_cast<uint32_t>(stretch - 1 >> 1) & 1u, &ctl.abort_flag,
                                      kStretchBudgetCycles)))
      break;
    load_q<S, 32>(a, ctl, u, stretch, threadIdx.x % 32, q_smem, true, [] { __syncwarp(); });
  }
}

// ---------------------------------------------------------------- records
// Of vector v of a unit, copy c of it.  Records lie side by side, [HD / 4][records][4]: a warp's stores are whole lines.
struct Record {
  float* sums;        // 4 of its sums
  long long chunk;    // floats to the next 4
  float2* md;
};
template <int HD>
__device__ __forceinline__ Record record_of(const ListArgs& a, const Stretch& u, bool pair, int v, int c) {
  const int heads = a.group * a.kv_heads, vec = u.unit * kTilesUnit + v, vr = vector_row(a, vec);
  const long long all = static_cast<long long>(a.rows) * heads;
  const long long at = static_cast<long long>(u.row0 + vr) * heads + u.head * a.group + vec - vr * a.group;
  const bool whole = u.whole();
  const long long n = whole ? 2 * all : kTilesUnit, i = whole ? at + c * all : c * 128 + v;
  float* rec = whole ? a.full[u.own ? 0 : 1]
                     : a.slots + (2 * static_cast<long long>(blockIdx.x) + (u.t0 == 0)) * kTilesUnit * kRecord<HD>;
  return {rec + 4 * i, 4 * n, reinterpret_cast<float2*>(rec + HD * n + 2 * i)};
}
// After a wait that ran out: whatever was written, the CTA's vectors are NaN (all threads).
template <int HD>
__device__ __noinline__ void lose_records(const ListArgs& a, const Plan& plan) {
  Walk<Units> walk(a, plan);
  Stretch u;
#pragma unroll 1
  while (walk.next(u)) {
    const bool pair = is_pair(u);
    const int vecs = min(u.vecs - u.unit * kTilesUnit, kTilesUnit);
#pragma unroll 1
    for (int i = threadIdx.x; i < vecs * (pair ? 1 : 2); i += blockDim.x)
      *record_of<HD>(a, u, pair, i % vecs, i / vecs).md = make_float2(kStart, NAN);
  }
}

// ---------------------------------------------------------------- softmax
template <class S>
__device__ __forceinline__ void soft_role(const ListArgs& a, Ctl& ctl, uint8_t* q_smem, uint32_t tmem) {
  constexpr int HD = S::HD;
  constexpr bool CODES = S::CODES;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, w = warp / 4, row = threadIdx.x % 128;
  const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
  const uint32_t s_at = tmem + lanes + static_cast<uint32_t>(w * 128);
  const uint32_t o_at = tmem + lanes + 256 + static_cast<uint32_t>(w * HD);
  volatile int* abort_flag = &ctl.abort_flag;
  Stretches walk(ctl);
  bool ok = true;
  int done = 0, tiles = 0, stretch = 0;      // steps of this warpgroup, tiles of the CTA, before this stretch
  auto wait = [&](uint64_t* bar, int phase) {
    ok = ok && __all_sync(~0u, wait_bounded(bar, static_cast<uint32_t>(phase) & 1u, abort_flag));
    return ok;
  };
  Stretch u;
#pragma unroll 1
  while (walk.next(u)) {
    const bool pair = is_pair(u);
    const int vec = u.unit * kTilesUnit + (pair ? w * 128 : 0) + row, end = u.end();
    const bool live = vec < u.vecs, warp_live = __any_sync(~0u, live);
    const Sight sight = live ? sight_of(a, u, vec) : Sight{-1, 0u};
    int scale_e = 0;     // codes: the scale is scale * 2^scale_e, with the vector's power of two
    float scale = fmaxf(fabsf(a.scale), kLeastScale);
    if constexpr (CODES) {
      scale = frexpf(scale, &scale_e);
      if (a.scale == 0.f) scale_e = -1024;
    }
    float m = kStart, l = 0.f;
    bool huge = false;   // some m of the warp's
    if (softmax_loads(u, stretch)) {
      named_bar_sync(1, kSoft);   // both warpgroups have seen the last S of the stretch before: Q is free
      load_q<S, kSoft>(a, ctl, u, stretch, threadIdx.x, q_smem, ok, [] { named_bar_sync(1, kSoft); });
    }
#pragma unroll 1
    for (int t = u.t0; ok && t < u.t1; ++t)
#pragma unroll 1
      for (int half = pair ? 0 : w; half < (pair ? 2 : w + 1); ++half, ++done) {
        const int buf = done & 1, key0 = t * kTile + half * kStep;
        const bool begins = t == u.t0 && (half == 0 || !pair);
        if (!wait(&ctl.s_full[w][buf], done >> 1)) break;
        tc_fence_after();
        if (warp_live) {
          if (CODES && begins) scale_e += ctl.q_exp[stretch & 3][vec - u.unit * kTilesUnit];
          const uint32_t s_buf = s_at + buf * kStep;
          // z = by * S + plus: of codes with the tile's references
          float by = scale, plus = 0.f, l_by = 1.f;
          if constexpr (CODES) {
            // (products are 2^17 at most: below 2^-126 it does not matter what they are times)
            const float4 ref = ctl.refs[(tiles + t - u.t0) % kRefs];
            by *= power(min(max(scale_e + __float_as_int(ref.x), -126), 127)), plus = ref.y, l_by = ref.z;
          }
          const bool edge = key0 + kStep > end || key0 + kStep > u.first;
          unsigned long long seen = ~0ull;   // bit e: the vector sees key key0 + e
          if (edge) {
            auto below = [](long long n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1; };
            const long long d = u.first - key0;
            seen = below(static_cast<long long>(sight.limit) + 1 - key0);
            seen |= d >= 64 || d <= -32 ? 0ull
                    : d >= 0            ? static_cast<unsigned long long>(sight.bits) << d
                                        : static_cast<unsigned long long>(sight.bits >> -d);
            seen &= below(end - key0);
            if (own_rows(u, t)) {   // values that are not finite, to those that see them
              const int tile = tiles + t - u.t0, s = slot_of(tile, 1);
              if (!wait(&ctl.full[s], use_of(tile))) break;
              const uint32_t* words = &ctl.bad[s & 1][half * 2];
              const unsigned long long bad = words[0] | static_cast<unsigned long long>(words[1]) << 32;
              if ((bad & seen) != 0ull) l = NAN;
            }
          }
          // scores c .. c + W - 1 of the step
          constexpr int W = S::kWidth;
          float z[W];
          auto scores = [&](int c) {
            if constexpr (W == 64) tmem_ld_x64(s_buf + c, z);
            if constexpr (W == 32) tmem_ld_x32(s_buf + c, z);
            if (edge) {
              const unsigned long long here = seen >> c;
#pragma unroll
              for (int e = 0; e < W; ++e)
                if (!(static_cast<uint32_t>(e < 32 ? here : here >> 32) >> (e & 31) & 1u)) z[e] = -INFINITY;
            }
          };
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll 1
          for (int c = 0; c < kStep; c += W) {
            scores(c);
#pragma unroll
            for (int e = 0; e < W; ++e) mx[e & 3] = fmaxf(mx[e & 3], z[e]);
          }
          float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
          top = fmaf(top, by, plus);
          const bool above = live && top - m > Weights<CODES>::kAbove;   // (rows without a vector have anything)
          if (__any_sync(~0u, above)) {
            const float now = above ? top - Weights<CODES>::kBelow : m, less = ex2(m - now);
            m = now;
            l *= less;
            huge = __any_sync(~0u, live && fabsf(m) > 0x1p20f && m != kStart);
            if (!begins) {
              if (!wait(&ctl.o_full[w][buf ^ 1], (done - 1) >> 1)) break;
              tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < HD; c += 32) {
                float o[32];
                tmem_ld_x32(o_at + c, o);
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] *= less;
                tmem_st_x32(o_at + c, reinterpret_cast<const uint32_t*>(o));
              }
            }
          }
          f32x2 sum[2] = {0ull, 0ull};
          if (huge) {
            // scores so large that m's rounding shows: they are rounded as m was, else those next to the largest
            // would be past fp16 or fp32
            if constexpr (W == kStep) {
#pragma unroll
              for (int e = 0; e < W; ++e) z[e] = fmaf(z[e], by, plus);
            } else {
#pragma unroll 1
              for (int c = 0; c < kStep; c += 32) {
                float x[32];
                tmem_ld_x32(s_buf + c, x);
#pragma unroll
                for (int e = 0; e < 32; ++e) x[e] = fmaf(x[e], by, plus);
                tmem_st_x32(s_buf + c, reinterpret_cast<const uint32_t*>(x));
              }
              tmem_st_wait();
            }
            by = 1.f, plus = 0.f;
          }
          const f32x2 by2 = pair_of(by, by), plus2 = pair_of(plus - m, plus - m);
#pragma unroll 1
          for (int c = 0; c < kStep; c += W) {
            if constexpr (W < kStep) scores(c);
            uint32_t p[W / 2];
#pragma unroll
            for (int e = 0; e < W; e += 2) {
              float x0, x1;
              split(fma2(pair_of(z[e], z[e + 1]), by2, plus2), x0, x1);
              x0 = ex2(x0), x1 = ex2(x1);
              sum[e / 2 & 1] = add2(sum[e / 2 & 1], pair_of(x0, x1));
              p[e / 2] = CODES ? pack_f16(x0, x1) : pack_bf16(x0, x1);
            }
            if constexpr (W == 64) tmem_st_x32(s_buf, p);
            if constexpr (W == 32) tmem_st_x16(s_buf + c / 2, p);
          }
          float l0, l1;
          split(add2(sum[0], sum[1]), l0, l1);
          l = fmaf(l0 + l1, l_by, l);
          tmem_st_wait();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl.p_full[w][buf]);
      }
    // ---- the record
    wait(&ctl.o_full[w][(done - 1) & 1], (done - 1) >> 1);
    tc_fence_after();
    if (ok && warp_live) {
      // a pair's warpgroups have different vectors, others the same: two records of each
      const Record to = record_of<HD>(a, u, pair, vec - u.unit * kTilesUnit, pair ? 0 : w);
      if (live) *to.md = make_float2(m, l);
      float* rec = to.sums;
#pragma unroll 1
      for (int c = 0; c < HD; c += 32) {
        float o[32];
        tmem_ld_x32(o_at + c, o);
        if (live) {
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            *reinterpret_cast<float4*>(rec) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
            rec += to.chunk;
          }
        }
      }
    }
    tc_fence_before();
    tiles += u.t1 - u.t0;
    ++stretch;
  }
}

// ---------------------------------------------------------------- MMAs
// A warp issues all MMAs of a warpgroup: its steps are both halves of every tile with the warpgroup's own
// vectors (pair), or half w.  S of step n + 2 follows P V of step n, whose P lies where it goes: MMAs of
// one thread run in order, so nothing waits for that between them.  (A tcgen05 fence after a wait holds a
// thread until its own earlier MMAs have completed; those of the other warpgroup are another thread's.)
// The warp stays converged, one lane issues.
template <class S>
__device__ __forceinline__ void mma_role(Ctl& ctl, int w, const uint8_t* ring, const uint8_t* q_smem, uint32_t tmem) {
  constexpr uint32_t kIdS = idesc<S::CODES>(128, kStep), kIdO = idesc<S::CODES>(128, S::HD) | (1u << 16);   // V N-major
  const uint64_t kdesc = make_smem_desc_sw128(smem_addr(ring));
  // V tile, N-major: 64-element columns kTile x 128 bytes apart, 8-key groups 1024
  const uint64_t vdesc = (kdesc & ~(0xFFFFull << 16)) | (static_cast<uint64_t>((kTile * 128) >> 4) << 16);
  const bool lead = elect_one();
  volatile int* abort_flag = &ctl.abort_flag;
  Stretches walk(ctl);
  bool ok = true;
  auto wait = [&](uint64_t* bar, int phase) {
    ok = ok && __all_sync(~0u, wait_bounded(bar, static_cast<uint32_t>(phase) & 1u, abort_flag));
    return ok;
  };
  int tiles = 0, stretch = 0, done = 0;   // before this stretch; done: steps
  Stretch u;
#pragma unroll 1
  while (ok && walk.next(u)) {
    const bool pair = is_pair(u);
    const int per_tile = pair ? 2 : 1, steps = (u.t1 - u.t0) * per_tile;
    const uint64_t qdesc = make_smem_desc_sw128(smem_addr(q_smem + (pair ? w * S::kQBytes : 0)));
    if (!wait(&ctl.q_full, stretch)) break;
    auto tile_of = [&](int n) { return tiles + (pair ? n >> 1 : n); };
    auto first_key = [&](int n) { return (pair ? n & 1 : w) * kStep; };
    // n = -2, -1: the first two S; then P V of step n, and S of step n + 2
#pragma unroll 1
    for (int n = -2; n < steps; ++n) {
      if (n >= 0) {
        const int g = done + n, buf = g & 1, s = slot_of(tile_of(n), 1);
        if (!wait(&ctl.full[s], use_of(tile_of(n))) || !wait(&ctl.p_full[w][buf], g >> 1)) break;
        tc_fence_after();
        if (lead) {
          const uint64_t vd = vdesc + static_cast<uint32_t>((s * S::kSlotBytes + first_key(n) * 128) >> 4);
#pragma unroll
          for (int ks = 0; ks < kStep / 16; ++ks)
            mma_ts(tmem + 256 + w * S::HD, tmem + w * 128 + buf * kStep + ks * 8, vd + static_cast<uint32_t>((ks * 2048) >> 4),
                   kIdO, n > 0 || ks > 0 ? 1u : 0u);
          tc_commit(&ctl.o_full[w][buf]);
          if (!pair || (n & 1)) tc_commit(&ctl.empty[s]);
        }
        __syncwarp();
      }
      if (n + 2 < steps) {
        const int g = done + n + 2, buf = g & 1, s = slot_of(tile_of(n + 2), 0);
        if (!wait(&ctl.full[s], use_of(tile_of(n + 2)))) break;
        if (lead) {
          const uint64_t kd = kdesc + static_cast<uint32_t>((s * S::kSlotBytes + first_key(n + 2) * 128) >> 4);
#pragma unroll
          for (int ks = 0; ks < S::HD / 16; ++ks) {
            const uint32_t off = static_cast<uint32_t>(((ks >> 2) * kTile * 128 + (ks & 3) * 32) >> 4);
            tc_mma_bf16(tmem + w * 128 + buf * kStep, qdesc + off, kd + off, kIdS, ks > 0 ? 1u : 0u);
          }
          tc_commit(&ctl.s_full[w][buf]);
          if (!pair || (n & 1)) tc_commit(&ctl.empty[s]);
          if (n + 3 == steps) tc_commit(&ctl.q_free[stretch & 1]);
        }
        __syncwarp();
      }
    }
    done += steps;
    tiles += u.t1 - u.t0;
    ++stretch;
  }
  if (lead) {   // every MMA issued completes before the CTA leaves
    tc_commit(&ctl.drain[w]);
    mbar_wait_drain(&ctl.drain[w], 0);
  }
  __syncwarp();
}

template <class S>
__global__ void __launch_bounds__(S::kThreads, 1) tiles_kernel(const __grid_constant__ ListArgs a, const __grid_constant__ TileMaps maps) {
  __shared__ Ctl ctl;
  extern __shared__ uint8_t dsmem_raw[];
  uint8_t* ring = dsmem_raw + ((1024u - (smem_addr(dsmem_raw) & 1023u)) & 1023u);
  uint8_t* q_smem = ring + kSlots * S::kSlotBytes;
  const int warp = threadIdx.x / 32;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(&ctl.full[s], S::CODES ? S::kCopy / 32 : 1);
      mbar_init(&ctl.empty[s], 2);
    }
    mbar_init(&ctl.raw[0], 1);
    mbar_init(&ctl.raw[1], 1);
    mbar_init(&ctl.q_full, 1);
    mbar_init(&ctl.q_free[0], 2);
    mbar_init(&ctl.q_free[1], 2);
    for (int i = 0; i < 4; ++i) {
      mbar_init(&ctl.s_full[i >> 1][i & 1], 1);
      mbar_init(&ctl.p_full[i >> 1][i & 1], 4);
      mbar_init(&ctl.o_full[i >> 1][i & 1], 1);
    }
    mbar_init(&ctl.drain[0], 1);
    mbar_init(&ctl.drain[1], 1);
    for (int i = 0; i < kListed; ++i) mbar_init(&ctl.listed[i], 1);
    ctl.abort_flag = 0;
    fence_mbar_init();
  }
  constexpr int kMma = (kSoft + 2 * S::kCopy) / 32;   // the first warp of the MMAs
  if (warp == kMma) {
    tmem_alloc(&ctl.tmem_base, 512);
    tmem_relinquish();
  }
  if (!a.beside) pdl_wait();
  pdl_launch_dependents();
  tc_fence_before();
  make_plan<Units, S::kThreads>(a, ctl.plan);
  tc_fence_after();
  const uint32_t tmem = ctl.tmem_base;
  if (warp < 8) {
    soft_role<S>(a, ctl, q_smem, tmem);
  } else if (warp < kMma) {
    const int w = warp - kSoft / 32;
    if constexpr (S::CODES) {
      codes_role<S>(a, ctl, w / (S::kCopy / 32), ring, ctl.codes[w / (S::kCopy / 32)]);
    } else if (w < 2) {
      tma_role<S>(a, maps, ctl, w, ring);
    } else {
      edge_role<S>(ctl, ring);
    }
  } else if (warp < kMma + 2) {
    mma_role<S>(ctl, warp - kMma, ring, q_smem, tmem);
  } else if (warp == kMma + 2) {
    q_role<S>(a, ctl, q_smem);
  } else {
    if (threadIdx.x % 32 == 0) walk_role(a, ctl);
    __syncwarp();
    if (blockIdx.x == 0)
      for (int b = threadIdx.x % 32; b <= list_len(a); b += 32) a.bases[b] = ctl.plan.bases[b];
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kMma) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
  if (ctl.abort_flag) lose_records<S::HD>(a, ctl.plan);
  // The launch after this one waits for both.  (By now the tensor memory is free: a CTA of the launch before this one may
  // still be waiting for it.)
  if (a.beside) pdl_wait();
}

template <class S>
cudaError_t launch(const ListArgs& a, cudaLaunchConfig_t cfg) {
  static_assert(S::kSmem + sizeof(Ctl) <= 227 * 1024, "shared memory");
  static std::atomic<bool> set[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev >= 64 || !set[dev].load(std::memory_order_relaxed))) {
    e = cudaFuncSetAttribute(tiles_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    if (e == cudaSuccess && dev < 64) set[dev].store(true, std::memory_order_relaxed);
  }
  if (e != cudaSuccess) return e;
  TileMaps maps{};
  if constexpr (!S::CODES)
    for (int i = a.n_own > 0 ? 0 : 1; i < (a.prefix_len > 0 ? 2 : 1); ++i) {
      const KvView& kv = a.kv[i];
      if (!encode_cache(&maps.k[i], kv.k, S::HD, kv.max_pos, kv.n_heads, kv.n_seq, kv.pos, kv.head, kv.seq) ||
          !encode_cache(&maps.v[i], kv.v, S::HD, kv.max_pos, kv.n_heads, kv.n_seq, kv.pos, kv.head, kv.seq))
        return cudaErrorInvalidValue;
    }
  cfg.gridDim = dim3(kTilesCtas);
  cfg.blockDim = dim3(S::kThreads);
  cfg.dynamicSmemBytes = S::kSmem;
  return cudaLaunchKernelEx(&cfg, tiles_kernel<S>, a, maps);
}

}  // namespace

cudaError_t launch_attn_tiles(int hd, bool codes, const ListArgs& a, cudaLaunchConfig_t cfg) {
  return hd == 64 ? (codes ? launch<Shape<64, true>>(a, cfg) : launch<Shape<64, false>>(a, cfg))
                  : (codes ? launch<Shape<128, true>>(a, cfg) : launch<Shape<128, false>>(a, cfg));
}

}  // namespace memspec
