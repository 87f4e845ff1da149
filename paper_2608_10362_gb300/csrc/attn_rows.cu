// attn_rows.cu - attention of a batch's rows over a layer's cache (memspec_op_attention).
//
// A unit is the query vectors (rows x heads of a group) of one sequence and one head of k and
// v, up to VT of them, against all keys: S^T = K Q^T, P = exp2(S^T - m), O^T += V^T P^T with
// mma.sync (m16n8k16, fp32 sums), keys and then the vectors' elements as M, query vectors as N.
// Few vectors per key: the bound is reading K and V once, so work is cut by keys: all units'
// tiles of 128 keys, one after another, are split evenly over the CTAs (whatever the lengths
// are; every CTA works its share out from the lengths itself), a warp takes 16 keys at a time
// through a cp.async ring of its own.  What a unit's CTAs found is joined by a second launch.
// 64 sequences of up to 32768 positions, 8 heads of codes: 267 us, 6.8 TB/s (the measured copy's 6.8); one row of
// 32 heads over 2048 positions 12.7 us of which 5 are reading, the others two launches' beginnings and the join.  The form for
// 16 vectors of 128 over codes spills 88 bytes a thread at two CTAs an SM.
//
// Scores are kept in units of log2: z = log2(e) scale q.k.  The running maximum m of a vector is
// taken again only when a score passes what Weights allows, so that O is rarely rescaled.
// Codes: exact in fp16 (1024 + 128 + code by one byte permutation, less 1152).  K's scale
// multiplies the score, V's is added to it as a logarithm: weights are w' = p * scale_v with a
// maximum of their own kind, and the sum of p is that of w' / scale_v; so no range of scales
// overflows fp16.
#include <algorithm>
#include <atomic>

#include "attn_plan.cuh"
#include "ptx.cuh"

namespace memspec {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
static_assert(kTile == 16 * kWarps, "a turn of a CTA's warps is a tile");

template <int HD_, bool CODES_, int NT_>
struct Shape {
  static constexpr int HD = HD_, NT = NT_, VT = 8 * NT_;
  static constexpr bool CODES = CODES_;
  static constexpr int kRowBytes = HD * (CODES ? 1 : 2);
  static constexpr int kStage = 2 * 16 * kRowBytes + (CODES ? 128 : 0);
  static constexpr int kQBytes = VT * HD * 2;
  static constexpr int kFixed = sizeof(Plan) + kQBytes + VT * 16;
  // CTAs of an SM: codes take more instructions a byte, and more warps hide them (64 long sequences: 287 us, one: 332)
  static constexpr int kPerSm = CODES ? 2 : 1;
  static constexpr int kBudget = (kPerSm == 2 ? 113 : 226) * 1024 - kFixed;
  static constexpr int kDepth = std::min(8, kBudget / (kWarps * kStage));
  static constexpr int kRing = kWarps * kDepth * kStage;
  static constexpr int kSmem = kFixed + kRing;
  static_assert(kFixed % 128 == 0 && kDepth >= 2 && kSmem <= (kPerSm == 2 ? 113 : 227) * 1024, "shared memory");
  static_assert(kRing >= VT * (kWarps * (HD * 4 + 8) + 8), "the warps' sums lie where the ring was");
};

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

template <class S>
struct Smem {
  Plan* plan;
  char* q;
  Sight* sight;     // [VT]
  float* q_scale;   // [VT]
  int* q_exp;       // [VT]
  char* ring;
  __device__ explicit Smem(char* p) {
    plan = reinterpret_cast<Plan*>(p);
    q = p + sizeof(Plan);
    sight = reinterpret_cast<Sight*>(q + S::kQBytes);
    q_scale = reinterpret_cast<float*>(sight + S::VT);
    q_exp = reinterpret_cast<int*>(q_scale + S::VT);
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
                                     uint32_t stage, int kb, int end, int lane) {
  constexpr int C = S::kRowBytes / 16, R = 32 / C;   // chunks of a row, rows at a time
  int key = kb + lane / C;
  const int c = lane % C;
  const long long at = key * kv.pos + c * 16, step = kv.pos * R;
  k += at;
  v += at;
#pragma unroll
  for (int i = 0; i < 16 / R; ++i) {
    const int row = lane / C + i * R;
    const bool on = key < end;
    const uint32_t dst = stage + row * S::kRowBytes;
    cp_async16(dst + k_chunk<S>(row, c) * 16, on ? k : kv.k, on);
    cp_async16(dst + 16 * S::kRowBytes + v_chunk<S>(row, c) * 16, on ? v : kv.v, on);
    key += R;
    k += step;
    v += step;
  }
  if constexpr (S::CODES) {
    const int s_key = kb + (lane & 15);
    const bool on = s_key < end;
    cp_async4(stage + 32 * S::kRowBytes + lane * 4, (lane < 16 ? ks : vs) + (on ? s_key * kv.s_pos : 0), on);
  }
}

// scale * 2^e * k_s where scale * 2^e, which a vector is held with, is not a normal number: the product may be one.
__device__ __noinline__ float far_factor(float scale, int e, float k_s) {
  int scale_e;
  const float fraction = frexpf(scale, &scale_e);
  const float by = ldexpf(fraction * (k_s * 0x1p-32f), scale_e + e + 32);
  return isinf(by) && k_s <= FLT_MAX ? copysignf(FLT_MAX, by) : by;   // (it meets products of 0)
}

template <class S>
__global__ void __launch_bounds__(kThreads, S::kPerSm) rows_kernel(const __grid_constant__ ListArgs a) {
  constexpr int HD = S::HD, NT = S::NT, VT = S::VT, KS = HD / 16, MT = HD / 16;
  constexpr bool CODES = S::CODES;
  typedef Walk<RowUnits<VT>> Stretches;
  extern __shared__ __align__(128) char smem_raw[];
  const Smem<S> sm(smem_raw);
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, g = lane >> 2, t = lane & 3;
  if (!a.beside) pdl_wait();
  pdl_launch_dependents();
  make_plan<RowUnits<VT>, kThreads>(a, *sm.plan);
  if (blockIdx.x == 0)
    for (int b = tid; b <= list_len(a); b += kThreads) a.bases[b] = sm.plan->bases[b];
  const uint32_t ring = smem_addr(sm.ring) + warp * S::kDepth * S::kStage, q_smem = smem_addr(sm.q);

  Stretches walk(a, *sm.plan);
  Stretch u;
#pragma unroll 1
  while (walk.next(u)) {
    const KvView& kv = a.kv[u.own ? 0 : 1];
    const int end = u.end();
    const int seq = u.own ? u.b : 0;
    const char* k = kv.k + seq * kv.seq + u.head * kv.head;
    const char* v = kv.v + seq * kv.seq + u.head * kv.head;
    const float* ks = CODES ? kv.k_scale + seq * kv.s_seq + u.head * kv.s_head : nullptr;
    const float* vs = CODES ? kv.v_scale + seq * kv.s_seq + u.head * kv.s_head : nullptr;
    const int kb0 = u.t0 * kTile + warp * 16;
    // the stages ahead of key kb's, one more in every turn
    int ahead = kb0, to = 0;
    auto fill_next = [&] {
      if (ahead < end) fill<S>(kv, k, v, ks, vs, ring + to * S::kStage, ahead, end, lane);
      cp_commit();
      ahead += kTile;
      to = to + 1 == S::kDepth ? 0 : to + 1;
    };
    // the unit's vectors first, a chunk a thread
    constexpr int C = HD / 8;
    static_assert(VT * C <= kThreads, "a thread per chunk");
    const int q_vec = tid / C, q_c = tid % C, id = u.unit * VT + q_vec;
    const uint32_t q_at = q_vec * HD * 2 + (q_c ^ (q_vec & 7)) * 16;
    if (tid < VT * C) {
      const int j = vector_row(a, id);
      const bool on = id < u.vecs;
      cp_async16(q_smem + q_at, on ? a.q + (u.row0 + j) * a.ldq + (u.head * a.group + id - j * a.group) * HD + q_c * 8 : a.q, on);
    }
    cp_commit();
#pragma unroll 1
    for (int d = 0; d < S::kDepth - 1; ++d) fill_next();
    if (tid < VT) sm.sight[tid] = sight_of(a, u, u.unit * VT + tid);
    cp_wait<S::kDepth - 1>();
    if constexpr (CODES) {   // to fp16, and in the order of the fragments
      if (tid < VT * C) {    // (whole warps, and a vector's threads are of one)
        const uint4 in = *reinterpret_cast<const uint4*>(sm.q + q_at);
        const uint32_t w[4] = {in.x, in.y, in.z, in.w};
        const int e = exponent_of_lanes<C>(in);
        const float up = power(-e);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          // a lane's word of four codes is one step's pairs k = 2t, 2t + 1 and 2t + 8, 2t + 9
          const int hd = q_c * 8 + j * 2, to = hd / 64 * 64 + hd % 16 / 4 * 16 + hd % 64 / 16 * 2 + hd % 4 / 2 * 8;
          *reinterpret_cast<uint32_t*>(sm.q + q_vec * HD * 2 + (to / 8 ^ (q_vec & 7)) * 16 + to % 8 * 2) = scaled_f16(w[j], up);
        }
        if (q_c == 0) sm.q_scale[q_vec] = a.scale * power(e), sm.q_exp[q_vec] = e;
      }
    }
    __syncthreads();
    float scale[NT][2];   // of the lane's vectors
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 2; ++i) scale[nt][i] = CODES ? sm.q_scale[nt * 8 + 2 * t + i] : a.scale;
    bool far = false;
    if (CODES && a.scale != 0.f) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 2; ++i) far |= !(fabsf(scale[nt][i]) >= FLT_MIN && fabsf(scale[nt][i]) <= FLT_MAX);
      far = __any_sync(~0u, far);
    }
    uint32_t qf[NT][KS][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < KS; i += 2) {
        uint32_t r[4];
        ldsm4(r, q_smem + (nt * 8 + (lane & 7)) * HD * 2 + ((i * 2 + (lane >> 3)) ^ (lane & 7)) * 16);
        qf[nt][i][0] = r[0], qf[nt][i][1] = r[1], qf[nt][i + 1][0] = r[2], qf[nt][i + 1][1] = r[3];
      }

    // ---- the keys
    float o[MT][NT][4] = {}, m[NT][2], l[NT][2] = {};
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) m[nt][0] = m[nt][1] = kStart;
    int slot = 0;
#pragma unroll 1
    for (int kb = kb0; kb < end; kb += kTile) {
      fill_next();
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
              mma<true>(z[nt], f[0], qf[nt][4 * h + p][0], qf[nt][4 * h + p][1]);
              mma<true>(z[nt], f[1], qf[nt][4 * h + p + 1][0], qf[nt][4 * h + p + 1][1]);
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
            mma<false>(z[nt], f[0], qf[nt][ks][0], qf[nt][ks][1]);
            mma<false>(z[nt], f[1], qf[nt][ks + 1][0], qf[nt][ks + 1][1]);
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
          const float lv = __log2f(v_s);
          rv[i] = __frcp_rn(v_s);
          if (isnan(rv[i])) rv[i] = 0.f;   // the weight is a NaN already where it counts
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float by[2] = {k_s * scale[nt][0], k_s * scale[nt][1]};
            if (far) {
#pragma unroll
              for (int j = 0; j < 2; ++j) by[j] = far_factor(a.scale, sm.q_exp[nt * 8 + 2 * t + j], k_s);
            }
            z[nt][2 * i] = fmaf(z[nt][2 * i], by[0], lv);
            z[nt][2 * i + 1] = fmaf(z[nt][2 * i + 1], by[1], lv);
          }
        }
      } else {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 4; ++i) z[nt][i] *= a.scale;
      }
      const bool edge = kb + 16 > end || kb + 15 >= u.first;
      if (edge) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = kb + g + (i >> 1) * 8;
            const Sight s = sm.sight[nt * 8 + 2 * t + (i & 1)];
            if (key >= end || !sees(s, u.first, key)) z[nt][i] = -INFINITY;
          }
      }
      bool above = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 2; ++i) above |= fmaxf(z[nt][i], z[nt][2 + i]) - m[nt][i] > Weights<CODES>::kAbove;
      if (__any_sync(~0u, above)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float top = fmaxf(z[nt][i], z[nt][2 + i]);
#pragma unroll
            for (int d = 4; d < 32; d *= 2) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
            const float now = top - m[nt][i] > Weights<CODES>::kAbove ? top - Weights<CODES>::kBelow : m[nt][i], by = ex2(m[nt][i] - now);
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
                const int key = kb + 2 * t + 8 * i;
                keep[i] = (key < end && sees(s, u.first, key) ? 0xffffu : 0u) |
                          (key + 1 < end && sees(s, u.first, key + 1) ? 0xffff0000u : 0u);
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

    // ---- the warps' sums into one
    cp_wait<0>();
    __syncthreads();
    float* part = reinterpret_cast<float*>(sm.ring);                        // [warp][VT][HD]
    float2* ml = reinterpret_cast<float2*>(part + kWarps * VT * HD);        // [warp][VT]
    float2* all = ml + kWarps * VT;                                         // [VT]
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int d = 4; d < 32; d *= 2) l[nt][i] += __shfl_xor_sync(~0u, l[nt][i], d);
        if (g == 0) ml[warp * VT + nt * 8 + 2 * t + i] = make_float2(m[nt][i], l[nt][i]);
      }
    __syncthreads();
    auto top_of_warps = [&](int vec) {
      float top = kStart;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float x = ml[w * VT + vec].x;
        top = x > top || isnan(x) ? x : top;
      }
      return top;
    };
    if (tid < VT) {
      const float top = top_of_warps(tid);
      float den = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) den = fmaf(ex2(ml[w * VT + tid].x - top), ml[w * VT + tid].y, den);
      all[tid] = make_float2(top, den);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int vec = nt * 8 + 2 * t + i;
        const float by = ex2(m[nt][i] - top_of_warps(vec));
        float* to = part + (warp * VT + vec) * HD;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          // elements as the fragments have them, turned by the vector so that lanes meet no bank twice
          if constexpr (CODES)
            *reinterpret_cast<float2*>(to + ((mt * 16 + 2 * g) ^ t * 8)) =
                make_float2(o[mt][nt][i] * by, o[mt][nt][2 + i] * by);
          else
            to[(mt * 16 + g) ^ t * 8] = o[mt][nt][i] * by, to[(mt * 16 + g + 8) ^ t * 8] = o[mt][nt][2 + i] * by;
        }
      }
    __syncthreads();
    float* const rec0 = u.whole() ? a.full[u.own ? 0 : 1]
                                  : a.slots + (2 * static_cast<long long>(blockIdx.x) + (u.t0 == 0)) * VT * kRecord<HD>;
    for (int i = tid; i < VT * HD / 4; i += kThreads) {
      const int vec = i / (HD / 4), e = i % (HD / 4) * 4, id = u.unit * VT + vec;
      if (id >= u.vecs) continue;
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float4 x = *reinterpret_cast<const float4*>(part + (w * VT + vec) * HD + (e ^ (vec >> 1 & 3) * 8));
        sum.x += x.x, sum.y += x.y, sum.z += x.z, sum.w += x.w;
      }
      const float2 md = all[vec];
      const long long row = u.row0 + id / a.group;
      const int head = u.head * a.group + id % a.group;
      if (u.whole() && a.out != nullptr) {
        const float by = md.y == 0.f ? 0.f : 1.f / md.y;
        *reinterpret_cast<uint2*>(a.out + row * a.ldo + head * HD + e) =
            make_uint2(pack_bf16(sum.x * by, sum.y * by), pack_bf16(sum.z * by, sum.w * by));
        continue;
      }
      float* rec = rec0 + (u.whole() ? row * a.group * a.kv_heads + head : vec) * kRecord<HD>;
      *reinterpret_cast<float4*>(rec + e) = sum;
      if (e == 0) rec[HD] = md.x, rec[HD + 1] = md.y;
    }
    __syncthreads();
  }
  if (a.beside) pdl_wait();   // the launch after this one waits for both
}

template <class S>
cudaError_t launch(const ListArgs& a, cudaLaunchConfig_t cfg) {
  static std::atomic<bool> set[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev >= 64 || !set[dev].load(std::memory_order_relaxed))) {
    e = cudaFuncSetAttribute(rows_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    if (e == cudaSuccess && dev < 64) set[dev].store(true, std::memory_order_relaxed);
  }
  if (e != cudaSuccess) return e;
  cfg.gridDim = dim3(152 * S::kPerSm);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = S::kSmem;
  return cudaLaunchKernelEx(&cfg, rows_kernel<S>, a);
}
template <int HD, bool CODES>
cudaError_t launch_nt(int nt, const ListArgs& a, const cudaLaunchConfig_t& cfg) {
  return nt == 1 ? launch<Shape<HD, CODES, 1>>(a, cfg) : launch<Shape<HD, CODES, 2>>(a, cfg);
}

}  // namespace

int rows_ctas(bool codes) { return 152 * (codes ? Shape<128, true, 2>::kPerSm : Shape<128, false, 2>::kPerSm); }

cudaError_t launch_attn_rows(int hd, bool codes, int nt, const ListArgs& a, cudaLaunchConfig_t cfg) {
  return hd == 64 ? (codes ? launch_nt<64, true>(nt, a, cfg) : launch_nt<64, false>(nt, a, cfg))
                  : (codes ? launch_nt<128, true>(nt, a, cfg) : launch_nt<128, false>(nt, a, cfg));
}

}  // namespace memspec
