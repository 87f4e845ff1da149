// kv.cuh - what the cache and attention operators (kv_append.cu, attn_*.cu) share: a
// layer's keys and values as the caller laid them out, which rows of a call belong to which
// sequence, and their checks.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/memspec_ops.h"
#include "internal.h"

namespace memspec {

constexpr int kMaxSeqs = 1024;        // sequences of one call
constexpr int kMaxCallRows = 65535;   // rows of one call
// A vector's scale is at least this, so that 1 / scale and sums of it stay within fp32
constexpr float kSmallestScale = 0x1p-64f;

// Keys and values of one layer; strides in bytes, those of the scales in floats.
struct KvView {
  char* k;
  char* v;
  float* k_scale;   // nullptr: bf16
  float* v_scale;
  long long seq, head, pos;
  long long s_seq, s_head, s_pos;
  int n_seq, n_heads, max_pos;
};

// The rows of sequence b: starts[b] .. starts[b + 1] - 1, at the end of its lens[b] positions.
// What the device arrays hold cannot be checked beforehand: rows outside the call do not count.
struct SeqRows {
  int row0, n, len;
};
__device__ __forceinline__ SeqRows seq_rows(const int* starts, const int* lens, int b, int rows) {
  const int r0 = min(max(starts[b], 0), rows), r1 = min(max(starts[b + 1], r0), rows);
  return {r0, r1 - r0, lens[b]};
}

// The sequence that a row belongs to (of several, where starts do not ascend, the first), -1: none.  All
// threads call it.
__device__ __forceinline__ int find_sequence(const int* starts, const int* lens, int n_seq, int rows, int row, int* shared) {
  if (threadIdx.x == 0) *shared = n_seq;
  __syncthreads();
  for (int b = threadIdx.x; b < n_seq; b += blockDim.x) {
    const SeqRows s = seq_rows(starts, lens, b, rows);
    if (row >= s.row0 && row < s.row0 + s.n) atomicMin(shared, b);
  }
  __syncthreads();
  return *shared < n_seq ? *shared : -1;
}

// Why `kv` cannot be used, or nullptr.
const char* kv_problem(const memspec_kv* kv, bool write);
KvView kv_view(const memspec_kv* kv);
const char* batch_problem(const memspec_batch* b, const memspec_kv* kv);

// Tensor map of a bf16 cache of a caller's strides (bytes; 0: one place), in boxes of 128 positions by all of hd: 64 column
// halves one after the other, each with the 128-byte swizzle (cache_map.cu).
bool encode_cache(CUtensorMap* map, const void* base, int hd, int positions, int heads, int seqs, long long pos,
                  long long head, long long seq);

}  // namespace memspec
