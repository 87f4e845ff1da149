// lora.cu - low-rank adapters of many requests beside a shared projection
// (memspec_op_lora): y[r] = base[r] + scale[a] * B[a] (A[a] x[r]), a = ids[r].
//
// Two launches: t[r][j] = A[a][j] . x[r] into the scratch (fp32), then the expansion.
#include <cuda_runtime.h>

#include <string>

#include "../../include/memspec_ops.h"
#include "internal.h"
#include "ptx.cuh"

namespace memspec {
namespace {

constexpr int kMaxLoraRows = 256;
constexpr int kMaxRank = 128;

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
};

__device__ __forceinline__ int rank_of(const LoraArgs& a, int id) {
  return a.ranks == nullptr ? a.rank : max(0, min(a.ranks[id], a.rank));
}

__global__ void __launch_bounds__(128) shrink_kernel(const __grid_constant__ LoraArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  const int row = blockIdx.x, j = blockIdx.y * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int id = a.ids[row];
  if (id < 0 || id >= a.n_adapters || j >= rank_of(a, id)) return;
  const bf16* x = a.x + row * a.ldx;
  const bf16* w = a.a + (static_cast<long long>(id) * a.rank + j) * a.k;
  float s = 0.f;
  for (int i = lane; i < a.k; i += 32) s += __bfloat162float(x[i]) * __bfloat162float(w[i]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane == 0) a.t[row * a.rank + j] = s;
}

__global__ void __launch_bounds__(128) expand_kernel(const __grid_constant__ LoraArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  const int row = blockIdx.x, c = blockIdx.y * 128 + threadIdx.x;
  if (c >= a.n) return;
  const int id = a.ids[row];
  float s = 0.f;
  if (id >= 0 && id < a.n_adapters) {
    const bf16* w = a.b + (static_cast<long long>(id) * a.n + c) * a.rank;
    const int rank = rank_of(a, id);
    for (int j = 0; j < rank; ++j) s += a.t[row * a.rank + j] * __bfloat162float(w[j]);
    if (a.scales != nullptr) s *= a.scales[id];
  }
  a.y[row * a.ldy + c] = (a.base != nullptr ? a.base[row * a.ld_base + c] : 0.f) + s;
}

cudaError_t launch_lora(const LoraArgs& a, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(128);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cfg.gridDim = dim3(a.rows, (a.rank + 3) / 4);
  const cudaError_t e = cudaLaunchKernelEx(&cfg, shrink_kernel, a);
  if (e != cudaSuccess) return e;
  cfg.gridDim = dim3(a.rows, (a.n + 127) / 128);
  return cudaLaunchKernelEx(&cfg, expand_kernel, a);
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
  const cudaError_t e = launch_lora(a, static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) {
    set_op_error(std::string("lora launch: ") + cudaGetErrorString(e));
    return MEMSPEC_ERR_CUDA;
  }
  return MEMSPEC_OK;
}

}  // extern "C"
