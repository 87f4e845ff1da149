// cache_map.cu - the tensor map of a caller's cache (attn_tiles.cu).
#include <cuda.h>
#include <cuda_runtime.h>

#include <mutex>

#include "kv.cuh"

namespace memspec {

namespace {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeTiledFn>(p);
  });
  return fn;
}

}  // namespace

bool encode_cache(CUtensorMap* map, const void* base, int hd, int positions, int heads, int seqs, long long pos,
                  long long head, long long seq) {
  const EncodeTiledFn fn = encode_fn();
  if (fn == nullptr) return false;
  auto dim = [](int n, long long stride) { return static_cast<cuuint64_t>(stride == 0 ? 1 : n); };
  auto bytes = [](long long stride) { return static_cast<cuuint64_t>(stride == 0 ? 128 : stride); };
  cuuint64_t dims[5] = {64, dim(positions, pos), static_cast<cuuint64_t>(hd / 64), dim(heads, head), dim(seqs, seq)};
  cuuint64_t strides[4] = {bytes(pos), 128, bytes(head), bytes(seq)};
  cuuint32_t box[5] = {64, 128, static_cast<cuuint32_t>(hd / 64), 1, 1};
  cuuint32_t estr[5] = {1, 1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace memspec
