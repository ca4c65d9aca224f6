// Tensor-map (TMA descriptor) helpers for the K/V cache, shared by the kernels
// that stream strips through shared memory.  Host side only.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <mutex>

namespace ngc {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// cuTensorMapEncodeTiled through the runtime's driver entry point lookup (no link against libcuda).
inline EncodeTiledFn encode_tiled_fn() {
  static EncodeTiledFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* sym = nullptr;
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &qres) == cudaSuccess &&
        qres == cudaDriverEntryPointSuccess)
      fn = (EncodeTiledFn)sym;
  });
  return fn;
}

// K or V of a bf16 cache with d = 128 (or 64) as a 3-D tensor (channel, row in plane, plane);
// box = 64 channels x `box_rows` rows, 128-byte swizzle.  A row of 128 channels
// is fetched as two boxes (x = 0 and x = 64).
inline bool make_kv_map(CUtensorMap* map, const void* base, int64_t rows, int planes, int box_rows, int d = 128) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)rows, (cuuint64_t)planes};
  cuuint64_t strides[2] = {(cuuint64_t)d * 2, (cuuint64_t)rows * d * 2};
  cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The same rows as a 4-D tensor (channel in its group of 64, row, group, plane), so that ONE load fetches all d channels
// of `box_rows` rows: groups one behind the other in shared memory, each 64 channels x box_rows rows.
inline bool make_strip_map(CUtensorMap* map, const void* base, int64_t rows, int planes, int box_rows, int d) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  cuuint64_t dims[4] = {64, (cuuint64_t)rows, (cuuint64_t)(d / 64), (cuuint64_t)planes};
  cuuint64_t strides[3] = {(cuuint64_t)d * 2, 128, (cuuint64_t)rows * d * 2};
  cuuint32_t box[4] = {64, (cuuint32_t)box_rows, (cuuint32_t)(d / 64), 1};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A bf16 matrix of `rows` rows of 128 (or d = 64) channels as a 2-D tensor (channel, row); box = 64 channels x `box_rows`
// rows, 128-byte swizzle.  box_rows = 1 is the shape the TMA row gather (tile::gather4) takes.
inline bool make_rows_map(CUtensorMap* map, const void* base, int64_t rows, int box_rows, int d = 128) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn || rows <= 0 || rows > 0x7fffffffLL) return false;
  cuuint64_t dims[2] = {(cuuint64_t)d, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)d * 2};
  cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A row-major matrix of `rows` rows of 128 elements (bf16 or fp32) as a 2-D tensor for TMA stores of 32-column,
// `box_rows`-row boxes; the shared-memory side uses the swizzle whose span equals the box's row (64 bytes for bf16,
// 128 bytes for fp32), so that a thread per row can fill the box without bank conflicts.
inline bool make_out_map(CUtensorMap* map, void* base, bool bf16, int64_t rows, int box_rows) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn || rows <= 0 || rows > 0x7fffffffLL) return false;
  const cuuint64_t elt = bf16 ? 2 : 4;
  cuuint64_t dims[2] = {128, (cuuint64_t)rows};
  cuuint64_t strides[1] = {128 * elt};
  cuuint32_t box[2] = {32, (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1, 1};
  return fn(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, base, dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, bf16 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace ngc
