// Host-side checks that the decoder-layer operators share.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/gmgop.h"

namespace gop {

inline bool cache_ok(const op_cache_t* c) {
  if (!c || !c->pool || !c->table || !c->lens || !c->refs || !c->status) return false;
  if (c->dtype != GMG_OP_BF16 && c->dtype != GMG_OP_F16) return false;
  if (c->n_pages < 1 || c->n_layers < 1 || c->n_kv_heads < 1 || c->n_seq < 1 || c->max_pages < 1 ||
      c->max_pages > (1 << 22))
    return false;
  if (c->page_tokens < 8 || c->page_tokens > 256 || (c->page_tokens & (c->page_tokens - 1))) return false;
  if (c->head_dim < 8 || c->head_dim > 128 || c->head_dim % 8) return false;
  return (reinterpret_cast<uintptr_t>(c->pool) & 15) == 0;
}

// A page in 8 bits: codes [n_layers][2][n_kv_heads][page_tokens][head_dim], then fp32 scales
// [n_layers][2][n_kv_heads][page_tokens / 16], up to a whole 128 bytes.
constexpr int kScaleTokens = 16;
inline int64_t page8_scales(const op_cache_t& c) {   // where they begin
  return int64_t(c.n_layers) * 2 * c.n_kv_heads * c.page_tokens * c.head_dim;
}
inline int64_t page8_bytes(const op_cache_t& c) {
  return (page8_scales(c) + int64_t(c.n_layers) * 2 * c.n_kv_heads * (c.page_tokens / kScaleTokens) * 4 + 127) / 128 * 128;
}
inline bool cache8_ok(const op_cache_t* c) {
  if (!c || c->dtype != GMG_OP_E4M3 || c->page_tokens < kScaleTokens || c->head_dim % 16) return false;
  op_cache_t as = *c;
  as.dtype = GMG_OP_BF16;
  return cache_ok(&as);
}

// Whether every row of a tensor with these strides (in elements of e bytes) starts on 16 bytes.
inline bool aligned(const void* p, int64_t s0, int64_t s1, int e) {
  return ((reinterpret_cast<uintptr_t>(p) | uintptr_t(s0 * e) | uintptr_t(s1 * e)) & 15) == 0;
}

// Lets a kernel have `bytes` of dynamic shared memory, and its SM give all it can to shared
// memory (left to itself the driver may leave room for one block where two would fit).
template <class K>
bool allow_smem(K kernel, int bytes) {
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess &&
         cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared) ==
             cudaSuccess;
}

// The driver's encoder of tensor maps, looked up once; NULL if it has none.
using MapEncoder = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline MapEncoder map_encoder() {
  static const MapEncoder found = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q);
    return e == cudaSuccess && q == cudaDriverEntryPointSuccess ? reinterpret_cast<MapEncoder>(f) : nullptr;
  }();
  return found;
}

// A map of 16-bit elements whose boxes are 64 elements (128 bytes) wide, in the 128-byte
// swizzle; what lies outside reads as zero.  stride: in elements, of dimensions 1 .. rank - 1.
inline bool make_map(CUtensorMap* m, int32_t dtype, int rank, const void* base, const int64_t* size,
                     const int64_t* stride, const int32_t* box) {
  const MapEncoder encode = map_encoder();
  if (!encode) return false;
  cuuint64_t dims[5], bytes[5];
  cuuint32_t boxes[5], step[5];
  for (int i = 0; i < rank; ++i) {
    dims[i] = (cuuint64_t)size[i];
    boxes[i] = (cuuint32_t)box[i];
    step[i] = 1;
    if (i > 0) bytes[i - 1] = (cuuint64_t)stride[i - 1] * 2;
  }
  return encode(m, dtype == GMG_OP_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                (cuuint32_t)rank, const_cast<void*>(base), dims, bytes, boxes, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The same for bytes, in boxes of 64 or 128 bytes and their swizzle.
inline bool make_map8(CUtensorMap* m, int rank, const void* base, const int64_t* size, const int64_t* stride,
                      const int32_t* box) {
  const MapEncoder encode = map_encoder();
  if (!encode) return false;
  cuuint64_t dims[5], bytes[5];
  cuuint32_t boxes[5], step[5];
  for (int i = 0; i < rank; ++i) {
    dims[i] = (cuuint64_t)size[i];
    boxes[i] = (cuuint32_t)box[i];
    step[i] = 1;
    if (i > 0) bytes[i - 1] = (cuuint64_t)stride[i - 1];
  }
  return encode(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, (cuuint32_t)rank, const_cast<void*>(base), dims, bytes, boxes, step,
                CU_TENSOR_MAP_INTERLEAVE_NONE, box[0] == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace gop
