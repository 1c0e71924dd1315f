// Tensor maps of the paged pool (host side).
#pragma once

#include "tc_ptx.cuh"

namespace actkv {
namespace tc {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver entry point is looked up through the runtime, so the library does not link libcuda.
inline EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = []() -> EncodeTiledFn {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      return nullptr;
    return (EncodeTiledFn)p;
  }();
  return fn;
}

// The four-dimensional K map needs the slots of consecutive pages to continue at the slot stride.
inline bool pool_needs_5d(const actkv_pool_t* pool) { return pool->stride_page != (int64_t)pool->page_size * pool->stride_slot; }

inline bool make_kvmap(const actkv_pool_t* pool, int kv, CUtensorMap* kmap) {
  void* base = (char*)pool->base + (kv ? pool->stride_kv * 2 : 0);
  EncodeTiledFn enc = encode_fn();
  if (!enc) return false;
  // The K (or V) half of the pool.  Slot-major pages whose slots continue across pages: [layer][slot (page*16 + s)]
  // [head][dim], four dimensions (measured 13 % faster than five on the K stream).  Any other page layout
  // (head-major pages): [layer][page][head][slot][dim] with the caller's strides.  A box is one page of
  // one head, 64 dims: page_size rows of 128 B.
  CUresult res;
  if (!pool_needs_5d(pool)) {
    cuuint64_t dims[4] = {(cuuint64_t)pool->head_dim, (cuuint64_t)pool->n_kv_heads, (cuuint64_t)pool->n_pages * pool->page_size,
                          (cuuint64_t)pool->n_layers};
    cuuint64_t strides[3] = {(cuuint64_t)pool->stride_head * 2, (cuuint64_t)pool->stride_slot * 2,
                             (cuuint64_t)pool->stride_layer * 2};
    cuuint32_t box[4] = {64, 1, (cuuint32_t)pool->page_size, 1};
    cuuint32_t es[4] = {1, 1, 1, 1};
    res = enc(kmap, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, base, dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  } else {
    cuuint64_t dims[5] = {(cuuint64_t)pool->head_dim, (cuuint64_t)pool->page_size, (cuuint64_t)pool->n_kv_heads,
                          (cuuint64_t)pool->n_pages, (cuuint64_t)pool->n_layers};
    cuuint64_t strides[4] = {(cuuint64_t)pool->stride_slot * 2, (cuuint64_t)pool->stride_head * 2,
                             (cuuint64_t)pool->stride_page * 2, (cuuint64_t)pool->stride_layer * 2};
    cuuint32_t box[5] = {64, (cuuint32_t)pool->page_size, 1, 1, 1};
    cuuint32_t es[5] = {1, 1, 1, 1, 1};
    res = enc(kmap, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, base, dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  }
  return res == CUDA_SUCCESS;
}
inline bool make_kmap(const actkv_pool_t* pool, CUtensorMap* kmap) { return make_kvmap(pool, 0, kmap); }

}  // namespace tc
}  // namespace actkv
