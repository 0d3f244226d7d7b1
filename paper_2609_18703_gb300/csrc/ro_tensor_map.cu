// ro_tensor_map.cu — TMA tensor maps of the model-step kernels' operands.
#include "ro_tcgen05.cuh"

namespace ro {

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeTiled encode_tiled() {
  static EncodeTiled f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) != cudaSuccess ||
        r != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      p = nullptr;
    }
    return (EncodeTiled)p;
  }();
  return f;
}
bool tile_map(CUtensorMap* m, int dtype, const void* p, int dims, const uint64_t* size, const uint64_t* stride,
              const uint32_t* box) {
  const EncodeTiled f = encode_tiled();
  if (!f) return false;
  cuuint64_t sz[5], st[5];
  cuuint32_t bx[5], el[5];
  for (int i = 0; i < dims; ++i) {
    sz[i] = size[i];
    bx[i] = box[i];
    el[i] = 1;
    if (i) st[i - 1] = stride[i] * 2;
  }
  return f(m, dtype == RO_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, (cuuint32_t)dims,
           const_cast<void*>(p), sz, st, bx, el, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool pool_map(CUtensorMap* m, const PagedArgs& c, const void* pool, int dtype, uint32_t box) {
  const uint64_t size[4] = {c.head_dim, c.page_size, c.n_heads, c.n_pages};
  const uint64_t stride[4] = {1, c.slot_stride, c.head_stride, c.page_stride};
  const uint32_t boxes[4] = {64, box, 1, 1};
  return tile_map(m, dtype, pool, 4, size, stride, boxes);
}

bool rows_map(CUtensorMap* m, const RowsArgs& r, uint32_t head_dim, uint32_t n_q_heads, int dtype, uint32_t heads,
              uint32_t toks) {
  const uint64_t size[3] = {head_dim, n_q_heads, r.n_tokens};
  const uint64_t stride[3] = {1, r.q_head, r.q_tok};
  const uint32_t boxes[3] = {64, heads, toks};
  return tile_map(m, dtype, r.q, 3, size, stride, boxes);
}

}  // namespace ro
