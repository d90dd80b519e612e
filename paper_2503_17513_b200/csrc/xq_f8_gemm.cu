// Which kernel a block-scaled E4M3 product runs in, and what the kernels' launchers share.
#include "xq_f8.h"
#include "xq_internal.h"

bool xq_f8_map_rows(CUtensorMap* map, const void* p, int rows, int pitch, int box_rows) {
  XqEncodeTiledFn enc = xq_encode_tiled_fn();
  if (!enc) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)pitch, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)pitch};
  const cuuint32_t box[2] = {128, (cuuint32_t)box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Above 128 tokens the weights are no longer the only traffic that counts: tiles of pairs of multiprocessors.
cudaError_t xq_f8_launch_gemm(const XqF8GemmArgs& a, cudaStream_t st) {
  return a.M > 128 ? xq_f8_launch_tile(a, 256, st) : xq_f8_launch_stream(a, st);
}
