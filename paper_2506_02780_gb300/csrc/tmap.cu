// Host-side TMA tensor-map encoding for libee's bf16 and 8-bit operands.  The driver
// entry point is looked up once through the runtime, so libee does not link
// libcuda directly.
#include <cuda.h>
#include <cudaTypedefs.h>

#include "block_mma.cuh"
#include "ee_common.cuh"

namespace ee {

static PFN_cuTensorMapEncodeTiled_v12000 get_encode() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
  if (!fn) {
    cudaDriverEntryPointQueryResult q;
    void* ptr = nullptr;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &ptr, 12000, cudaEnableDefault,
                                         &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      return nullptr;
    fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(ptr);
  }
  return fn;
}

bool encode_bf16_tmap(CUtensorMap* map, const void* base, int rank, const uint64_t* dims,
                      const uint64_t* strides_bytes, const uint32_t* box) {
  auto fn = get_encode();
  if (!fn || rank < 1 || rank > 5) return false;
  cuuint64_t d[5];
  cuuint64_t s[4];
  cuuint32_t bx[5];
  cuuint32_t es[5];
  for (int i = 0; i < rank; ++i) {
    d[i] = dims[i];
    bx[i] = box[i];
    es[i] = 1;
    if (i + 1 < rank) s[i] = strides_bytes[i];
  }
  CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void*>(base), d,
                  s, bx, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS;
}

static bool encode_2d(CUtensorMap* map, CUtensorMapDataType type, CUtensorMapSwizzle swizzle, const void* base, uint64_t cols,
                      uint64_t rows, uint64_t stride_bytes, uint32_t box_cols, uint32_t box_rows) {
  auto fn = get_encode();
  if (!fn) return false;
  const cuuint64_t d[2] = {cols, rows}, s[1] = {stride_bytes};
  const cuuint32_t bx[2] = {box_cols, box_rows}, es[2] = {1, 1};
  return fn(map, type, 2, const_cast<void*>(base), d, s, bx, es, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool encode_u8_tmap_2d(CUtensorMap* map, const void* base, uint64_t cols, uint64_t rows, uint64_t stride_bytes,
                       uint32_t box_cols, uint32_t box_rows) {
  return encode_2d(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, CU_TENSOR_MAP_SWIZZLE_128B, base, cols, rows, stride_bytes, box_cols,
                   box_rows);
}
bool encode_u32_tmap_2d(CUtensorMap* map, const void* base, uint64_t cols, uint64_t rows, uint64_t stride_bytes,
                        uint32_t box_cols, uint32_t box_rows) {
  return encode_2d(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, CU_TENSOR_MAP_SWIZZLE_NONE, base, cols, rows, stride_bytes, box_cols,
                   box_rows);
}

}  // namespace ee
