// Tensor maps of a pool's codes.
#include "tensor.cuh"

namespace kvq {
namespace paged {

int make_pool_map(CUtensorMap* map, const void* codes, const Pool& pool, int head_dim) {
  using Encode = decltype(&cuTensorMapEncodeTiled);
  static std::atomic<Encode> cached{nullptr};
  Encode encode = cached.load(std::memory_order_acquire);
  if (!encode) {
    void* sym = nullptr;
    cudaDriverEntryPointQueryResult found;
    KVQ_CUDA_TRY(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &found));
    if (found != cudaDriverEntryPointSuccess || !sym) return record_cuda_error(cudaErrorSymbolNotFound);
    encode = reinterpret_cast<Encode>(sym);
    cached.store(encode, std::memory_order_release);
  }
  const cuuint64_t d = (cuuint64_t)head_dim, page = d * pool.page;
  const cuuint64_t dims[4] = {d, (cuuint64_t)pool.page, (cuuint64_t)pool.kv_heads, (cuuint64_t)pool.pages};
  const cuuint64_t strides[3] = {d, page, page * pool.kv_heads};
  const cuuint32_t box[4] = {(cuuint32_t)d, (cuuint32_t)pool.page, 1, 1}, steps[4] = {1, 1, 1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void*>(codes), dims, strides, box, steps,
                            CU_TENSOR_MAP_INTERLEAVE_NONE, head_dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? KVQ_OK : record_cuda_error(cudaErrorInvalidValue);
}

uint32_t wait_budget() { return attn_wait_budget(); }

}  // namespace paged
}  // namespace kvq
