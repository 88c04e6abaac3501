// Host side of the paged decode (paged_decode.cuh): its tensor map, its workspace and the
// choice of the kernel.
#include "paged_decode.cuh"

namespace aoh {

cudaError_t launch_paged_decode_f8_128(const PagedDecodeArgs& a, int num_sms, cudaStream_t s);
cudaError_t launch_paged_decode_f8_64(const PagedDecodeArgs& a, int num_sms, cudaStream_t s);
cudaError_t launch_paged_decode_bf16_128(const PagedDecodeArgs& a, int num_sms, cudaStream_t s);
cudaError_t launch_paged_decode_bf16_64(const PagedDecodeArgs& a, int num_sms, cudaStream_t s);

// 3D map over a pool as [page, K or V, head][row][D], box one block of up to 128 bytes a row,
// swizzled over that width.
bool make_pages_map(CUtensorMap* map, const PagePool& p) {
  auto fn = encode_fn();
  if (!fn) return false;
  const int es = p.form ? 1 : 2;
  const cuuint32_t width = p.form ? (cuuint32_t)p.D : 64;
  cuuint64_t dims[3] = {(cuuint64_t)p.D, (cuuint64_t)p.ps, (cuuint64_t)p.n_pages * 2 * p.Hkv};
  cuuint64_t strides[2] = {(cuuint64_t)p.D * es, (cuuint64_t)p.D * es * p.ps};
  cuuint32_t box[3] = {width, (cuuint32_t)p.ps, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(map, p.form ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, p.data, dims, strides, box,
            estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            width * es == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

size_t paged_state_floats(int num_sms, int D) { return (size_t)num_sms * 4 * pdec::state_floats(D); }

cudaError_t launch_paged_decode(const PagedDecodeArgs& a, int num_sms, cudaStream_t s) {
  if (a.pool.D == 128)
    return a.pool.form ? launch_paged_decode_f8_128(a, num_sms, s) : launch_paged_decode_bf16_128(a, num_sms, s);
  return a.pool.form ? launch_paged_decode_f8_64(a, num_sms, s) : launch_paged_decode_bf16_64(a, num_sms, s);
}

}  // namespace aoh
