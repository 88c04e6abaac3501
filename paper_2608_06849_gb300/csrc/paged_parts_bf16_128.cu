// Instances of the paged decode over parts of sequences for bf16 pages and d_head 128; a unit of its own.
#include "paged_decode.cuh"

namespace aoh {
cudaError_t launch_paged_parts_bf16_128(const PagedPartsArgs& a, int num_sms, int cluster, cudaStream_t s) {
  return pdec::launch_parts<128, false>(a, num_sms, cluster, s);
}
}  // namespace aoh
