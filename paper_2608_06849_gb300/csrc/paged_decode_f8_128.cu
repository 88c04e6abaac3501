// Instances of the paged decode for 8-bit pages and d_head 128; a unit of its own, compiled beside the others.
#include "paged_decode.cuh"

namespace aoh {
cudaError_t launch_paged_decode_f8_128(const PagedDecodeArgs& a, int num_sms, int cluster, cudaStream_t s) {
  return pdec::launch_heads<128, true>(a, num_sms, cluster, s);
}
}  // namespace aoh
