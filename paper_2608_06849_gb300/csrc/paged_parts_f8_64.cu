// Instances of the paged decode over parts of sequences for 8-bit pages and d_head 64; a unit of its own.
#include "paged_decode.cuh"

namespace aoh {
cudaError_t launch_paged_parts_f8_64(const PagedPartsArgs& a, int num_sms, int cluster, cudaStream_t s) {
  return pdec::launch_parts<64, true>(a, num_sms, cluster, s);
}
}  // namespace aoh
