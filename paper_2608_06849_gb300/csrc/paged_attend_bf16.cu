// Instances of the attention of chunks over pages of bf16 (paged_attend.cuh); a unit of its own, compiled
// beside the other.
#include "paged_attend.cuh"

namespace aoh {
cudaError_t launch_paged_attend_bf16(const PagedAttendArgs& a, const std::vector<uint64_t>& items, int split, bool is_short,
                                     int num_sms, cudaStream_t s) {
  return a.pool.D == 128 ? pf::launch_attend<false, 128>(a, items, split, is_short, num_sms, s)
                         : pf::launch_attend<false, 64>(a, items, split, is_short, num_sms, s);
}
}  // namespace aoh
