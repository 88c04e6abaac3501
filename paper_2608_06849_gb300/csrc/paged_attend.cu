// The choice of the kernel of an attention over pages (paged_attend.cuh).
#include "internal.h"

namespace aoh {

cudaError_t launch_paged_attend_f8(const PagedAttendArgs& a, const std::vector<uint64_t>& items, int split, bool is_short,
                                   int num_sms, cudaStream_t s);
cudaError_t launch_paged_attend_bf16(const PagedAttendArgs& a, const std::vector<uint64_t>& items, int split, bool is_short,
                                int num_sms, cudaStream_t s);

cudaError_t launch_paged_attend(const PagedAttendArgs& a, const std::vector<uint64_t>& items, int split, bool is_short,
                                int num_sms, cudaStream_t s) {
  if (items.empty()) return cudaSuccess;
  return a.pool.form ? launch_paged_attend_f8(a, items, split, is_short, num_sms, s)
                     : launch_paged_attend_bf16(a, items, split, is_short, num_sms, s);
}

}  // namespace aoh
