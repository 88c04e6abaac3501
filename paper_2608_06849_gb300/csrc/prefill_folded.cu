// Packed prompts in folded items (prefill_packed.cuh).
#include "prefill_packed_launch.cuh"

namespace aoh {
namespace {

using namespace pf;

template <int D>
cudaError_t launch_d(const FoldedArgs& a, const std::vector<uint64_t>& items, int split, bool is_short, int num_sms,
                     cudaStream_t s) {
  if (split > 1)
    return launch_items<FoldedArgs, D, kSplit, kPrefillSplitMost>(a, items.data(), (int)items.size(), split, s);
  return launch_all<FoldedArgs, D>(a, items, is_short, num_sms, s);
}

}  // namespace

cudaError_t launch_prefill_folded(const FoldedArgs& a, const std::vector<uint64_t>& items, int split, bool is_short,
                                  int num_sms, cudaStream_t s) {
  if (items.empty()) return cudaSuccess;
  if (a.geom.D == 128) return launch_d<128>(a, items, split, is_short, num_sms, s);
  if (a.geom.D == 64) return launch_d<64>(a, items, split, is_short, num_sms, s);
  return cudaErrorInvalidValue;
}

}  // namespace aoh
