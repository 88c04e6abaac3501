// The prefill calls of a cache whose items are short (prefill_short.cuh).
#include "prefill_short.cuh"

namespace aoh {
namespace {

using namespace pf;

template <int D, int CAP>
cudaError_t launch_short_cfg(const PrefillTcArgs& a, const std::vector<uint64_t>& items, int num_sms, cudaStream_t s) {
  using X = ShortCfg<D>;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = once_per_device(done, [] {
    return cudaFuncSetAttribute(prefill_short_kernel<PrefillTcArgs, D, CAP>, cudaFuncAttributeMaxDynamicSharedMemorySize, X::SMEM);
  });
  if (e != cudaSuccess) return e;
  const int n = (int)items.size();
  WorkList<CAP> wl;
  if (CAP > 0) memcpy(wl.item, items.data(), items.size() * sizeof(uint64_t));
  prefill_short_kernel<PrefillTcArgs, D, CAP><<<n < num_sms ? n : num_sms, kThreads, X::SMEM, s>>>(a, wl, n);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_prefill_short(const PrefillTcArgs& a, const std::vector<uint64_t>& items, int num_sms,
                                 cudaStream_t s) {
  const bool by_value = items.size() <= (size_t)kPrefillByValue;
  if (a.geom.D == 128)
    return by_value ? launch_short_cfg<128, kPrefillByValue>(a, items, num_sms, s)
                    : launch_short_cfg<128, 0>(a, items, num_sms, s);
  if (a.geom.D == 64)
    return by_value ? launch_short_cfg<64, kPrefillByValue>(a, items, num_sms, s)
                    : launch_short_cfg<64, 0>(a, items, num_sms, s);
  return cudaErrorInvalidValue;
}

}  // namespace aoh
