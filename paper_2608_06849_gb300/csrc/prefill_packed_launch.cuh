// Launches of the prefill kernels on packed prompts, for both kinds of items.
#pragma once

#include <string.h>

#include "prefill_packed.cuh"
#include "prefill_short.cuh"
#include "prefill_tc.cuh"

namespace aoh {
namespace pf {

// items of a launch that copies 2 or 7 KB of arguments instead of 32
constexpr int kTiny = 64, kSmall = 640;

// The launch overlaps the kernel before it.
template <class A, class K, int CAP, class... More>
cudaError_t launch(K kernel, int smem, int grid, int cluster, const A& a, const uint64_t* items, int n, cudaStream_t s,
                   More... more) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(CallOf<A>::kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  if (cluster > 1) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
    attr[cfg.numAttrs].val.clusterDim.x = cluster;
    attr[cfg.numAttrs].val.clusterDim.y = attr[cfg.numAttrs].val.clusterDim.z = 1;
    ++cfg.numAttrs;
  }
  attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[cfg.numAttrs].val.programmaticStreamSerializationAllowed = 1;
  ++cfg.numAttrs;
  cfg.attrs = attr;
  WorkList<CAP> wl;
  memcpy(wl.item, items, n * sizeof(uint64_t));
  return cudaLaunchKernelEx(&cfg, kernel, a, wl, more...);
}

// each: CTAs of an entry (kSplit: its cluster).
template <class A, int D, int MODE, int CAP>
cudaError_t launch_items(const A& a, const uint64_t* items, int n, int each, cudaStream_t s) {
  auto kernel = prefill_tc_kernel<A, D, MODE, CAP>;
  constexpr int smem = PfCfg<D>::SMEM;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = once_per_device(done, [&] {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess && CallOf<A>::kF8) {
      // its warpgroups exchange registers: more than the block is launched with would wait forever
      cudaFuncAttributes at;
      e = cudaFuncGetAttributes(&at, kernel);
      if (e == cudaSuccess && at.numRegs != kExchanged) e = cudaErrorInvalidConfiguration;
    }
    if (e == cudaSuccess && MODE == kSplit)
      e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    return e;
  });
  if (e != cudaSuccess) return e;
  return launch<A, decltype(kernel), CAP>(kernel, smem, n * each, MODE == kPairs ? 2 : each, a, items, n, s);
}

template <class A, int D, int CAP = kPrefillByValue>
cudaError_t launch_short(const A& a, const uint64_t* items, int n, int num_sms, cudaStream_t s) {
  auto kernel = prefill_short_kernel<A, D, CAP>;
  constexpr int smem = ShortCfg<D>::SMEM;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = once_per_device(
      done, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem); });
  if (e != cudaSuccess) return e;
  return launch<A, decltype(kernel), CAP>(kernel, smem, n < num_sms ? n : num_sms, 1, a, items, n, s, n);
}

// The items travel as kernel arguments, at most kPrefillByValue a launch.
template <class A, int D>
cudaError_t launch_all(A a, const std::vector<uint64_t>& items, bool is_short, int num_sms, cudaStream_t s) {
  const size_t n = items.size();
  if (n <= kTiny && !is_short) return launch_items<A, D, kWhole, kTiny>(a, items.data(), (int)n, 1, s);
  if (n <= kSmall && !is_short) return launch_items<A, D, kWhole, kSmall>(a, items.data(), (int)n, 1, s);
  for (size_t i = 0; i < n; i += kPrefillByValue) {
    const int m = (int)(n - i < (size_t)kPrefillByValue ? n - i : (size_t)kPrefillByValue);
    a.follows = i > 0;
    const cudaError_t e = is_short ? launch_short<A, D>(a, items.data() + i, m, num_sms, s)
                                   : launch_items<A, D, kWhole, kPrefillByValue>(a, items.data() + i, m, 1, s);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace pf
}  // namespace aoh
