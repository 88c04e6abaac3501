// Launches of the packed prompt attention (prefill_packed.cuh).
#include "prefill_packed.cuh"

#include <string.h>

#include "prefill_short.cuh"
#include "prefill_tc.cuh"

namespace aoh {
namespace {

using namespace pf;

constexpr int kSmall = 640;  // items of a launch that copies 7 KB of arguments instead of 32

// `follows`: another launch of the same call comes before this one, whose items are
// independent of it: its CTAs start as that one's last run, and end after it.
template <class K, int CAP, class... More>
cudaError_t launch(K kernel, int smem, int grid, int cluster, bool follows, const PackedArgs& a, const uint64_t* items,
                   int n, cudaStream_t s, More... more) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  if (cluster > 1) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
    attr[cfg.numAttrs].val.clusterDim.x = cluster;
    attr[cfg.numAttrs].val.clusterDim.y = attr[cfg.numAttrs].val.clusterDim.z = 1;
    ++cfg.numAttrs;
  }
  if (follows) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[cfg.numAttrs].val.programmaticStreamSerializationAllowed = 1;
    ++cfg.numAttrs;
  }
  cfg.attrs = attr;
  WorkList<CAP> wl;
  memcpy(wl.item, items, n * sizeof(uint64_t));
  return cudaLaunchKernelEx(&cfg, kernel, a, wl, more...);
}

template <int D, bool PAIRS, int CAP>
cudaError_t launch_items(const PackedArgs& a, const uint64_t* items, int n, bool follows, cudaStream_t s) {
  auto kernel = prefill_tc_kernel<PackedArgs, D, PAIRS, CAP>;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = once_per_device(
      done, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, PfCfg<D>::SMEM); });
  if (e != cudaSuccess) return e;
  return launch<decltype(kernel), CAP>(kernel, PfCfg<D>::SMEM, n, PAIRS ? 2 : 1, follows, a, items, n, s);
}

template <int D>
cudaError_t launch_short(const PackedArgs& a, const uint64_t* items, int n, int num_sms, bool follows, cudaStream_t s) {
  auto kernel = prefill_short_kernel<PackedArgs, D, kPrefillByValue>;
  constexpr int smem = ShortCfg<D>::SMEM;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = once_per_device(
      done, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem); });
  if (e != cudaSuccess) return e;
  return launch<decltype(kernel), kPrefillByValue>(kernel, smem, n < num_sms ? n : num_sms, 1, follows, a, items, n, s,
                                                   n);
}

// The items travel as kernel arguments, at most kPrefillByValue a launch.
template <int D>
cudaError_t launch_d(const PackedArgs& a, const std::vector<uint64_t>& items, const std::vector<uint64_t>& pairs,
                     bool is_short, int num_sms, cudaStream_t s) {
  if (!pairs.empty())
    return launch_items<D, true, 2 * kPrefillSplitMost>(a, pairs.data(), (int)pairs.size(), false, s);
  const size_t n = items.size();
  if (n <= kSmall && !is_short) return launch_items<D, false, kSmall>(a, items.data(), (int)n, false, s);
  for (size_t i = 0; i < n; i += kPrefillByValue) {
    const int m = (int)(n - i < (size_t)kPrefillByValue ? n - i : (size_t)kPrefillByValue);
    const cudaError_t e = is_short ? launch_short<D>(a, items.data() + i, m, num_sms, i > 0, s)
                                   : launch_items<D, false, kPrefillByValue>(a, items.data() + i, m, i > 0, s);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

__global__ void upload_kernel(int4* dst, const __grid_constant__ PackedUpload u) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < u.n) dst[u.first + i] = u.seq[i];
}

}  // namespace

cudaError_t launch_packed_seqs(int4* table, const std::vector<int4>& seqs, cudaStream_t s) {
  for (size_t i = 0; i < seqs.size(); i += PackedUpload::kMost) {
    PackedUpload u;
    u.first = (int)i;
    u.n = (int)(seqs.size() - i < (size_t)PackedUpload::kMost ? seqs.size() - i : (size_t)PackedUpload::kMost);
    memcpy(u.seq, seqs.data() + i, u.n * sizeof(int4));
    upload_kernel<<<(u.n + 255) / 256, 256, 0, s>>>(table, u);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_prefill_packed(const PackedArgs& a, const std::vector<uint64_t>& items,
                                  const std::vector<uint64_t>& pairs, bool is_short, int num_sms, cudaStream_t s) {
  if (items.empty()) return cudaSuccess;
  if (a.geom.D == 128) return launch_d<128>(a, items, pairs, is_short, num_sms, s);
  if (a.geom.D == 64) return launch_d<64>(a, items, pairs, is_short, num_sms, s);
  return cudaErrorInvalidValue;
}

}  // namespace aoh
