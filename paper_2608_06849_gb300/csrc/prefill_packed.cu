// Packed prompts in plain items, and the upload of their sequences (prefill_packed.cuh).
#include "prefill_packed_launch.cuh"

namespace aoh {
namespace {

using namespace pf;

template <int D>
cudaError_t launch_d(const PackedArgs& a, const std::vector<uint64_t>& items, const std::vector<uint64_t>& pairs,
                     bool is_short, int num_sms, cudaStream_t s) {
  if (!pairs.empty())
    return launch_items<PackedArgs, D, kPairs, 2 * kPrefillSplitMost>(a, pairs.data(), (int)pairs.size(), 1, s);
  return launch_all<PackedArgs, D>(a, items, is_short, num_sms, s);
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
