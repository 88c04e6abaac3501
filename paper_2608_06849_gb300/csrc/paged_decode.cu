// Host side of the paged decode (paged_decode.cuh): its tensor map, its workspace and the
// choice of the kernel.
#include "paged_decode.cuh"

namespace aoh {

cudaError_t launch_paged_decode_f8_128(const PagedDecodeArgs& a, int num_sms, int cluster, cudaStream_t s);
cudaError_t launch_paged_decode_f8_64(const PagedDecodeArgs& a, int num_sms, int cluster, cudaStream_t s);
cudaError_t launch_paged_decode_bf16_128(const PagedDecodeArgs& a, int num_sms, int cluster, cudaStream_t s);
cudaError_t launch_paged_decode_bf16_64(const PagedDecodeArgs& a, int num_sms, int cluster, cudaStream_t s);

// 3D map over a pool as [page, K or V, head][row][D], box one block of up to 128 bytes a row,
// swizzled over that width.
bool make_pages_map(CUtensorMap* map, const PagePool& p) {
  auto fn = encode_fn();
  if (!fn) return false;
  const int es = p.form ? 1 : 2;
  const cuuint32_t width = p.form ? (cuuint32_t)p.D : 64;
  cuuint64_t dims[3] = {(cuuint64_t)p.D, (cuuint64_t)p.ps, (cuuint64_t)p.n_pages * 2 * p.Hkv};
  cuuint64_t strides[2] = {(cuuint64_t)p.D * es, (cuuint64_t)p.D * es * p.ps};
  cuuint32_t box[3] = {width, (cuuint32_t)p.ps, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(map, p.form ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, p.data, dims, strides, box,
            estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            width * es == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

size_t paged_state_floats(int num_sms, int D) { return (size_t)num_sms * 4 * pdec::state_floats(D); }

// CTAs of a cluster an item, or 0: all SMs in equal runs, by what they take in tenths of a
// microsecond beyond what both do, with sequences of at most a.max_len tokens: a tile of 64 KB
// 0.95 us on an SM whose neighbours leave it the bandwidth, 1.47 us on all SMs at once; joining
// an item's states through global memory 3.3 us, 5.5 in two levels. Measured, us a step in
// equal runs / on clusters (8-bit, 32/8 heads of 128): 1 x 4096 9.4 / 6.0, 4 x 8192 15.7 /
// 11.5, 8 streaming heads (S = 64, W = 2048) of 8 x 20000 13.1 / 8.9; bf16, 28/4 heads, half
// streaming, 1 x 4096 9.8 / 6.0; 16/1 heads, 8 x 8000 19.3 / 12.1, bf16 21.4 / 11.7.
static int cluster_size(const PagedDecodeArgs& a, int num_sms) {
  const CacheGeom& g = a.geom;
  const long long items = (long long)a.n_seqs * g.Hkv;
  const long long keys = 32768 / (g.D * (a.pool.form ? 1 : 2)), ring = (long long)g.S + g.W + 2 * a.pool.ps;
  const long long tr = (a.max_len + keys - 1) / keys, ts = ((a.max_len < ring ? a.max_len : ring) + keys - 1) / keys;
  const long long widest = g.n_r > 0 ? tr : ts, total = a.n_seqs * (g.n_r * tr + g.n_s * ts);
  const bool two_levels = widest * num_sms > pdec::kGroup * (total > num_sms ? total : num_sms);
  double best = 14.7 * (double)((total + num_sms - 1) / num_sms) + (two_levels ? 55 : 33);
  int pick = 0;
  for (int c = pdec::kClusterMost; c >= 2; c /= 2) {
    if (items > num_sms / c) continue;
    const double share = 14.7 * (double)(items * c) / num_sms, tile = share > 9.5 ? share : 9.5;
    const double cost = tile * (double)((widest + c - 1) / c);
    if (cost < best && items <= decode_tc_max_clusters(c)) {
      best = cost;
      pick = c;
    }
  }
  return pick;
}

cudaError_t launch_paged_decode(const PagedDecodeArgs& a, int num_sms, cudaStream_t s) {
  const int c = cluster_size(a, num_sms);
  if (a.pool.D == 128)
    return a.pool.form ? launch_paged_decode_f8_128(a, num_sms, c, s) : launch_paged_decode_bf16_128(a, num_sms, c, s);
  return a.pool.form ? launch_paged_decode_f8_64(a, num_sms, c, s) : launch_paged_decode_bf16_64(a, num_sms, c, s);
}

}  // namespace aoh
