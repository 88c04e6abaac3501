// The prefill calls of a cache (prefill_tc.cuh): tensor maps and launches.
#include "prefill_tc.cuh"

namespace aoh {

using namespace pf;

PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
  if (!fn) {
    cudaDriverEntryPointQueryResult q;
    void* p = nullptr;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) ==
            cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
  }
  return fn;
}

bool make_rows_map(CUtensorMap* map, const void* base, int B, long long T, int H, int D, long long stride, int rows,
                   int heads) {
  auto fn = encode_fn();
  if (!fn) return false;
  if (stride == 0) stride = (long long)H * D;
  cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)H, (cuuint64_t)T, (cuuint64_t)B};
  cuuint64_t strides[3] = {(cuuint64_t)D * 2, (cuuint64_t)stride * 2, (cuuint64_t)T * stride * 2};
  cuuint32_t box[4] = {64, (cuuint32_t)heads, (cuuint32_t)rows, 1};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, estr,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS;
}

namespace {

constexpr int kSmall = 640;  // items of a launch that copies 5 KB of arguments instead of 30

template <int D, int MODE, int CAP>
cudaError_t launch_cfg(const PrefillTcArgs& a, const std::vector<uint64_t>& items, cudaStream_t s) {
  using C = PfCfg<D>;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = once_per_device(done, [] {
    return cudaFuncSetAttribute(prefill_tc_kernel<PrefillTcArgs, D, MODE, CAP>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
  });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)items.size());
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = C::SMEM;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = MODE == kPairs ? 1 : 0;
  WorkList<CAP> wl;
  if (CAP > 0) memcpy(wl.item, items.data(), items.size() * sizeof(uint64_t));
  return cudaLaunchKernelEx(&cfg, prefill_tc_kernel<PrefillTcArgs, D, MODE, CAP>, a, wl);
}

template <int D>
cudaError_t launch_d(const PrefillTcArgs& a, const std::vector<uint64_t>& items, const std::vector<uint64_t>& pairs,
                     cudaStream_t s) {
  if (!pairs.empty()) return launch_cfg<D, kPairs, 2 * kPrefillSplitMost>(a, pairs, s);
  if (items.size() <= kSmall) return launch_cfg<D, kWhole, kSmall>(a, items, s);
  if (items.size() <= kPrefillByValue) return launch_cfg<D, kWhole, kPrefillByValue>(a, items, s);
  return launch_cfg<D, kWhole, 0>(a, items, s);
}

}  // namespace

bool prefill_tc_make_maps(PrefillTcArgs* a, const void* q, const void* k, const void* v, int B, int T) {
  const CacheGeom& g = a->geom;
  return make_rows_map(&a->tq, q, B, T, g.Hq, g.D, 0) && make_rows_map(&a->tk, k, B, T, g.Hkv, g.D, 0) &&
         make_rows_map(&a->tv, v, B, T, g.Hkv, g.D, 0);
}

// 4D map over one kind of cache region: [regions][K, V][cap rows][D], box
// [1][1][128][64], 128-byte swizzle. Rows past `cap` read as zeros.
// With `step` 2 the map holds every second of the cap rows, `base` being the
// first of them and `rows` their number.
static bool make_region_map(CUtensorMap* map, const void* base, int regions, int cap, int D, int step = 1,
                            int rows = 0) {
  auto fn = encode_fn();
  if (!fn) return false;
  if (step == 1) rows = cap;
  cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)rows, 2, (cuuint64_t)regions};
  cuuint64_t strides[3] = {(cuuint64_t)D * 2 * step, (cuuint64_t)cap * D * 2, (cuuint64_t)cap * D * 2 * 2};
  cuuint32_t box[4] = {64, 128, 1, 1};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, estr,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS;
}

bool make_cache_region_maps(CUtensorMap* tcr, CUtensorMap* tcs, const CacheGeom& g, const void* kv) {
  const bf16* base = static_cast<const bf16*>(kv);
  bool ok = true;
  if (g.n_r > 0) ok = ok && make_region_map(tcr, base + g.r_region(0, 0), g.B * g.n_r, g.max_seq, g.D);
  if (g.n_s > 0) ok = ok && make_region_map(tcs, base + g.s_region(0, 0), g.B * g.n_s, g.S + g.W, g.D);
  return ok;
}

bool make_decode_maps(DecodeArgs* a, const CacheGeom& g, const void* kv) {
  if (g.D != 64) return make_cache_region_maps(&a->tcr, &a->tcs, g, kv);
  const bf16* base = static_cast<const bf16*>(kv);
  bool ok = true;
  for (int odd = 0; odd < 2; ++odd) {
    auto pair_map = [&](CUtensorMap* map, const bf16* first, int regions, int cap) {
      // a region of one row has no odd row: its map repeats the even one
      const int shift = odd && cap > 1 ? g.D : 0;
      return make_region_map(map, first + shift, regions, cap, g.D, 2, odd && cap > 1 ? cap / 2 : (cap + 1) / 2);
    };
    if (g.n_r > 0)
      ok = ok && pair_map(odd ? &a->tcr_odd : &a->tcr, base + g.r_region(0, 0), g.B * g.n_r, g.max_seq);
    if (g.n_s > 0)
      ok = ok && pair_map(odd ? &a->tcs_odd : &a->tcs, base + g.s_region(0, 0), g.B * g.n_s, g.S + g.W);
  }
  return ok;
}

bool prefill_tc_make_cache_maps(PrefillTcArgs* a, const void* kv) {
  return make_cache_region_maps(&a->tcr, &a->tcs, a->geom, kv);
}

cudaError_t launch_prefill_tc(const PrefillTcArgs& a, const std::vector<uint64_t>& items,
                              const std::vector<uint64_t>& pairs, cudaStream_t s) {
  if (items.empty()) return cudaSuccess;
  if (a.geom.D == 128) return launch_d<128>(a, items, pairs, s);
  if (a.geom.D == 64) return launch_d<64>(a, items, pairs, s);
  return cudaErrorInvalidValue;
}

}  // namespace aoh
