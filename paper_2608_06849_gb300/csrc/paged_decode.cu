// Attention of one new token of every sequence over a paged cache. A block per
// (sequence, KV head): each warp takes every eighth visible key, its lanes D / 32
// numbers of the row each, with a softmax state (running max and sum, output) a query
// head; the warps' states are joined in shared memory.
#include <cuda_fp8.h>
#include <math.h>

#include "common.cuh"
#include "internal.h"

namespace aoh {
namespace {

constexpr int kWarps = 8;
constexpr int kMostG = 16;

template <int D, bool E4M3>
__global__ void __launch_bounds__(32 * kWarps) paged_decode_kernel(const __grid_constant__ PagedDecodeArgs a) {
  constexpr int PL = D / 32;
  __shared__ float sO[kWarps][D], sM[kWarps], sL[kWarps];
  const CacheGeom& g = a.geom;
  const int kvh = blockIdx.x, b = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int len = __ldg(a.lens + b);
  if (len < 0 || (long long)len > (long long)a.table_stride * a.pool.ps) {
    if (threadIdx.x == 0) atomicOr(a.err, kErrPages);
    len = len < 0 ? 0 : a.table_stride * a.pool.ps;
  }
  const int pos = len - 1;
  const int w0 = g.kind[kvh] ? max(g.wstart(pos), 0) : 0, skip = g.kind[kvh] ? max(w0 - g.S, 0) : 0;
  for (int h = 0; h < g.G; ++h) {
    const __nv_bfloat16* qp = static_cast<const __nv_bfloat16*>(a.q) + b * a.q_stride + (size_t)(kvh * g.G + h) * D + lane * PL;
    float q[PL], o[PL], m = -INFINITY, l = 0.f;
    for (int i = 0; i < PL; ++i) {
      q[i] = __bfloat162float(qp[i]) * a.scale_log2;
      o[i] = 0.f;
    }
    for (int r = warp; r < len - skip; r += kWarps) {
      const int j = r < g.S || skip == 0 ? r : r + skip;
      const int page = __ldg(a.table + (size_t)b * a.table_stride + (j >> a.pool.lg_ps));
      if ((unsigned)page >= (unsigned)a.pool.n_pages) {
        if (lane == 0) atomicOr(a.err, kErrPages);
        continue;
      }
      const size_t row = (((size_t)page * 2 * g.Hkv + kvh) << a.pool.lg_ps) + (j & (a.pool.ps - 1));
      const size_t vrow = row + ((size_t)g.Hkv << a.pool.lg_ps);
      float s = 0.f, v[PL];
      if constexpr (E4M3) {
        const size_t pw = ((((size_t)page * g.Hkv + kvh) * 2) << a.pool.lg_ps) + (j & (a.pool.ps - 1));
        const float ks = exp2f((float)a.pool.powers[pw]), vs = exp2f((float)a.pool.powers[pw + a.pool.ps]);
        const __nv_fp8_e4m3* d = static_cast<const __nv_fp8_e4m3*>(a.pool.data);
        for (int i = 0; i < PL; ++i) {
          s += (float)d[row * D + lane * PL + i] * ks * q[i];
          v[i] = (float)d[vrow * D + lane * PL + i] * vs;
        }
      } else {
        const __nv_bfloat16* d = static_cast<const __nv_bfloat16*>(a.pool.data);
        for (int i = 0; i < PL; ++i) {
          s += __bfloat162float(d[row * D + lane * PL + i]) * q[i];
          v[i] = __bfloat162float(d[vrow * D + lane * PL + i]);
        }
      }
      for (int x = 16; x >= 1; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
      const float mn = fmaxf(m, s), al = m == -INFINITY ? 0.f : exp2f(m - mn), p = exp2f(s - mn);
      l = l * al + p;
      for (int i = 0; i < PL; ++i) o[i] = o[i] * al + p * v[i];
      m = mn;
    }
    for (int i = 0; i < PL; ++i) sO[warp][lane * PL + i] = o[i];
    if (lane == 0) {
      sM[warp] = m;
      sL[warp] = l;
    }
    __syncthreads();
    if (threadIdx.x < D) {
      float M = -INFINITY, L = 0.f, O = 0.f;
      for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sM[w]);
      for (int w = 0; w < kWarps; ++w)
        if (sL[w] != 0.f) {
          const float f = exp2f(sM[w] - M);
          L += f * sL[w];
          O += f * sO[w][threadIdx.x];
        }
      static_cast<__nv_bfloat16*>(a.out)[((size_t)b * g.Hq + kvh * g.G + h) * D + threadIdx.x] =
          __float2bfloat16_rn(L == 0.f ? 0.f : O / L);
    }
    __syncthreads();
  }
}

}  // namespace

cudaError_t launch_paged_decode(const PagedDecodeArgs& a, cudaStream_t s) {
  const dim3 grid(a.geom.Hkv, a.n_seqs);
  if (a.pool.D == 128)
    (a.pool.form ? paged_decode_kernel<128, true> : paged_decode_kernel<128, false>)<<<grid, 32 * kWarps, 0, s>>>(a);
  else
    (a.pool.form ? paged_decode_kernel<64, true> : paged_decode_kernel<64, false>)<<<grid, 32 * kWarps, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace aoh
