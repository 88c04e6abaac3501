// Rows of a paged cache: a call's new keys and values written to their pages, and
// cached rows read back (include/aoh.h gives the layout).
//
// e4m3 rows. A row x of D numbers is stored as codes c_i and one power of two e, x_i ~
// c_i 2^e, with e the least power for which the largest finite |x_i| 2^-e is at most 448,
// in [-80, 120]. A power of two is no worse than any other scale here: the codes are
// floating-point numbers, whose relative precision does not depend on where in their
// range the row lies, x 2^-e is exact in fp32, so that each code is the nearest one to
// the exact quotient, and c 2^e is exact in bf16, so that a row read back is the stored
// one. NaN and infinities become the NaN code and do not count for e.
//
// Both kernels only move bytes: a lane holds 16 bytes of bf16 and D / 8 neighbouring lanes
// one row of one head, the heads of a token next to each other, so that a token's K (or V)
// is read as one run of Hkv * D * 2 bytes, while each head's row goes to its own page block.
#include <cuda_fp8.h>

#include "common.cuh"
#include "internal.h"

namespace aoh {
namespace {

constexpr int kThreads = 256;
constexpr int kMostRows = 8;  // rows of a block

// Where row r of the call lies: its page, or -1, and its place in it.
struct Place {
  int page, row;
};

__device__ __forceinline__ int seq_of(const PageRows& rows, int r) {
  if (rows.cu == nullptr) return r;
  int lo = 0, hi = rows.n_seqs;  // cu[lo] <= r < cu[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (__ldg(rows.cu + mid) <= r)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

__device__ __forceinline__ Place place_of(const PagePool& pool, const PageRows& rows, int b, long long pos, uint32_t* err) {
  Place p{-1, (int)(pos & (pool.ps - 1))};
  const long long slot = pos >> pool.lg_ps;
  if (pos >= 0 && slot < rows.table_stride) p.page = __ldg(rows.table + (size_t)b * rows.table_stride + slot);
  if ((unsigned)p.page >= (unsigned)pool.n_pages) {
    p.page = -1;
    atomicOr(err, kErrPages);
  }
  return p;
}

// Vector `vec` of a token: head vec % Hkv of its K (vec < Hkv) or V.
__device__ __forceinline__ size_t data_row(const PagePool& pool, const Place& p, int vec) {
  return (((size_t)p.page * 2 * pool.Hkv + vec) << pool.lg_ps) + p.row;
}
__device__ __forceinline__ size_t power_at(const PagePool& pool, const Place& p, int vec) {
  const int sel = vec >= pool.Hkv, h = vec - sel * pool.Hkv;
  return ((((size_t)p.page * pool.Hkv + h) * 2 + sel) << pool.lg_ps) + p.row;
}

// 8 numbers of a row of CPR lanes as e4m3 codes; *e: the row's power.
template <int CPR>
__device__ __forceinline__ uint2 encode(const uint4& x, int* e) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t most = 0;  // bits of the largest finite |x|
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = w[i] & 0x7fffu, b = (w[i] >> 16) & 0x7fffu;
    most = max(most, a < 0x7f80u ? a : 0u);
    most = max(most, b < 0x7f80u ? b : 0u);
  }
#pragma unroll
  for (int o = CPR / 2; o >= 1; o >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
  // most = 1.f * 2^(E - 127): 448 = 1.75 * 2^8
  *e = min(max((int)(most >> 7) - ((most & 0x7fu) <= 0x60u ? 135 : 134), -80), 120);
  const float scale = __uint_as_float((uint32_t)(127 - *e) << 23);
  uint32_t c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float2 f = bf16x2_to_float2(w[i]);
    if ((w[i] & 0x7f80u) == 0x7f80u) f.x = __uint_as_float(0x7fffffffu);
    if ((w[i] & 0x7f800000u) == 0x7f800000u) f.y = __uint_as_float(0x7fffffffu);
    c[i] = __nv_cvt_float2_to_fp8x2(make_float2(f.x * scale, f.y * scale), __NV_SATFINITE, __NV_E4M3);
  }
  return make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
}

__device__ __forceinline__ uint4 decode(const uint2& c, int e) {
  const float scale = __uint_as_float((uint32_t)(127 + e) << 23);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t two = (i < 2 ? c.x : c.y) >> (16 * (i & 1));
    const float2 f = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(two & 0xffffu), __NV_E4M3)));
    w[i] = float2_to_bf16x2(f.x * scale, f.y * scale);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int D, bool E4M3>
__global__ void __launch_bounds__(kThreads) append_kernel(const __grid_constant__ PagedAppendArgs a, int rows_per_block) {
  constexpr int CPR = D / 8;
  __shared__ Place place[kMostRows];
  const int r0 = blockIdx.x * rows_per_block, n = min(rows_per_block, a.rows.n_rows - r0);
  if ((int)threadIdx.x < n) {
    const int r = r0 + threadIdx.x, b = seq_of(a.rows, r);
    const int end = a.rows.cu ? __ldg(a.rows.cu + b + 1) : r + 1;
    place[threadIdx.x] = place_of(a.pool, a.rows, b, (long long)__ldg(a.lens + b) - (end - r), a.err);
  }
  __syncthreads();
  const int ch = threadIdx.x % CPR, per_row = 2 * a.pool.Hkv;
  for (int u = threadIdx.x / CPR; u < n * per_row; u += kThreads / CPR) {
    const int i = u / per_row, vec = u - i * per_row;
    const bool is_v = vec >= a.pool.Hkv;
    const int h = is_v ? vec - a.pool.Hkv : vec;
    const __nv_bfloat16* src =
        is_v ? static_cast<const __nv_bfloat16*>(a.v) + (r0 + i) * a.v_stride : static_cast<const __nv_bfloat16*>(a.k) + (r0 + i) * a.k_stride;
    const uint4 x = *reinterpret_cast<const uint4*>(src + h * D + ch * 8);
    const Place p = place[i];
    if constexpr (E4M3) {
      int e;
      const uint2 c = encode<CPR>(x, &e);
      if (p.page < 0) continue;
      *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.pool.data) + data_row(a.pool, p, vec) * D + ch * 8) = c;
      if (ch == 0) a.pool.powers[power_at(a.pool, p, vec)] = (int8_t)e;
    } else {
      if (p.page < 0) continue;
      *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.pool.data) + data_row(a.pool, p, vec) * D + ch * 8) = x;
    }
  }
}

template <int D, bool E4M3>
__global__ void __launch_bounds__(kThreads) read_kernel(const __grid_constant__ PagedReadArgs a, int rows_per_block) {
  constexpr int CPR = D / 8;
  __shared__ Place place[kMostRows];
  const int r0 = blockIdx.x * rows_per_block, n = min(rows_per_block, a.rows.n_rows - r0);
  if ((int)threadIdx.x < n) {
    const int r = r0 + threadIdx.x, b = seq_of(a.rows, r);
    const long long pos = (a.first ? __ldg(a.first + b) : 0) + (long long)(a.rows.cu ? r - __ldg(a.rows.cu + b) : 0);
    place[threadIdx.x] = place_of(a.pool, a.rows, b, pos, a.err);
  }
  __syncthreads();
  const int ch = threadIdx.x % CPR, per_row = 2 * a.pool.Hkv;
  for (int u = threadIdx.x / CPR; u < n * per_row; u += kThreads / CPR) {
    const int i = u / per_row, vec = u - i * per_row;
    const bool is_v = vec >= a.pool.Hkv;
    const int h = is_v ? vec - a.pool.Hkv : vec;
    const Place p = place[i];
    uint4 x = make_uint4(0, 0, 0, 0);
    if (p.page >= 0) {
      const size_t at = data_row(a.pool, p, vec) * D + ch * 8;
      if constexpr (E4M3)
        x = decode(*reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(a.pool.data) + at),
                   a.pool.powers[power_at(a.pool, p, vec)]);
      else
        x = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.pool.data) + at);
    }
    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(is_v ? a.v : a.k) + ((size_t)(r0 + i) * a.pool.Hkv + h) * D + ch * 8) = x;
  }
}

// Rows of a block: one while the blocks of eight would leave SMs idle.
int rows_per_block(int n_rows, int num_sms) { return n_rows >= 4 * kMostRows * num_sms ? kMostRows : 1; }

}  // namespace

cudaError_t launch_paged_append(const PagedAppendArgs& a, int num_sms, cudaStream_t s) {
  const int per = rows_per_block(a.rows.n_rows, num_sms);
  const int grid = (a.rows.n_rows + per - 1) / per;
  if (a.pool.D == 128)
    (a.pool.form ? append_kernel<128, true> : append_kernel<128, false>)<<<grid, kThreads, 0, s>>>(a, per);
  else
    (a.pool.form ? append_kernel<64, true> : append_kernel<64, false>)<<<grid, kThreads, 0, s>>>(a, per);
  return cudaGetLastError();
}

cudaError_t launch_paged_read(const PagedReadArgs& a, int num_sms, cudaStream_t s) {
  const int per = rows_per_block(a.rows.n_rows, num_sms);
  const int grid = (a.rows.n_rows + per - 1) / per;
  if (a.pool.D == 128)
    (a.pool.form ? read_kernel<128, true> : read_kernel<128, false>)<<<grid, kThreads, 0, s>>>(a, per);
  else
    (a.pool.form ? read_kernel<64, true> : read_kernel<64, false>)<<<grid, kThreads, 0, s>>>(a, per);
  return cudaGetLastError();
}

}  // namespace aoh
