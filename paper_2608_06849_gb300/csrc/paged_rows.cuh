// What the kernels over rows of a paged cache share (paged_rows.cu, rotate.cu, paged_attend.cuh,
// paged_decode.cuh): where a row of a call lies, and numbers of it.
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"
#include "internal.h"

namespace aoh {
namespace rows {

// Where row r of the call lies: its page, or -1, and its place in it.
struct Place {
  int page, row;
};

// Sequence of row r, for rows r0 .. r0 + 31 in the lanes of a warp (r0 and cu alike): the
// sequence of r0 by a search that splits in 32 at each step, and a few steps on from there.
__device__ __forceinline__ int seq_of(const PageRows& rows, int r0, int r) {
  if (rows.cu == nullptr) return r;
  const int lane = threadIdx.x & 31;
  int lo = 0, n = rows.n_seqs;  // cu[lo] <= r0 < cu[lo + n]
  while (n > 1) {
    const int step = (n + 31) / 32, at = lo + (lane + 1) * step;
    const int past = __popc(__ballot_sync(0xffffffffu, at < lo + n && __ldg(rows.cu + at) <= r0));
    lo += past * step;
    n = min(step, n - past * step);
  }
  while (lo + 1 < rows.n_seqs && __ldg(rows.cu + lo + 1) <= r) ++lo;
  return lo;
}

// The sequence of row r of the call, and where its rows begin and end; a row that cu gives to
// no sequence (before its first number or behind its last) lies outside of them.
struct Owner {
  int b, begin, end;
  __device__ __forceinline__ bool has(int r) const { return begin <= r && r < end; }
};
__device__ __forceinline__ Owner owner_of(const PageRows& rows, int r0, int r) {
  const int b = seq_of(rows, r0, r);
  return rows.cu ? Owner{b, __ldg(rows.cu + b), __ldg(rows.cu + b + 1)} : Owner{b, r, r + 1};
}

// The place of position pos of sequence b; an error where there is none.
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

// 16 bf16 numbers: 32 aligned bytes, but for tensors that are only 16-byte aligned.
struct Sixteen {
  uint32_t w[8];
};
template <bool WIDE>
__device__ __forceinline__ Sixteen load16(const void* p) {
  Sixteen x;
  if constexpr (WIDE) {
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(x.w[0]), "=r"(x.w[1]), "=r"(x.w[2]), "=r"(x.w[3]), "=r"(x.w[4]), "=r"(x.w[5]), "=r"(x.w[6]),
                   "=r"(x.w[7])
                 : "l"(p)
                 : "memory");
  } else {
    const uint4 a = *static_cast<const uint4*>(p), b = *(static_cast<const uint4*>(p) + 1);
    x = Sixteen{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
  }
  return x;
}
template <bool WIDE>
__device__ __forceinline__ void store16(void* p, const Sixteen& x) {
  if constexpr (WIDE) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(x.w[0]), "r"(x.w[1]), "r"(x.w[2]),
                 "r"(x.w[3]), "r"(x.w[4]), "r"(x.w[5]), "r"(x.w[6]), "r"(x.w[7])
                 : "memory");
  } else {
    *static_cast<uint4*>(p) = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
    *(static_cast<uint4*>(p) + 1) = make_uint4(x.w[4], x.w[5], x.w[6], x.w[7]);
  }
}

// What 16 e4m3 codes of a row with power e stand for: exactly, in bf16.
__device__ __forceinline__ Sixteen decode(const uint4& c, int e) {
  const float scale = __uint_as_float((uint32_t)(127 + e) << 23);
  const uint32_t w[4] = {c.x, c.y, c.z, c.w};
  Sixteen x;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t two = w[i / 2] >> (16 * (i & 1));
    const float2 f = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(two & 0xffffu), __NV_E4M3)));
    const float2 y = __fmul2_rn(f, make_float2(scale, scale));
    x.w[i] = float2_to_bf16x2(y.x, y.y);
  }
  return x;
}

// A lane's D / 32 numbers of key j of one head, of K (sel 0) or V, of a sequence with these pages (a page out of
// range: zeros).
template <int D>
__device__ __forceinline__ void load_key(const PagePool& pool, const int32_t* pages, int head, int j, int sel, int lane,
                                         float (&to)[D / 32]) {
  const int page = __ldg(pages + (j >> pool.lg_ps)), row = j & (pool.ps - 1);
  if ((unsigned)page >= (unsigned)pool.n_pages) {
#pragma unroll
    for (int n = 0; n < D / 32; ++n) to[n] = 0.f;
    return;
  }
  const size_t at = (((((size_t)page * 2 + sel) * pool.Hkv + head) << pool.lg_ps) + row) * D + lane * (D / 32);
  if (pool.form == 0) {
#pragma unroll
    for (int n = 0; n < D / 32; n += 2) {
      const float2 f = bf16x2_to_float2(*reinterpret_cast<const uint32_t*>(static_cast<const __nv_bfloat16*>(pool.data) + at + n));
      to[n] = f.x;
      to[n + 1] = f.y;
    }
  } else {
    const int e = pool.powers[((((size_t)page * pool.Hkv + head) * 2 + sel) << pool.lg_ps) + row];
    const float scale = __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
    for (int n = 0; n < D / 32; n += 2) {
      const uint16_t two = *reinterpret_cast<const uint16_t*>(static_cast<const uint8_t*>(pool.data) + at + n);
      const float2 f = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2(two, __NV_E4M3)));
      to[n] = f.x * scale;
      to[n + 1] = f.y * scale;
    }
  }
}

// What earlier kernels wrote is visible from here on; the next one may start its prologue.
__device__ __forceinline__ void after_the_last_kernel() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

}  // namespace rows
}  // namespace aoh
