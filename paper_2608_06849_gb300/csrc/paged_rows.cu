// Rows of a paged cache: a call's new keys and values written to their pages, and
// cached rows read back (include/aoh.h gives the layout).
//
// e4m3 rows. A row x of D numbers is stored as codes c_i and one power of two e, x_i ~
// c_i 2^e, with e the least power for which the largest finite |x_i| 2^-e is at most 448,
// in [-80, 120]. A power of two is no worse than any other scale here: the codes are
// floating-point numbers, whose relative precision does not depend on where in their
// range the row lies, x 2^-e is exact in fp32, so that each code is the nearest one to
// the exact quotient, and c 2^e is exact in bf16, so that a row read back is the stored
// one. At e = 120 codes end at 240: 256 * 2^120 and above are no bf16 numbers, and a finite number
// stays finite. NaN and infinities become the NaN code and do not count for e.
//
// Both kernels only move bytes: a lane holds 16 numbers (32 bytes of bf16) and D / 16
// neighbouring lanes one row of one head, the heads of a token next to each other, so that a
// token's K (or V) is read as one run of Hkv * D * 2 bytes, while each head's row goes to its
// own page block. Bound by HBM: 22,490 rows of 8 heads of 128 to 8-bit pages 27.7 us, back 24.9
// (139 MB, 5.0 and 5.6 TB/s); 65,536 rows 65.6 and 62.4 (6.2 and 6.5); 32,768 rows of 8 heads of 64,
// bf16, 20.5 and 20.6 (6.5). A step's 64 rows written and read back 5.3 us in a graph, two launches
// (10.9 us as calls, the host's time). With 8 numbers a lane the 8-bit append was bound by its integer
// instructions (132 for 8 numbers, 61% of their rate).
#include <cuda_fp8.h>

#include "common.cuh"
#include "internal.h"

namespace aoh {
namespace {

constexpr int kThreads = 256;
constexpr int kMostRows = 32;  // rows of a block, a lane of warp 0 each

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

// 16 numbers of a row of LPR lanes as e4m3 codes; *e: the row's power. Magnitudes of bf16
// numbers are ordered as their bits, two to a word; a row with an infinity or NaN is looked
// at again number by number.
template <int LPR>
__device__ __forceinline__ uint4 encode(const Sixteen& x, int* e) {
  // the row's lanes (another row of the warp may have ended)
  const unsigned lanes = ((1u << LPR) - 1u) << (threadIdx.x & 31 & ~(LPR - 1));
  auto row_max = [&](uint32_t two) {
#pragma unroll
    for (int o = LPR / 2; o >= 1; o >>= 1) two = __vmaxu2(two, __shfl_xor_sync(lanes, two, o));
    return max(two & 0xffffu, two >> 16);
  };
  uint32_t two = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) two = __vmaxu2(two, x.w[i] & 0x7fff7fffu);
  uint32_t most = row_max(two);
  const bool odd = most >= 0x7f80u;
  if (odd) {
    two = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t a = x.w[i] & 0x7fff7fffu;
      two = __vmaxu2(two, a & ~__vcmpgeu2(a, 0x7f807f80u));
    }
    most = row_max(two);
  }
  // most = 1.f * 2^(E - 127): 448 = 1.75 * 2^8
  *e = min(max((int)(most >> 7) - ((most & 0x7fu) <= 0x60u ? 135 : 134), -80), 120);
  const float scale = __uint_as_float((uint32_t)(127 - *e) << 23);
  const bool largest = *e == 120;
  uint32_t c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float2 f = __fmul2_rn(bf16x2_to_float2(x.w[i]), make_float2(scale, scale));
    if (odd || largest) {  // codes end at 240; infinities: NaN
      if (largest) f = make_float2(fminf(fmaxf(f.x, -240.f), 240.f), fminf(fmaxf(f.y, -240.f), 240.f));
      if ((x.w[i] & 0x7f80u) == 0x7f80u) f.x = __uint_as_float(0x7fffffffu);
      if ((x.w[i] & 0x7f800000u) == 0x7f800000u) f.y = __uint_as_float(0x7fffffffu);
    }
    c[i] = __nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E4M3);
  }
  return make_uint4(__byte_perm(c[0], c[1], 0x5410), __byte_perm(c[2], c[3], 0x5410), __byte_perm(c[4], c[5], 0x5410),
                    __byte_perm(c[6], c[7], 0x5410));
}

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

// A block's threads as (row of several at a time, vector of a token, 16 numbers of it): the
// vectors of a token side by side, up to as many as the block holds, and several tokens where
// it holds more. Each thread has U rows on their way at once.
template <int LPR>
struct Split {
  static constexpr int U = 4;
  int ch, vec, sub, vecs, rows;
  __host__ __device__ static int vecs_of(int per_row) {
    int vecs = kThreads / LPR;
    while (vecs >= 2 * per_row) vecs >>= 1;
    return vecs;
  }
  // rows that a block has on their way at once
  static int at_once(int per_row) { return U * (kThreads / LPR / vecs_of(per_row)); }
  __device__ __forceinline__ explicit Split(int per_row) {
    vecs = vecs_of(per_row);
    rows = kThreads / LPR / vecs;
    const int v = threadIdx.x / LPR;
    ch = threadIdx.x % LPR;
    sub = v / vecs;
    vec = v - sub * vecs;
  }
};

// What earlier kernels wrote is visible from here on; the next one may start its prologue.
__device__ __forceinline__ void after_the_last_kernel() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// WIDE: k, v and the strides are multiples of 32 bytes. The first rows are on their way while
// warp 0 looks up where they go, a chain of three or four loads.
template <int D, bool E4M3, bool WIDE>
__global__ void __launch_bounds__(kThreads, 4) append_kernel(const __grid_constant__ PagedAppendArgs a, int rows_per_block) {
  constexpr int LPR = D / 16, U = Split<LPR>::U;
  __shared__ Place place[kMostRows];
  __shared__ int8_t power[E4M3 ? 2 * kMaxKvHeads * kMostRows : 1];
  const int r0 = blockIdx.x * rows_per_block, n = min(rows_per_block, a.rows.n_rows - r0);
  const int per_row = 2 * a.pool.Hkv;
  const Split<LPR> t(per_row);
  const int lg_power = rows_per_block > 16 ? 5 : 4;  // powers are [vector][16 or 32 rows]
  after_the_last_kernel();
  Sixteen x[U];
  auto load = [&](int vec, int i0) {
    const bool is_v = vec >= a.pool.Hkv;
    const long long stride = is_v ? a.v_stride : a.k_stride;
    const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(is_v ? a.v : a.k) + (r0 + i0) * stride +
                               (is_v ? vec - a.pool.Hkv : vec) * D + t.ch * 16;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * t.rows < n) x[u] = load16<WIDE>(src + u * t.rows * stride);
  };
  auto store = [&](int vec, int i0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * t.rows;  // alike for a row's lanes
      if (i >= n) continue;
      const Place p = place[i];
      if constexpr (E4M3) {
        int e;
        const uint4 c = encode<LPR>(x[u], &e);
        if (t.ch == 0) power[(vec << lg_power) + i] = (int8_t)e;
        if (p.page < 0) continue;
        *reinterpret_cast<uint4*>(static_cast<uint8_t*>(a.pool.data) + data_row(a.pool, p, vec) * D + t.ch * 16) = c;
      } else {
        if (p.page < 0) continue;
        store16<true>(static_cast<__nv_bfloat16*>(a.pool.data) + data_row(a.pool, p, vec) * D + t.ch * 16, x[u]);
      }
    }
  };
  int vec = t.vec, i0 = t.sub;
  if (vec < per_row) load(vec, i0);
  if (threadIdx.x < 32) {
    const int r = r0 + min((int)threadIdx.x, n - 1);
    const Owner o = owner_of(a.rows, r0, r);
    const int len = __ldg(a.lens + o.b);
    const bool fits = len <= a.rows.table_stride << a.pool.lg_ps;
    const long long pos = o.has(r) && fits ? (long long)len - (o.end - r) : -1;
    if ((int)threadIdx.x < n)  // a step's slot without a request has no row
      place[threadIdx.x] = a.rows.cu == nullptr && len == 0 ? Place{-1, 0} : place_of(a.pool, a.rows, o.b, pos, a.err);
  }
  __syncthreads();
  while (vec < per_row) {
    store(vec, i0);
    i0 += U * t.rows;
    if (i0 >= n) {
      i0 = t.sub;
      vec += t.vecs;
    }
    if (vec < per_row) load(vec, i0);
  }
  if constexpr (E4M3) {
    // a head's powers of neighbouring tokens lie side by side: stored by neighbouring lanes
    __syncthreads();
    for (int u = threadIdx.x; u < per_row << lg_power; u += kThreads) {
      const int v = u >> lg_power, i = u & ((1 << lg_power) - 1);
      if (i < n && place[i].page >= 0) a.pool.powers[power_at(a.pool, place[i], v)] = power[u];
    }
  }
}

template <int D, bool E4M3, bool WIDE>
__global__ void __launch_bounds__(kThreads, 4) read_kernel(const __grid_constant__ PagedReadArgs a, int rows_per_block) {
  constexpr int LPR = D / 16, U = Split<LPR>::U;
  __shared__ Place place[kMostRows];
  const int r0 = blockIdx.x * rows_per_block, n = min(rows_per_block, a.rows.n_rows - r0);
  after_the_last_kernel();
  if (threadIdx.x < 32) {
    const int r = r0 + min((int)threadIdx.x, n - 1);
    const Owner o = owner_of(a.rows, r0, r);
    const long long pos = (a.first ? __ldg(a.first + o.b) : 0) + (long long)(r - o.begin);
    if ((int)threadIdx.x < n) place[threadIdx.x] = place_of(a.pool, a.rows, o.b, o.has(r) ? pos : -1, a.err);
  }
  __syncthreads();
  const int per_row = 2 * a.pool.Hkv;
  const Split<LPR> t(per_row);
  for (int vec = t.vec; vec < per_row; vec += t.vecs) {
    const bool is_v = vec >= a.pool.Hkv;
    __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(is_v ? a.v : a.k) +
                         ((size_t)r0 * a.pool.Hkv + (is_v ? vec - a.pool.Hkv : vec)) * D + t.ch * 16;
    for (int i0 = t.sub; i0 < n; i0 += U * t.rows) {
      Sixteen x[U];  // e4m3: 16 codes in the first four words
      int e[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * t.rows;
#pragma unroll
        for (int w = 0; w < 8; ++w) x[u].w[w] = 0;
        e[u] = 0;
        if (i >= n) continue;
        const Place p = place[i];
        if (p.page < 0) continue;
        const size_t at = data_row(a.pool, p, vec) * D + t.ch * 16;
        if constexpr (E4M3) {
          const uint4 c = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(a.pool.data) + at);
          x[u].w[0] = c.x;
          x[u].w[1] = c.y;
          x[u].w[2] = c.z;
          x[u].w[3] = c.w;
          e[u] = a.pool.powers[power_at(a.pool, p, vec)];
        } else {
          x[u] = load16<true>(static_cast<const __nv_bfloat16*>(a.pool.data) + at);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * t.rows;
        if (i >= n) continue;
        if constexpr (E4M3) x[u] = decode(make_uint4(x[u].w[0], x[u].w[1], x[u].w[2], x[u].w[3]), e[u]);
        store16<WIDE>(dst + (size_t)i * a.pool.Hkv * D, x[u]);
      }
    }
  }
}

// Rows of a block: the call's rows on four blocks an SM (which run at once), up to 16, or, of
// few heads, to as many as its threads have on their way at once (written and read, 4 x
// 2,090-10,231 rows of 2 heads of 64 16.4 -> 12.9 us, 3 x 3,000-9,000 of one of 128 11.8 -> 10.4; 8
// heads in blocks of 32 lose 2%). The launch overlaps the end of the kernel before it.
template <int D, class K, class A>
cudaError_t launch(K kernel, const A& a, int num_sms, cudaStream_t s) {
  const int fill = Split<D / 16>::at_once(2 * a.pool.Hkv), most = fill <= 16 ? 16 : kMostRows;
  const int n = a.rows.n_rows, even = (n + 4 * num_sms - 1) / (4 * num_sms), per = even < most ? even : most;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((n + per - 1) / per));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, a, per);
}

bool whole(const void* p, long long elements) {  // of 32 bytes
  return reinterpret_cast<uintptr_t>(p) % 32 == 0 && elements % 16 == 0;
}

template <int D, bool E4M3>
cudaError_t append(const PagedAppendArgs& a, int num_sms, cudaStream_t s) {
  return whole(a.k, a.k_stride) && whole(a.v, a.v_stride) ? launch<D>(append_kernel<D, E4M3, true>, a, num_sms, s)
                                                          : launch<D>(append_kernel<D, E4M3, false>, a, num_sms, s);
}
template <int D, bool E4M3>
cudaError_t read(const PagedReadArgs& a, int num_sms, cudaStream_t s) {
  return whole(a.k, 0) && whole(a.v, 0) ? launch<D>(read_kernel<D, E4M3, true>, a, num_sms, s)
                                        : launch<D>(read_kernel<D, E4M3, false>, a, num_sms, s);
}

}  // namespace

cudaError_t launch_paged_append(const PagedAppendArgs& a, int num_sms, cudaStream_t s) {
  if (a.pool.D == 128) return a.pool.form ? append<128, true>(a, num_sms, s) : append<128, false>(a, num_sms, s);
  return a.pool.form ? append<64, true>(a, num_sms, s) : append<64, false>(a, num_sms, s);
}

cudaError_t launch_paged_read(const PagedReadArgs& a, int num_sms, cudaStream_t s) {
  if (a.pool.D == 128) return a.pool.form ? read<128, true>(a, num_sms, s) : read<128, false>(a, num_sms, s);
  return a.pool.form ? read<64, true>(a, num_sms, s) : read<64, false>(a, num_sms, s);
}

}  // namespace aoh
