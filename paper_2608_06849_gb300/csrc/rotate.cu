// Norms of queries and keys for each head and their rotation by position, in one pass: into
// dense rows, or into the pages of a paged cache (include/aoh.h: aoh_norm_rotate,
// aoh_paged_append_rotated).
//
// A row x of D numbers becomes y = x w / sqrt(mean(x^2) + eps), and pairs (a, b) of its first 2 p
// numbers (a cos t - b sin t, a sin t + b cos t), times the rope's scale, with t = position *
// frequency; all in 32 bits, rounded once.
//
// Angles. A frequency is kept as the fraction of a turn that one position makes, in 64 bits behind the
// binary point. position * fraction modulo 2^64 is then the fraction of a turn itself, exact but for
// the fraction's own rounding (2^-64 a position: 2^-33 of a turn at the farthest), in one integer
// product, whatever the position; sincospif of its 32 leading bits gives the cosine and sine. A block
// forms those of its rows once for all heads.
//
// Both only move bytes: D / 16 neighbouring lanes hold a row of one head, a lane two runs of 8
// numbers, so chosen that the numbers of a pair are in one lane: 8 c .. and p + 8 c .. where the pairs
// are p apart. The vectors of a token lie side by side, four of a thread's on their way at once.
#include <cuda_fp8.h>

#include "paged_rows.cuh"

namespace aoh {
namespace {

using namespace rows;

constexpr int kThreads = 256;
constexpr int kMostRows = 16;    // rows of a block
constexpr int kDense = 0, kPagesBf16 = 1, kPagesF8 = 2;

// 16 numbers in 32 bits as e4m3 codes (the first 8 in x and y) with the row's power of two, as
// paged_rows.cu has them; LPR lanes hold the row.
template <int LPR>
__device__ __forceinline__ uint4 encode(const float (&f)[16], int* e) {
  const unsigned lanes = ((1u << LPR) - 1u) << (threadIdx.x & 31 & ~(LPR - 1));
  auto row_max = [&](float m) {
#pragma unroll
    for (int o = LPR / 2; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor_sync(lanes, m, o));
    return m;
  };
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) most = fmaxf(most, fabsf(f[i]));  // (no NaN)
  most = row_max(most);
  const bool odd = isinf(most);
  if (odd) {
    most = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (!isinf(f[i])) most = fmaxf(most, fabsf(f[i]));
    most = row_max(most);
  }
  const int bits = __float_as_int(most);
  // most = 1.f * 2^(E - 127): 448 = 1.75 * 2^8
  *e = min(max((bits >> 23) - ((bits & 0x7fffff) <= 0x600000 ? 135 : 134), -80), 120);
  const float scale = __uint_as_float((uint32_t)(127 - *e) << 23);
  const bool largest = *e == 120;  // codes end at 240
  uint32_t c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float2 y = __fmul2_rn(make_float2(f[2 * i], f[2 * i + 1]), make_float2(scale, scale));
    if (odd || largest) {
      if (largest) {
        y.x = isnan(y.x) ? y.x : fminf(fmaxf(y.x, -240.f), 240.f);
        y.y = isnan(y.y) ? y.y : fminf(fmaxf(y.y, -240.f), 240.f);
      }
      if (isinf(f[2 * i])) y.x = __uint_as_float(0x7fffffffu);
      if (isinf(f[2 * i + 1])) y.y = __uint_as_float(0x7fffffffu);
    }
    c[i] = __nv_cvt_float2_to_fp8x2(y, __NV_SATFINITE, __NV_E4M3);
  }
  return make_uint4(__byte_perm(c[0], c[1], 0x5410), __byte_perm(c[2], c[3], 0x5410), __byte_perm(c[4], c[5], 0x5410),
                    __byte_perm(c[6], c[7], 0x5410));
}

// A row's cosines and sines as float4 (two neighbouring pairs): for halves [4][8 lanes], so that
// the lanes of a row read neighbouring ones; for neighbouring pairs [2][16 runs of 8 numbers].
__device__ __forceinline__ int turn_at(bool interleaved, int pair) {
  return interleaved ? ((pair & 3) >> 1) * 32 + (pair >> 2) * 2 + (pair & 1) : ((pair & 7) >> 1) * 16 + (pair >> 3) * 2 + (pair & 1);
}

template <int D, int FORM>
__global__ void __launch_bounds__(kThreads, 3) rotate_kernel(const __grid_constant__ RotateArgs a, int rows_per_block) {
  constexpr int LPR = D / 16, GROUPS = kThreads / LPR, U = 4;
  __shared__ float2 turns[kMostRows][64];
  __shared__ __align__(16) float weights[2][D];
  __shared__ Place place[kMostRows];
  __shared__ int position[kMostRows], given[kMostRows];  // given: whether the row is of a sequence
  __shared__ int8_t power[FORM == kPagesF8 ? 2 * kMaxKvHeads * kMostRows : 1];
  const int r0 = blockIdx.x * rows_per_block, n = min(rows_per_block, a.rows.n_rows - r0);
  const int ch = threadIdx.x % LPR, group = threadIdx.x / LPR;
  const int nq = a.Hq, nk = a.Hkv, per_row = nq + nk + (FORM == kDense ? 0 : nk);
  const bool il = a.rope.interleaved != 0;
  // the lane's two runs of 8 numbers: numbers 8 * run0 .., 8 * run1 ..
  const int pr = a.rope.n_pairs >> 3, rest = D / 16 - pr;
  const int run0 = ch < pr ? ch : 2 * pr + (ch - pr), run1 = run0 + (ch < pr ? pr : rest);
  const bool turned = ch < pr;
  after_the_last_kernel();

  // items: row and vector, neighbouring vectors in neighbouring groups
  int row = 0, vec = group;
  auto settle = [&]() {
    while (vec >= per_row) {
      vec -= per_row;
      ++row;
    }
  };
  settle();
  struct Item {
    int row, vec;
  } it[U];
  uint4 x[U][2];
  auto load = [&]() {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      it[u] = {row, vec};
      if (row < n) {
        const int kind = vec < nq ? 0 : vec < nq + nk ? 1 : 2;
        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(kind == 0 ? a.q : kind == 1 ? a.k : a.v) +
                                   (r0 + row) * (kind == 0 ? a.q_stride : kind == 1 ? a.k_stride : a.v_stride) +
                                   (vec - (kind == 0 ? 0 : kind == 1 ? nq : nq + nk)) * D;
        x[u][0] = *reinterpret_cast<const uint4*>(src + run0 * 8);
        x[u][1] = *reinterpret_cast<const uint4*>(src + run1 * 8);
      }
      vec += GROUPS;
      settle();
    }
  };
  load();
  if (threadIdx.x < 32) {
    const int i = min((int)threadIdx.x, n - 1), r = r0 + i;
    int pos = 0;
    bool has = true;
    Place p{-1, 0};
    if constexpr (FORM != kDense) {
      const Owner o = owner_of(a.rows, r0, r);
      const int len = __ldg(a.lens + o.b);
      const bool fits = len <= a.rows.table_stride << a.pool.lg_ps;
      const long long at = o.has(r) && fits ? (long long)len - (o.end - r) : -1;
      const bool empty = a.rows.cu == nullptr && len == 0;  // a step's slot without a request has no row
      if ((int)threadIdx.x < n && !empty) p = place_of(a.pool, a.rows, o.b, at, a.err);
      has = at >= 0 && !empty;
      pos = (int)at;
    }
    if (a.positions) pos = __ldg(a.positions + r);
    if ((int)threadIdx.x < n) {
      place[threadIdx.x] = p;
      position[threadIdx.x] = pos;
      given[threadIdx.x] = has;
    }
  }
  for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
    const void* w = i < D ? a.q_norm : a.k_norm;
    const int j = i & (D - 1);
    // [half of a run][run][4]
    float f = 1.f;
    if (w) f = a.norm_f32 ? static_cast<const float*>(w)[j] : __bfloat162float(static_cast<const __nv_bfloat16*>(w)[j]);
    weights[i >= D][((j >> 2) & 1) * (D / 2) + (j >> 3) * 4 + (j & 3)] = f;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n * a.rope.n_pairs; i += kThreads) {
    const int r = i / a.rope.n_pairs, p = i - r * a.rope.n_pairs;
    const uint64_t t = (uint64_t)(int64_t)position[r] * a.rope.turns[p] + (1ull << 31);
    float s, c;
    sincospif((float)(int)(t >> 32) * 0x1p-31f, &s, &c);
    turns[r][turn_at(il, p)] = make_float2(c * a.rope.scale, s * a.rope.scale);
  }
  __syncthreads();

  const unsigned lanes = ((1u << LPR) - 1u) << (threadIdx.x & 31 & ~(LPR - 1));
  while (it[0].row < n) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (it[u].row >= n) continue;  // alike for a row's lanes
      const int i = it[u].row, kind = it[u].vec < nq ? 0 : it[u].vec < nq + nk ? 1 : 2;
      if (FORM != kDense && !given[i]) continue;
      float f[16];
      {
        const uint32_t w[8] = {x[u][0].x, x[u][0].y, x[u][0].z, x[u][0].w, x[u][1].x, x[u][1].y, x[u][1].z, x[u][1].w};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float2 y = bf16x2_to_float2(w[j]);
          f[2 * j] = y.x;
          f[2 * j + 1] = y.y;
        }
      }
      if (kind < 2) {
        if (kind == 0 ? a.q_norm != nullptr : a.k_norm != nullptr) {
          float2 s2 = make_float2(0.f, 0.f);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float2 y = make_float2(f[2 * j], f[2 * j + 1]);
            s2 = __ffma2_rn(y, y, s2);
          }
          float s = s2.x + s2.y;
#pragma unroll
          for (int o = LPR / 2; o >= 1; o >>= 1) s += __shfl_xor_sync(lanes, s, o);
          const float inv = rsqrtf(s * (1.f / D) + a.eps);
          const float4* wt = reinterpret_cast<const float4*>(weights[kind]);
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            const float4 w = wt[(h & 1) * (D / 8) + (h < 2 ? run0 : run1)];
            f[4 * h] *= inv * w.x;
            f[4 * h + 1] *= inv * w.y;
            f[4 * h + 2] *= inv * w.z;
            f[4 * h + 3] *= inv * w.w;
          }
        }
        if (turned) {
          const float4* tr = reinterpret_cast<const float4*>(turns[i]);
          if (il) {
#pragma unroll
            for (int h = 0; h < 4; ++h) {
              const float4 t = tr[(h & 1) * 16 + (h < 2 ? run0 : run1)];
              float* y = f + 4 * h;
              const float a0 = y[0], b0 = y[1], a1 = y[2], b1 = y[3];
              y[0] = a0 * t.x - b0 * t.y;
              y[1] = a0 * t.y + b0 * t.x;
              y[2] = a1 * t.z - b1 * t.w;
              y[3] = a1 * t.w + b1 * t.z;
            }
          } else {
#pragma unroll
            for (int h = 0; h < 4; ++h) {
              const float4 t = tr[h * 8 + run0];
              const float a0 = f[2 * h], b0 = f[8 + 2 * h], a1 = f[2 * h + 1], b1 = f[9 + 2 * h];
              f[2 * h] = a0 * t.x - b0 * t.y;
              f[8 + 2 * h] = a0 * t.y + b0 * t.x;
              f[2 * h + 1] = a1 * t.z - b1 * t.w;
              f[9 + 2 * h] = a1 * t.w + b1 * t.z;
            }
          }
        }
      }
      if (FORM == kPagesF8 && kind > 0) {
        int e;
        const uint4 c = encode<LPR>(f, &e);
        const int v = it[u].vec - nq;
        if (ch == 0) power[v * kMostRows + i] = (int8_t)e;
        if (place[i].page < 0) continue;
        uint8_t* dst = static_cast<uint8_t*>(a.pool.data) + data_row(a.pool, place[i], v) * D;
        *reinterpret_cast<uint2*>(dst + run0 * 8) = make_uint2(c.x, c.y);
        *reinterpret_cast<uint2*>(dst + run1 * 8) = make_uint2(c.z, c.w);
        continue;
      }
      __nv_bfloat16* dst;
      if (kind == 0) {
        dst = static_cast<__nv_bfloat16*>(a.q_out) + (r0 + i) * a.q_out_stride + it[u].vec * D;
      } else if (FORM == kDense) {
        dst = static_cast<__nv_bfloat16*>(a.k_out) + (r0 + i) * a.k_out_stride + (it[u].vec - nq) * D;
      } else {
        if (place[i].page < 0) continue;
        dst = static_cast<__nv_bfloat16*>(a.pool.data) + data_row(a.pool, place[i], it[u].vec - nq) * D;
      }
      uint4 lo, hi;
      lo.x = float2_to_bf16x2(f[0], f[1]);
      lo.y = float2_to_bf16x2(f[2], f[3]);
      lo.z = float2_to_bf16x2(f[4], f[5]);
      lo.w = float2_to_bf16x2(f[6], f[7]);
      hi.x = float2_to_bf16x2(f[8], f[9]);
      hi.y = float2_to_bf16x2(f[10], f[11]);
      hi.z = float2_to_bf16x2(f[12], f[13]);
      hi.w = float2_to_bf16x2(f[14], f[15]);
      *reinterpret_cast<uint4*>(dst + run0 * 8) = lo;
      *reinterpret_cast<uint4*>(dst + run1 * 8) = hi;
    }
    load();
  }
  if constexpr (FORM == kPagesF8) {
    // a head's powers of neighbouring tokens lie side by side: stored by neighbouring lanes
    __syncthreads();
    for (int u = threadIdx.x; u < 2 * nk * kMostRows; u += kThreads) {
      const int v = u / kMostRows, i = u % kMostRows;
      if (i < n && place[i].page >= 0) a.pool.powers[power_at(a.pool, place[i], v)] = power[u];
    }
  }
}

// Rows of a block: the call's rows on three blocks an SM (which run at once), up to 16. The launch
// overlaps the end of the kernel before it.
template <int D, int FORM>
cudaError_t launch(const RotateArgs& a, int num_sms, cudaStream_t s) {
  const int n = a.rows.n_rows, even = (n + 3 * num_sms - 1) / (3 * num_sms), per = even < kMostRows ? even : kMostRows;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((n + per - 1) / per));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, rotate_kernel<D, FORM>, a, per);
}

template <int D>
cudaError_t launch_form(const RotateArgs& a, int num_sms, cudaStream_t s) {
  if (a.rows.table == nullptr) return launch<D, kDense>(a, num_sms, s);
  return a.pool.form ? launch<D, kPagesF8>(a, num_sms, s) : launch<D, kPagesBf16>(a, num_sms, s);
}

}  // namespace

cudaError_t launch_rotate(const RotateArgs& a, int d_head, int num_sms, cudaStream_t s) {
  return d_head == 128 ? launch_form<128>(a, num_sms, s) : launch_form<64>(a, num_sms, s);
}

}  // namespace aoh
