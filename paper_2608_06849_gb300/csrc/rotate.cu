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
// D / 16 neighbouring lanes hold a row of one head, a lane two runs of 8 numbers, so chosen that the
// numbers of a pair are in one lane: 8 c .. and p + 8 c .. where the pairs are p apart. The vectors of a token
// lie side by side, and token after token: blocks that run at once walk through memory as it lies, next vectors
// on their way while others are worked on. (With a thread's vector fixed, one row after the other, the
// addresses cost a third of the instructions and the kernel was 3 to 18% slower.)
//
// Bound by HBM and, with norms, by the chain of a vector's sum, shuffles and root: 32,768 rows of 32/8 heads
// of 128 without norms 111 us (671 MB, 6.1 TB/s), with them 125 (5.4); 22,490 rows with norms to bf16 pages
// 107 (5.2), to 8-bit ones and read back 138; 16,384 rows of 32/8 heads of 64 to bf16 pages of 16 41 (4.9). One
// token of 28/4 heads 2.9 us in a graph (10 as calls, the host's time).
#include <cuda_fp8.h>

#include "paged_rows.cuh"

namespace aoh {
namespace {

using namespace rows;

constexpr int kThreads = 256;
constexpr int kBlocks = 3;       // of an SM
constexpr int kMostRows = 8;     // rows of a group
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

// A row's cosines and sines as float4 (two neighbouring pairs): for halves [4][8 lanes], so that the lanes of
// a row read neighbouring ones; for neighbouring pairs [2][16 runs of 8 numbers]. The float of a pair's
// cosine, which its sine follows.
__device__ __forceinline__ int turn_at(bool interleaved, int pair) {
  return 2 * (interleaved ? ((pair & 3) >> 1) * 32 + (pair >> 2) * 2 + (pair & 1)
                          : ((pair & 7) >> 1) * 16 + (pair >> 3) * 2 + (pair & 1));
}
__device__ __forceinline__ void turn_one(float& a, float& b, float c, float s) {
  const float x = a * c - b * s;
  b = a * s + b * c;
  a = x;
}

// Where a vector comes from and goes to: rows `stride` bytes apart.
struct Side {
  const uint8_t* in;
  uint8_t* out;
  uint32_t in_stride, out_stride;
  int first;  // of the token's vectors
  int norm;   // whether it is normalised: 1
};

// Blocks that run at once go through groups of rows; a thread through every 32nd (d_head 64: 64th) vector of a
// group, row after row, two of them in registers while it works on two.
template <int D, int FORM>
__global__ void __launch_bounds__(kThreads, kBlocks) rotate_kernel(const __grid_constant__ RotateArgs a, int rows_per_group) {
  constexpr int LPR = D / 16, SIDE = kThreads / LPR, U = 2;
  __shared__ __align__(16) float turns[2][kMostRows][128];
  __shared__ __align__(16) float weights[2][D];
  __shared__ Place place[4][kMostRows];
  __shared__ int position[4][kMostRows], given[4][kMostRows];  // given: whether the row is of a sequence
  __shared__ int8_t power[FORM == kPagesF8 ? 2 : 1][FORM == kPagesF8 ? 2 * kMaxKvHeads * kMostRows : 1];
  __shared__ Side sides[3];  // of q, k and v
  const int ch = threadIdx.x % LPR, n_rows = a.rows.n_rows, groups = (n_rows + rows_per_group - 1) / rows_per_group;
  const int nq = a.Hq, nk = a.Hkv, per_row = nq + nk + (FORM == kDense ? 0 : nk);
  const bool il = a.rope.interleaved != 0;
  // the lane's two runs of 8 numbers: numbers 8 * run0 .., and to_run1 bytes of bf16 behind them
  const int pr = a.rope.n_pairs >> 3, rest = D / 16 - pr;
  const int run0 = ch < pr ? ch : 2 * pr + (ch - pr), to_run1 = (ch < pr ? pr : rest) * 16;
  auto rows_of = [&](int g) { return min(rows_per_group, n_rows - g * rows_per_group); };
  auto kind_of = [&](int vec) { return vec < nq ? 0 : vec < nq + nk ? 1 : 2; };
  if (threadIdx.x < 3) {
    const int k = threadIdx.x;
    sides[k] = {static_cast<const uint8_t*>(k == 0 ? a.q : k == 1 ? a.k : a.v), static_cast<uint8_t*>(k == 0 ? a.q_out : a.k_out),
                (uint32_t)(2 * (k == 0 ? a.q_stride : k == 1 ? a.k_stride : a.v_stride)),
                (uint32_t)(2 * (k == 0 ? a.q_out_stride : a.k_out_stride)), k == 0 ? 0 : k == 1 ? nq : nq + nk,
                k < 2 && (k == 0 ? a.q_norm : a.k_norm) != nullptr};
  }
  __syncthreads();
  after_the_last_kernel();

  struct Batch {
    uint4 x[U][2];
    int row[U], vec[U];  // row: of the group, or one beyond
  };
  int at_group = blockIdx.x, at_row = 0, at_vec = threadIdx.x / LPR;  // of the next vector to be loaded
  auto load = [&](Batch& b) {  // of one group alone
    const int n = at_group < groups ? rows_of(at_group) : 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      while (at_vec >= per_row) {
        at_vec -= per_row;
        ++at_row;
      }
      b.row[u] = at_row;
      b.vec[u] = at_vec;
      if (at_row < n) {
        const Side& s = sides[kind_of(at_vec)];
        const uint8_t* from = s.in + (uint64_t)(uint32_t)(at_group * rows_per_group + at_row) * s.in_stride +
                              (uint32_t)((at_vec - s.first) * (2 * D) + run0 * 16);
        b.x[u][0] = *reinterpret_cast<const uint4*>(from);
        b.x[u][1] = *reinterpret_cast<const uint4*>(from + to_run1);
      }
      at_vec += SIDE;
    }
  };
  auto next_group = [&]() {
    at_group += gridDim.x;
    at_row = 0;
    at_vec = threadIdx.x / LPR;
  };
  // where group g's rows lie, and their positions; warp 0
  auto look = [&](int g, int slot) {
    if (threadIdx.x >= 32 || g >= groups) return;
    const int n = rows_of(g), r0 = g * rows_per_group, r = r0 + min((int)threadIdx.x, n - 1);
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
      place[slot][threadIdx.x] = p;
      position[slot][threadIdx.x] = pos;
      given[slot][threadIdx.x] = has;
    }
  };
  auto turn = [&](int g, int slot, int to) {
    if (g >= groups) return;
    for (int i = threadIdx.x; i < rows_of(g) * a.rope.n_pairs; i += kThreads) {
      const int r = i / a.rope.n_pairs, p = i - r * a.rope.n_pairs;
      const uint64_t t = (uint64_t)(int64_t)position[slot][r] * a.rope.turns[p] + (1ull << 31);
      float s, c;
      sincospif((float)(int)(t >> 32) * 0x1p-31f, &s, &c);
      float* at = turns[to][r] + turn_at(il, p);
      at[0] = c * a.rope.scale;
      at[1] = s * a.rope.scale;
    }
  };

  const unsigned lanes = ((1u << LPR) - 1u) << (threadIdx.x & 31 & ~(LPR - 1));
  auto work = [&](const Batch& b, int g, int n, int slot, int buf) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = b.row[u], vec = b.vec[u], kind = kind_of(vec);
      if (i >= n || (FORM != kDense && !given[slot][i])) continue;  // alike for a row's lanes
      const Side& side = sides[kind];
      float f[16];
      {
        const uint4 lo = b.x[u][0], hi = b.x[u][1];
        const uint32_t y[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float2 two = bf16x2_to_float2(y[j]);
          f[2 * j] = two.x;
          f[2 * j + 1] = two.y;
        }
      }
      if (side.norm) {
        float2 s2 = make_float2(0.f, 0.f);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float2 two = make_float2(f[2 * j], f[2 * j + 1]);
          s2 = __ffma2_rn(two, two, s2);
        }
        float s = s2.x + s2.y;
#pragma unroll
        for (int o = LPR / 2; o >= 1; o >>= 1) s += __shfl_xor_sync(lanes, s, o);
        const float inv = rsqrtf(s * (1.f / D) + a.eps);
        const float4* wt = reinterpret_cast<const float4*>(weights[kind & 1]) + run0;
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          const float4 w = wt[(h & 1) * (D / 8) + (h < 2 ? 0 : to_run1 >> 4)];
          f[4 * h] *= inv * w.x;
          f[4 * h + 1] *= inv * w.y;
          f[4 * h + 2] *= inv * w.z;
          f[4 * h + 3] *= inv * w.w;
        }
      }
      if (kind < 2 && ch < pr) {
        const float4* tr = reinterpret_cast<const float4*>(turns[buf][i]) + run0;
        if (il) {
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            const float4 t = tr[(h & 1) * 16 + (h < 2 ? 0 : to_run1 >> 4)];
            turn_one(f[4 * h], f[4 * h + 1], t.x, t.y);
            turn_one(f[4 * h + 2], f[4 * h + 3], t.z, t.w);
          }
        } else {
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            const float4 t = tr[h * 8];
            turn_one(f[2 * h], f[8 + 2 * h], t.x, t.y);
            turn_one(f[2 * h + 1], f[9 + 2 * h], t.z, t.w);
          }
        }
      }
      if (FORM == kPagesF8 && kind > 0) {
        int e;
        const uint4 c = encode<LPR>(f, &e);
        const int v = vec - nq;
        if (ch == 0) power[buf][v * kMostRows + i] = (int8_t)e;
        if (place[slot][i].page < 0) continue;
        uint8_t* to = static_cast<uint8_t*>(a.pool.data) + data_row(a.pool, place[slot][i], v) * D + run0 * 8;
        *reinterpret_cast<uint2*>(to) = make_uint2(c.x, c.y);
        *reinterpret_cast<uint2*>(to + (to_run1 >> 1)) = make_uint2(c.z, c.w);
        continue;
      }
      uint8_t* to;
      if (FORM == kDense || kind == 0) {
        to = side.out + (uint64_t)(uint32_t)(g * rows_per_group + i) * side.out_stride +
             (uint32_t)((vec - side.first) * (2 * D) + run0 * 16);
      } else {
        if (place[slot][i].page < 0) continue;
        to = static_cast<uint8_t*>(a.pool.data) + data_row(a.pool, place[slot][i], vec - nq) * (2 * D) + run0 * 16;
      }
      *reinterpret_cast<uint4*>(to) = make_uint4(float2_to_bf16x2(f[0], f[1]), float2_to_bf16x2(f[2], f[3]),
                                                 float2_to_bf16x2(f[4], f[5]), float2_to_bf16x2(f[6], f[7]));
      *reinterpret_cast<uint4*>(to + to_run1) = make_uint4(float2_to_bf16x2(f[8], f[9]), float2_to_bf16x2(f[10], f[11]),
                                                           float2_to_bf16x2(f[12], f[13]), float2_to_bf16x2(f[14], f[15]));
    }
  };
  // a head's powers of neighbouring tokens lie side by side: stored by neighbouring lanes
  auto store_powers = [&](int g, int slot, int buf) {
    if constexpr (FORM == kPagesF8) {
      const int n = rows_of(g);
      for (int u = threadIdx.x; u < 2 * nk * kMostRows; u += kThreads) {
        const int v = u / kMostRows, i = u % kMostRows;
        if (i < n && place[slot][i].page >= 0) a.pool.powers[power_at(a.pool, place[slot][i], v)] = power[buf][u];
      }
    }
  };

  Batch now, next;
  load(now);
  look(blockIdx.x, 0);
  for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
    const void* w = i < D ? a.q_norm : a.k_norm;
    const int j = i & (D - 1);
    // [half of a run][run][4]
    float f = 1.f;
    if (w) f = a.norm_f32 ? static_cast<const float*>(w)[j] : __bfloat162float(static_cast<const __nv_bfloat16*>(w)[j]);
    weights[i >= D][((j >> 2) & 1) * (D / 2) + (j >> 3) * 4 + (j & 3)] = f;
  }
  __syncthreads();
  turn(blockIdx.x, 0, 0);
  look(blockIdx.x + gridDim.x, 1);
  int k_group = 0;  // of the block's
  for (int g = blockIdx.x; g < groups; g += gridDim.x, ++k_group) {
    // the group's turns, and the next one's positions, are there; the last one's powers too
    __syncthreads();
    const int slot = k_group & 3, buf = k_group & 1, n = rows_of(g);
    if (k_group > 0) store_powers(g - gridDim.x, (k_group - 1) & 3, buf ^ 1);
    const int batches = (n * per_row + SIDE * U - 1) / (SIDE * U);
    for (int k = 0; k < batches; ++k) {
      if (k + 1 == batches) next_group();
      load(next);
      if (k == 0) {
        look(g + 2 * (int)gridDim.x, (k_group + 2) & 3);
        turn(g + gridDim.x, (k_group + 1) & 3, buf ^ 1);
      }
      work(now, g, n, slot, buf);
      now = next;
    }
  }
  if constexpr (FORM == kPagesF8) {
    __syncthreads();
    store_powers(blockIdx.x + (k_group - 1) * (int)gridDim.x, (k_group - 1) & 3, (k_group - 1) & 1);
  }
}

// As many blocks as run at once go through groups of up to 8 rows. The launch overlaps the end of the
// kernel before it.
template <int D, int FORM>
cudaError_t launch(const RotateArgs& a, int num_sms, cudaStream_t s) {
  // groups of as few rows as take no more rounds of the blocks than groups of 8 would. (The last round is not
  // full: 19,277 rows are 5.3 groups a block, 22,490 6.2, 16,384 4.5, where 32,768 are 8.98; 10 to 12% of the blocks' time.)
  const int n = a.rows.n_rows, blocks = kBlocks * num_sms, even = (n + blocks - 1) / blocks;
  const int each = (even + kMostRows - 1) / kMostRows, per = (even + each - 1) / each, groups = (n + per - 1) / per;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(groups < blocks ? groups : blocks));
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
