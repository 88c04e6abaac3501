// Attention of one new token of every sequence over a paged cache, on tcgen05 tensor
// cores, the cache split over its length (include/aoh.h: aoh_paged_decode).
//
// With G query heads a KV head, the cached rows of 128 keys and G queries are two skinny
// matrix products with the keys (or d) as the 128 rows of the MMA:
//   S^T[128 keys][G] = K[128][d] . Q^T           A = K, K-major; B = Q, K-major
//   O^T[d][G]       += V^T[d][128] . P^T[128][G] A = V, MN-major; B = P, K-major
// so that K and V go from the pages to the tensor cores as they lie, by TMA, whatever
// their format. For d_head 64 two groups of 128 keys stand side by side in the rows of one O^T
// (V of the first in rows 0-63, of the second in rows 64-127, weights in columns of their own).
//
// 8-bit pages. The codes are multiplied as they are (kind::f8f6f4); a row's power of two
// is applied to its score, and its V power to its weight:
//   s_j = 2^ek_j (q . K8_j) c,  w_j = 2^(s_j + ev_j - m),  o = sum_j w_j V8_j / sum_j w_j 2^-ev_j
// with m the running maximum of s_j + ev_j, so that w_j is the size of key j's contribution (a key
// whose w_j is zero as a float adds nothing to the numerator, but may to the sum below it). q
// (8 significant bits) is the sum of two e4m3 numbers (4 bits each): exactly, down to 2^-17 of the
// row's largest. A weight is the sum of three e5m2 numbers (3 bits each, rounded to
// nearest: 2^-9 of it, as good as bf16, at 2^-16 .. 2^15.8, so a key counts down to 2^-28 of
// the heaviest). The parts are columns of the MMAs, which have sixteen at least.
//
// The items, (sequence, KV head), are cut into tiles of 64 KB of K and V; all tiles, item
// after item, are dealt to the CTAs in equal runs, so that every CTA streams as many bytes
// whatever the lengths. Where CTAs share an item each stores its state (O, max, sum), and the
// last to arrive adds them up (groups of 16 first). A streaming head's tiles are the pages
// of its sinks and then those of its window.
//
// Short steps of few items run on whole clusters instead (CL): a cluster an item, whose CTAs
// add up their states through distributed shared memory, each finishing D / C values of every
// head.
//
// What bounds it: the bytes of the visible rows. A tile is 64 KB because a smaller one leaves the
// chain S -> weights -> P V above its transfer time (64 KB: 0.95 us a tile on an SM alone, 1.47 with
// all SMs reading), and three tiles are what shared memory holds: 96 KB in flight an SM
// behind the tile that is worked on. 16 sequences of 32,768 tokens, 32/8 heads, pages of 64, us
// (floor: bytes at the 6.8 TB/s of a copy): 8-bit d_head 128 159 (159), 64 90 (80); bf16 128 315
// (316), 64 159 (158). Pages of 16 cost 5% (8-bit, 128) to 20% (8-bit, 64): eight copies a
// block. 16 query heads a KV head: 176 and 156, the softmax of 16 columns takes longer than the
// tile's transfer. A step in equal runs pays 8-9 us besides (launch, plan, first tile, last tile's
// chain, arrival, joins), one on clusters 5: 1 x 4096 5.9 us, 4 x 8192 11.2.
//
// Warps: 4 or 8 of softmax (a thread one or two keys of the tile), 4 that finish items, two
// producers, one MMA issuer. O and the sums have two buffers, so that a CTA's next item goes
// on while its last one is finished, stored and joined.
#pragma once

#include <cuda_fp8.h>
#include <math.h>

#include "cluster.cuh"
#include "common.cuh"
#include "internal.h"
#include "tc.cuh"

namespace aoh {
namespace pdec {

using bf16 = __nv_bfloat16;
constexpr int kGroup = 16;          // states joined at a time
constexpr int kLensCap = 1024;      // lengths mirrored in shared memory
constexpr int kClusterMost = 16;    // CTAs of a cluster

// Shapes of one head size, format and (padded) number of query heads a KV head.
template <int D_, bool F8_, int GP_, bool CL = false>
struct Lay {
  static constexpr int D = D_, GP = GP_;
  static constexpr bool F8 = F8_;
  static constexpr int ES = F8 ? 1 : 2;                    // bytes of a number
  static constexpr int ROWB = D * ES < 128 ? D * ES : 128;  // bytes of a row in a block: the swizzle's width
  static constexpr int BOX = 128 * ROWB;                   // a block: 128 keys
  static constexpr int DBLK = D * ES / ROWB;               // blocks of a group of 128 keys
  static constexpr int GRP = DBLK * BOX;
  // a tile's K, or V: 32 KB, but where the weights of 16 heads leave no room for three such tiles
  static constexpr int HALF = F8 && D == 64 && GP == 16 ? 16384 : 32768;
  static constexpr int STAGE = 2 * HALF;
  static constexpr int NS = 3 * 32768 / HALF;              // ring stages
  static constexpr int NK = HALF / GRP;                    // groups of a tile
  static constexpr int KEYS = NK * 128;
  static constexpr int MB = 128 / D;                       // groups side by side in a P V MMA
  static constexpr int SETS = NK / MB;
  static constexpr int PARTS = F8 ? 3 : 1;                 // columns of a weight
  static constexpr int NPV = (MB * PARTS * GP + 15) / 16 * 16;
  static constexpr int SN = F8 ? (2 * GP + 15) / 16 * 16 : 16;
  static constexpr int SBUF = NK * SN;                     // TMEM columns of one tile's S
  static constexpr int OCOL = 2 * SBUF;
  static constexpr int TMEM_COLS = next_pow2(cmax(OCOL + 2 * NPV, 32));
  static constexpr int KP = NK == 4 ? 2 : 1;               // keys of a softmax thread
  static constexpr int SOFT = 128 * NK / KP;               // softmax threads
  static constexpr int NW = SOFT / 32;
  static constexpr int REDH = GP + (F8 ? 1 : 0);           // maxima that warps exchange: the heads', and of the V powers
  static constexpr int THREADS = SOFT + 128 + 96;
  static constexpr int QBLK = SN * ROWB, QBUF = DBLK * QBLK;
  static constexpr int NQ = CL ? 1 : 2;                    // Q buffers: a cluster has one item
  static constexpr int PBLK = NPV * 128;                   // weights of 128 bytes of keys
  static constexpr int PSET = PBLK * ES;
  static constexpr int PBUF = SETS * PSET;
  static constexpr int POWB = F8 ? 2 * KEYS : 0;           // a stage's powers
  static constexpr int NBAR = 3 * NS + 16 + 1;
  // behind the barriers, lengths; with clusters the others' states: [C][G][D / C] values, then
  // [C][16] (m, l)
  static constexpr int TAIL = CL ? GP * D * 4 + kClusterMost * 16 * 8 : kLensCap * 4;
  static constexpr int XBYTES = D == 64 ? GP * 64 * 4 : 0;
  static constexpr int FIXED = NS * STAGE + NQ * QBUF + NS * POWB + 2 * (REDH + GP) * NW * 4 + 128 + XBYTES + 128 + NBAR * 8 + 32 +
                               4 * 32 + kMaxKvHeads + TAIL + 1024;
  static constexpr int NPB = FIXED + 2 * PBUF <= 232448 ? 2 : 1;  // P buffers that fit
  static constexpr int OFF_Q = NS * STAGE;
  static constexpr int OFF_P = OFF_Q + NQ * QBUF;
  static constexpr int OFF_POW = OFF_P + NPB * PBUF;
  static constexpr int OFF_RED = OFF_POW + NS * POWB;     // [2][REDH][NW] warp maxima
  static constexpr int OFF_SUM = OFF_RED + 2 * REDH * NW * 4;  // [2][GP][NW] sums of an item, [2][16] maxima
  static constexpr int OFF_X = OFF_SUM + 2 * GP * NW * 4 + 128;  // [GP][64] the upper rows of O (d_head 64)
  static constexpr int OFF_QF = OFF_X + XBYTES;            // [2][16] factors of the scores
  static constexpr int OFF_BAR = OFF_QF + 128;
  static constexpr int OFF_MISC = OFF_BAR + NBAR * 8;
  static constexpr int OFF_LENS = OFF_MISC + 32 + 4 * 32 + kMaxKvHeads;
  static constexpr int SMEM = OFF_LENS + TAIL + 1024;
  // kind::f16 with bf16, or kind::f8f6f4 with e4m3 (weights: e5m2); V is MN-major
  static constexpr uint32_t IDESC_S = F8 ? idesc_f8(128, SN, false, 0) : idesc_bf16(128, SN, false, false);
  static constexpr uint32_t IDESC_PV = F8 ? idesc_f8(128, NPV, true, 1) : idesc_bf16(128, NPV, false, true);
  static constexpr float kRaise = F8 ? 12.f : 0.f;         // weights are 2^(s - m + kRaise)
  static constexpr float kLag = F8 ? 3.75f : 8.f;          // the maximum follows the keys' once it is so far behind
  static_assert(SMEM <= 232448, "shared memory");
  static_assert(OFF_P % 1024 == 0 && PBLK % 1024 == 0 && QBLK % 1024 == 0, "operand alignment");
  static_assert(TMEM_COLS <= 512, "TMEM columns");
};

// What the heads of a sequence of len tokens see, as tiles of 2^LG keys: a retrieval head every
// page (tr tiles), a streaming head the pages of its sinks and those of its window (ts tiles; from
// its gslot-th page on, gap pages are left out; w0: first position of the window).
struct Seq {
  int len, tr, ts, w0, gslot, gap;
};
template <int LG>
__device__ __forceinline__ Seq make_seq(const PagedDecodeArgs& a, int len) {
  const CacheGeom& g = a.geom;
  const int lg = a.pool.lg_ps, round = (1 << (LG - lg)) - 1;
  Seq q;
  q.len = len;
  q.w0 = q.gslot = q.gap = 0;
  const int slots = (int)(((unsigned)len + a.pool.ps - 1) >> lg);
  if (len - g.W > g.S) {
    q.w0 = len - g.W;
    q.gslot = (g.S + a.pool.ps - 1) >> lg;
    q.gap = max((q.w0 >> lg) - q.gslot, 0);
  }
  q.tr = (slots + round) >> (LG - lg);
  q.ts = (slots - q.gap + round) >> (LG - lg);
  return q;
}

// The tokens of sequence b, within what its table holds.
__device__ __forceinline__ int seq_len(const PagedDecodeArgs& a, int b, bool report) {
  const int n = __ldcg(a.lens + b), most = a.table_stride << a.pool.lg_ps;
  if (n >= 0 && n <= most) return n;
  if (report) atomicOr(a.err, kErrPages);
  return n < 0 ? 0 : most;
}

// x / d for 0 <= x, 0 < d: by a reciprocal, put right, where floats hold x.
__device__ __forceinline__ int quotient(int x, int d) {
  if (x >= 1 << 23) return (int)((unsigned)x / (unsigned)d);
  const int q = (int)__fdividef((float)x, (float)d), r = x - q * d;
  return q + (r >= d ? 1 : 0) - (r < 0 ? 1 : 0);
}

// How the tiles are dealt: CTA p < P has tiles first(p) .. first(p + 1) - 1 of `total`.
struct Deal {
  int P, per, rem;
  int total;
  __device__ __forceinline__ int first(int p) const { return p * per + min(p, rem); }
  __device__ __forceinline__ int cta_of(int x) const {
    const int wide = rem * (per + 1);
    return x < wide ? quotient(x, per + 1) : rem + quotient(x - wide, per);
  }
};

// The items of a CTA's run of tiles [start, end), in order; used by whole warps. Head k of a
// sequence: retrieval heads before streaming ones.
template <int LG>
struct Walk {
  const PagedDecodeArgs& a;
  const int* lens_s;       // the lengths in shared memory, or null: lane b of the warp has sequence b's
  const uint8_t* heads_s;  // KV head of head k
  int len_reg;             // (neither above kLensCap sequences: they are loaded)
  int start, end, off;     // off: the first tile of the item
  int b, k, lo, hi, tiles = 0;
  Seq q;
  // seq_off: the first tile of sequence b, which holds tile `start`
  __device__ __forceinline__ Walk(const PagedDecodeArgs& a_, const int* ls, const uint8_t* hs, int lr, int s, int e, int b0,
                                  int seq_off)
      : a(a_), lens_s(ls), heads_s(hs), len_reg(lr), start(s), end(e), off(seq_off), b(b0), k(-1) {
    if (start >= end) return;
    enter();
    // the item that holds it: the last one that starts at or before it, a lane an item
    const int lane = threadIdx.x & 31, x = start - off;
    k = __popc(__ballot_sync(0xffffffffu, lane + 1 < a.geom.Hkv && first_tile(lane + 1) <= x)) - 1;
    if (a.geom.Hkv > 32) k += __popc(__ballot_sync(0xffffffffu, lane + 33 < a.geom.Hkv && first_tile(lane + 33) <= x));
    off += first_tile(k + 1);
  }
  __device__ __forceinline__ int first_tile(int i) const {
    const int n_r = a.geom.n_r;
    return min(i, n_r) * q.tr + max(i - n_r, 0) * q.ts;
  }
  __device__ __forceinline__ void enter() {
    q = make_seq<LG>(a, a.n_seqs <= 32 ? __shfl_sync(0xffffffffu, len_reg, b) : lens_s ? lens_s[b] : seq_len(a, b, false));
  }
  __device__ __forceinline__ bool streaming() const { return k >= a.geom.n_r; }
  __device__ __forceinline__ int kvh() const { return heads_s[k]; }
  // page of the item (a slot) -> page of the sequence
  __device__ __forceinline__ int page_of_slot(int slot) const { return !streaming() || slot < q.gslot ? slot : slot + q.gap; }
  __device__ __forceinline__ int slots() const {
    return (int)(((unsigned)q.len + a.pool.ps - 1) >> a.pool.lg_ps) - (streaming() ? q.gap : 0);
  }
  __device__ __forceinline__ bool next() {
    while (true) {
      off += tiles;
      if (off >= end) return false;
      if (++k == a.geom.Hkv) {
        k = 0;
        ++b;
        enter();
      }
      tiles = streaming() ? q.ts : q.tr;
      lo = max(start - off, 0);
      hi = min(end - off, tiles);
      if (lo < hi) return true;
    }
  }
};

// The one item of a cluster: its CTAs have equal runs of its tiles.
template <int LG>
struct ClusterWalk {
  const PagedDecodeArgs& a;
  const uint8_t* heads_s;
  int b, k, lo, hi, tiles, off = 0;
  bool left;
  Seq q;
  __device__ __forceinline__ ClusterWalk(const PagedDecodeArgs& a_, const uint8_t* hs, int len, int b_, int k_, int rank,
                                         int lg_ctas)
      : a(a_), heads_s(hs), b(b_), k(k_) {
    q = make_seq<LG>(a, len);
    tiles = streaming() ? q.ts : q.tr;
    const int per = (tiles + (1 << lg_ctas) - 1) >> lg_ctas;
    lo = min(tiles, rank * per);
    hi = min(tiles, lo + per);
    left = lo < hi;
  }
  __device__ __forceinline__ bool streaming() const { return k >= a.geom.n_r; }
  __device__ __forceinline__ int kvh() const { return heads_s[k]; }
  __device__ __forceinline__ int page_of_slot(int slot) const { return !streaming() || slot < q.gslot ? slot : slot + q.gap; }
  __device__ __forceinline__ int slots() const {
    return (int)(((unsigned)q.len + a.pool.ps - 1) >> a.pool.lg_ps) - (streaming() ? q.gap : 0);
  }
  __device__ __forceinline__ bool next() {
    const bool r = left;
    left = false;
    return r;
  }
};

// A state of an item that CTAs share: O [G][D], then the maxima and sums [G] each. Slots of
// a CTA: 0, 1 the state of its first and of its last item, 2, 3 the states joined by the group
// that it heads.
__host__ __device__ constexpr int state_floats(int D) { return 16 * (D + 2); }
__device__ __forceinline__ float* state_slot(const PagedDecodeArgs& a, int cta, int slot, int D) {
  return a.states + ((size_t)cta * 4 + slot) * state_floats(D);
}

// l * 2^d of a state's sum, d <= 0. With 8-bit pages 2^d alone may round to zero where the product does
// not: a part whose V rows are 2^-120 of the others' has a sum that much greater than its weights.
__device__ __forceinline__ float scaled(float l, float d) {
  const float half = fast_exp2(0.5f * d);
  return l * half * half;
}

// Adds up n <= kGroup states and stores the outputs (out) or the sum (dst); 4 warps. State 0
// is at `first`, state j > 0 at rest + j * stride. A lane owns four values at a time, all
// states' of them on their way at once, and the lanes of a head hold the states' maxima and
// sums between them.
template <int D>
__device__ __forceinline__ void join(int n, const float* first, const float* rest, int stride, int G, bf16* out, float* dst) {
  const int lane = threadIdx.x & 31, src = lane & 16;
#pragma unroll 1
  for (int v = threadIdx.x & 127; v < (G * (D / 4) + 31) / 32 * 32; v += 128) {
    const bool mine = v < G * (D / 4);  // d_head 64, odd G: the last half-warp has no head
    const int h = mine ? v / (D / 4) : 0, vv = mine ? v : 0;
    const int js = min(lane & 15, n - 1);
    const float* p = (js == 0 ? first : rest + (size_t)js * stride) + G * D + h;
    const float mj = (lane & 15) < n ? __ldcg(p) : -INFINITY, lj = __ldcg(p + G);
    float4 x[kGroup];
    const float* from = rest + vv * 4;
    x[0] = __ldcg(reinterpret_cast<const float4*>(first) + vv);
#pragma unroll
    for (int j = 1; j < kGroup; ++j) {
      from += stride;
      if (j < n) x[j] = __ldcg(reinterpret_cast<const float4*>(from));
    }
    float M = mj;
#pragma unroll
    for (int o = 8; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
    const float w = mj == -INFINITY ? 0.f : fast_exp2(mj - M);
    float L = mj == -INFINITY ? 0.f : scaled(lj, mj - M);
#pragma unroll
    for (int o = 8; o >= 1; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
    float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int j = 0; j < kGroup; ++j) {
      const float f = __shfl_sync(0xffffffffu, w, src | j);
      if (j < n) {
        O.x += f * x[j].x;
        O.y += f * x[j].y;
        O.z += f * x[j].z;
        O.w += f * x[j].w;
      }
    }
    if (!mine) continue;
    if (out) {
      const float inv = 1.f / L;
      *reinterpret_cast<uint2*>(out + v * 4) =
          make_uint2(float2_to_bf16x2(O.x * inv, O.y * inv), float2_to_bf16x2(O.z * inv, O.w * inv));
    } else {
      __stcg(reinterpret_cast<float4*>(dst) + v, O);
      if (v % (D / 4) == 0) {
        __stcg(dst + G * D + h, M);
        __stcg(dst + G * D + G + h, L);
      }
    }
  }
}

// After CTA p stored its state of an item that CTAs f .. last share: the last of a group to
// arrive joins the group, the last group the item. The 128 threads of named barrier 2.
template <int D>
__device__ __forceinline__ void join_item(const PagedDecodeArgs& a, int p, int f, int last, int G, bf16* out,
                                          volatile int* flag) {
  constexpr int kCta = 4 * state_floats(D);
  const int groups = (last - f) / kGroup + 1, p0 = f + (p - f) / kGroup * kGroup;
  // what is joined: CTA p0's slot `slot`, then slot `slot_rest` of every step-th CTA from there
  int first = p0, slot = p0 == f ? 1 : 0, slot_rest = 0, step = 1, n = min(kGroup, last - p0 + 1);
  uint32_t* counter = &a.counters[3 * p0 + slot];
#pragma unroll 1
  while (true) {
    named_barrier_sync(2, 128);
    if ((threadIdx.x & 127) == 0) {
      const bool done = atom_add_acq_rel_gpu(counter, 1u) == (uint32_t)(n - 1);
      if (done) *counter = 0u;
      *flag = done;
    }
    named_barrier_sync(2, 128);
    if (!*flag) return;
    const bool whole = step > 1 || groups == 1;
    join<D>(n, state_slot(a, first, slot, D), state_slot(a, first, slot_rest, D), step * kCta, G, whole ? out : nullptr,
            state_slot(a, p0, p0 == f ? 3 : 2, D));
    if (whole) return;
    first = f;
    slot = 3;
    slot_rest = 2;
    step = kGroup;
    n = groups;
    counter = &a.counters[3 * f + 2];
  }
}

// Powers of two as floats.
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

template <int D, bool F8, int GP, bool CL>
__global__ void __launch_bounds__(Lay<D, F8, GP>::THREADS, 1)
    paged_decode_kernel(const __grid_constant__ PagedDecodeArgs a) {
  using C = Lay<D, F8, GP, CL>;
  constexpr int NK = C::NK, NW = C::NW, KP = C::KP, LG = NK == 1 ? 7 : NK == 2 ? 8 : 9;
  static_assert(1 << LG == C::KEYS, "keys of a tile");
  constexpr int NT = C::THREADS;
  constexpr int kFinish = NW, kLoadK = NW + 4, kLoadV = NW + 5, kMma = NW + 6;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  uint8_t* sQ = smem + C::OFF_Q;
  uint8_t* sP = smem + C::OFF_P;
  int8_t* sPow = reinterpret_cast<int8_t*>(smem + C::OFF_POW);
  float* red = reinterpret_cast<float*>(smem + C::OFF_RED);
  float* lsum = reinterpret_cast<float*>(smem + C::OFF_SUM);  // [2][GP][NW]
  float* mfin = lsum + 2 * GP * NW;                           // [2][16]
  float* upper = reinterpret_cast<float*>(smem + C::OFF_X);
  float* qfac = reinterpret_cast<float*>(smem + C::OFF_QF);
  uint64_t* k_full = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);  // K and powers of a stage landed
  uint64_t* v_full = k_full + C::NS;
  uint64_t* empty = v_full + C::NS;
  uint64_t* s_full = empty + C::NS;  // [2] S(j) in TMEM
  uint64_t* s_free = s_full + 2;   // [2] S(j) read by the softmax
  uint64_t* p_full = s_free + 2;   // [2] P(j) written
  uint64_t* p_free = p_full + 2;   // [2] O += P(j) V(j) done
  uint64_t* q_set = p_free + 2;    // [2] the item's factors written
  uint64_t* l_full = q_set + 2;    // [2] the item's sums and maxima written
  uint64_t* o_full = l_full + 2;   // [2] the item's O final
  uint64_t* o_free = o_full + 2;   // [2] the item's O, sums and maxima read
  uint64_t* drain = o_free + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* flag = reinterpret_cast<volatile int*>(tmem_slot + 2);
  int* first_s = reinterpret_cast<int*>(tmem_slot + 3);  // [2] the run's first sequence, and its first tile
  int* wsum = reinterpret_cast<int*>(smem + C::OFF_MISC + 32);
  uint8_t* heads_s = smem + C::OFF_MISC + 32 + 128;
  int* lens_s = reinterpret_cast<int*>(smem + C::OFF_LENS);
  float* recv = reinterpret_cast<float*>(smem + C::OFF_LENS);         // clusters
  float2* recv_ml = reinterpret_cast<float2*>(recv + GP * D);

  const CacheGeom& g = a.geom;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int G = g.G, lg = a.pool.lg_ps;

  // rows of Q and P that no head fills stay zero for the whole launch
  for (int i = threadIdx.x; i < (C::NQ * C::QBUF + C::NPB * C::PBUF) / 16; i += NT)
    reinterpret_cast<uint4*>(sQ)[i] = make_uint4(0, 0, 0, 0);
  fence_proxy_async_smem();
  if (threadIdx.x < 32) qfac[threadIdx.x] = 0.f;
  if (threadIdx.x < g.Hkv)
    heads_s[threadIdx.x] = (int)threadIdx.x < g.n_r ? g.r_head[threadIdx.x] : g.s_head[threadIdx.x - g.n_r];
  if (threadIdx.x == 0) {
    for (int s = 0; s < C::NS; ++s) {
      mbar_init(&k_full[s], 1);
      mbar_init(&v_full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(&s_full[x], 1);
      mbar_init(&s_free[x], NW);
      mbar_init(&p_full[x], NW);
      mbar_init(&p_free[x], 1);
      mbar_init(&q_set[x], 1);
      mbar_init(&l_full[x], NW);
      mbar_init(&o_full[x], 1);
      mbar_init(&o_free[x], 4);
    }
    mbar_init(drain, 1);
    *abort_flag = 0;
    first_s[0] = first_s[1] = 0;
    fence_mbar_init();
  }
  if (warp == kLoadK && lane == 0) prefetch_tmap(&a.pages);
  if (warp == kMma) {
    tmem_alloc(tmem_slot, C::TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  if constexpr (CL) cluster_arrive();  // others write into this CTA's shared memory once it runs
  // everything earlier kernels wrote is visible from here on
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  const int p = blockIdx.x;
  const bool few = a.n_seqs <= 32, mirrored = !few && a.n_seqs <= kLensCap;
  Deal deal;
  int len_reg = 0;
  const int lg_ctas = CL ? __ffs((int)cluster_ctas()) - 1 : 0, rank = CL ? (int)cluster_rank() : 0;
  auto plan = [&]() {
    if constexpr (CL) {
      const int id = p >> lg_ctas, b = quotient(id, g.Hkv);
      return ClusterWalk<LG>(a, heads_s, seq_len(a, b, rank == 0 && threadIdx.x == 0), b, id - b * g.Hkv, rank, lg_ctas);
    } else {
      // ---- this CTA's run: a prefix sum of the sequences' tiles; up to 32 sequences every warp
      // forms it for itself, a lane a sequence, without a barrier
      auto seq_tiles = [&](int len) {
        const Seq q = make_seq<LG>(a, len);
        return g.n_r * q.tr + g.n_s * q.ts;
      };
      auto scan = [&](int x, int n) {  // over the first n lanes
        for (int o = 1; o < n; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, x, o);
          if (lane >= o) x += y;
        }
        return x;
      };
      int b_first = 0, seq_off = 0;
      auto set_deal = [&](int total) {
        deal.total = total;
        deal.P = min((int)gridDim.x, total);
        deal.per = quotient(total, max(deal.P, 1));
        deal.rem = total - deal.per * deal.P;
      };
      if (few) {
        if (lane < a.n_seqs) len_reg = seq_len(a, lane, p == 0 && warp == 0);
        const int mine = lane < a.n_seqs ? seq_tiles(len_reg) : 0;
        set_deal(__reduce_add_sync(0xffffffffu, mine));
        const int inc = scan(mine, a.n_seqs);
        const unsigned past = __ballot_sync(0xffffffffu, lane < a.n_seqs && inc > deal.first(p));
        b_first = past ? __ffs(past) - 1 : 0;
        seq_off = __shfl_sync(0xffffffffu, inc - mine, b_first);
      } else {
        const int per = (a.n_seqs + NT - 1) / NT;
        const int b0 = min(a.n_seqs, (int)threadIdx.x * per), b1 = min(a.n_seqs, b0 + per);
        int mine = 0;
        for (int b = b0; b < b1; ++b) {
          const int len = seq_len(a, b, p == 0);
          if (mirrored) lens_s[b] = len;
          mine += seq_tiles(len);
        }
        const int inc = scan(mine, 32);
        if (lane == 31) wsum[warp] = inc;
        __syncthreads();
        const int part = lane < NT / 32 ? wsum[lane] : 0, upto = scan(part, 32);
        set_deal(__shfl_sync(0xffffffffu, upto, 31));
        int before = __shfl_sync(0xffffffffu, upto - part, warp) + inc - mine;
        const int start = deal.first(p);
        if (p < deal.P && before <= start && start < before + mine) {
          int b = b0;
          while (true) {
            const int n = seq_tiles(mirrored ? lens_s[b] : seq_len(a, b, false));
            if (start < before + n) break;
            before += n;
            ++b;
          }
          first_s[0] = b;
          first_s[1] = before;
        }
        __syncthreads();
        b_first = first_s[0];
        seq_off = first_s[1];
      }
      const bool any = p < deal.P;
      return Walk<LG>(a, mirrored ? lens_s : nullptr, heads_s, len_reg, any ? deal.first(p) : deal.total,
                      any ? deal.first(p + 1) : deal.total, b_first, any ? seq_off : deal.total);
    }
  };
  auto walk = plan();
  if constexpr (CL) cluster_wait();

  if (warp == kLoadK || warp == kLoadV) {
    // ------------------------------------------------------------ producers
    // One for K (and the powers), one for V; a lane a page of the tile. A copy takes its warp
    // some 80 clocks, its operands being per-lane values that have to become uniform, and
    // 16-token pages of 8-bit numbers 32 of them a tile: with one producer, which copied the
    // powers page by page too, 16 sequences of 32K took 230 us at such pages, 165 at 64 tokens.
    const bool is_v = warp == kLoadV;
    uint64_t* full = is_v ? v_full : k_full;
    const int spt = C::KEYS >> lg;  // pages of a tile, at most 32
    int it = 0;
    bool ok = true;
    while (ok && walk.next()) {
      const int32_t* row = a.table + (size_t)walk.b * a.table_stride;
      const int slots = walk.slots(), kvh = walk.kvh();
      for (int j = walk.lo; j < walk.hi; ++j, ++it) {
        const int st = it % C::NS;
        const int n = min(spt, slots - j * spt);
        int page = 0;
        if (lane < n) page = __ldg(row + walk.page_of_slot(j * spt + lane));
        const bool bad = (unsigned)page >= (unsigned)a.pool.n_pages;
        if (bad && !is_v) atomicOr(a.err, kErrPages);
        if (it >= C::NS) ok = __all_sync(0xffffffffu, wait_bar(&empty[st], ((it / C::NS) & 1) ^ 1, a.err, abort_flag));
        if (!ok) break;
        if constexpr (F8) {
          if (!is_v) {
            // the pages' powers, 16 bytes a lane
#pragma unroll
            for (int c0 = 0; c0 < C::POWB / 16; c0 += 32) {
              const int c = c0 + lane, slot = c >> (lg - 3);
              const int pg = __shfl_sync(0xffffffffu, bad ? 0 : page, slot);
              if (slot < n)
                cp_async16(sPow + st * C::POWB + c * 16,
                           a.pool.powers + (((size_t)pg * g.Hkv + kvh) << (lg + 1)) + (c & ((1 << (lg - 3)) - 1)) * 16);
            }
            cp_async_mbar_arrive(&full[st]);
            __syncwarp();
          }
        }
        if (lane == 0) mbar_arrive_expect_tx(&full[st], (uint32_t)(n << lg) * (D * C::ES));
        __syncwarp();
        if (lane < n) {
          const int key = lane << lg;  // of the tile
          uint8_t* dst = smem + st * C::STAGE + (is_v ? C::HALF : 0) + (key >> 7) * C::GRP + (key & 127) * C::ROWB;
          // a page out of range reads as zeros (its coordinate is past the map's end)
          const int block = bad ? 2 * g.Hkv * a.pool.n_pages : (page * 2 + (is_v ? 1 : 0)) * g.Hkv + kvh;
#pragma unroll
          for (int db = 0; db < C::DBLK; ++db) tma_load_3d(dst + db * C::BOX, &a.pages, db * 64, 0, block, &full[st]);
        }
        __syncwarp();
      }
    }
    // every issued copy lands before the CTA can exit
    if (F8) asm volatile("cp.async.wait_all;" ::: "memory");
    if (lane == 0)
      for (int j = it > C::NS ? it - C::NS : 0; j < it; ++j) drain_wait(&full[j % C::NS], (j / C::NS) & 1, a.err);
    __syncwarp();
  } else if (warp == kMma) {
    // ------------------------------------------------------------ MMA issuer
    constexpr int SBO = 8 * C::ROWB;
    const uint64_t k_desc0 = sdesc_rows<C::ROWB>(smem_u32(smem), 16, SBO);
    const uint64_t v_desc0 = sdesc_rows<C::ROWB>(smem_u32(smem) + C::HALF, C::BOX, SBO);
    const uint64_t q_desc0 = sdesc_rows<C::ROWB>(smem_u32(sQ), 16, SBO);
    const uint64_t p_desc0 = sdesc_rows<128>(smem_u32(sP), 16, 1024);
    constexpr int KSTEPS = D * C::ES / 32;        // 32 bytes of d a step
    constexpr int PSTEPS = 128 * C::ES / 32;      // 32 bytes of keys a step
    int it = 0, item = 0;
    bool ok = true;
    auto wait_warp = [&](uint64_t* bar, uint32_t parity) {
      if (ok) ok = __all_sync(0xffffffffu, wait_bar(bar, parity, a.err, abort_flag));
      return ok;
    };
    // P V of tile j, which waits behind the S of the tile after it
    int pend = -1, pend_item = 0;
    bool pend_first = false, pend_last = false;
    auto issue_pv = [&]() {
      const int j = pend;
      pend = -1;
      wait_warp(&v_full[j % C::NS], (j / C::NS) & 1);
      wait_warp(&p_full[j & 1], (j >> 1) & 1);
      if (!ok) return;
      if (elect_one()) {
        tc_fence_after();
        const uint32_t o = tmem + C::OCOL + (pend_item & 1) * C::NPV;
        const uint64_t v_desc = v_desc0 + (uint32_t)((j % C::NS) * sdesc_step(C::STAGE));
        const uint64_t p_desc = p_desc0 + (uint32_t)((j % C::NPB) * sdesc_step(C::PBUF));
#pragma unroll
        for (int z = 0; z < C::SETS; ++z)
#pragma unroll
          for (int kk = 0; kk < PSTEPS; ++kk)
            tc_mma_any<F8>(o, v_desc + sdesc_step(z * C::MB * C::GRP + kk * (32 / C::ES) * C::ROWB),
                           p_desc + sdesc_step(z * C::PSET + (kk >> 2) * C::PBLK + (kk & 3) * 32), C::IDESC_PV,
                           pend_first && z == 0 && kk == 0 ? 0u : 1u);
        tc_commit(&p_free[j & 1]);
        tc_commit(&empty[j % C::NS]);
        if (pend_last) tc_commit(&o_full[pend_item & 1]);
      }
      __syncwarp();
    };
    // An item's queries: piece c of the G x D block; CPR neighbouring lanes hold a row. Those
    // of the next item are on their way while this one's tiles are multiplied.
    constexpr int CPR = D / 8;
    constexpr int QV = (GP * CPR + 31) / 32;
    uint4 qr[QV];
    auto fetch = [&](int b, int kvh) {
      const bf16* qg = static_cast<const bf16*>(a.q) + (size_t)b * a.q_stride + (size_t)kvh * G * D;
#pragma unroll
      for (int i = 0; i < QV; ++i) {
        const int c = lane + 32 * i;
        qr[i] = c < G * CPR ? *reinterpret_cast<const uint4*>(qg + c * 8) : make_uint4(0, 0, 0, 0);
      }
    };
    bool more = walk.next();
    if (more) fetch(walk.b, walk.kvh());
    while (ok && more) {
      const int lo = walk.lo, hi = walk.hi;
      // Q's buffer and O's were last in use by item - 2
      if (item >= 2) wait_warp(&o_free[item & 1], ((item >> 1) - 1) & 1);
      if (!ok) break;
      uint8_t* qs = sQ + item % C::NQ * C::QBUF;
#pragma unroll
      for (int i = 0; i < QV; ++i) {
        const int c = lane + 32 * i, h = c / CPR, cc = c % CPR;
        if constexpr (!F8) {
          if (c < G * CPR)
            *reinterpret_cast<uint4*>(qs + (cc >> 3) * C::QBLK + h * 128 + (((cc & 7) ^ (h & 7)) << 4)) = qr[i];
        } else {
          // the row times the power of two that brings its largest number into [128, 256),
          // as two e4m3 numbers each
          const uint32_t w[4] = {qr[i].x, qr[i].y, qr[i].z, qr[i].w};
          uint32_t most = 0;
#pragma unroll
          for (int u = 0; u < 4; ++u) most = max(most, max(w[u] & 0x7fffu, (w[u] >> 16) & 0x7fffu));
#pragma unroll
          for (int o = CPR / 2; o >= 1; o >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
          // (an infinity makes its row's outputs NaN, as a NaN does)
          const int e = min(max(134 - (int)(most >> 7), -119), 119);
          const float up = pow2i(e);
          uint32_t hi[2] = {0, 0}, lo[2] = {0, 0};
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            float2 f = bf16x2_to_float2(w[u]);
            f.x = (w[u] & 0x7f80u) == 0x7f80u ? __uint_as_float(0x7fffffffu) : f.x * up;
            f.y = (w[u] & 0x7f800000u) == 0x7f800000u ? __uint_as_float(0x7fffffffu) : f.y * up;
            const uint32_t c2 = __nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E4M3);
            const float2 r = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)c2, __NV_E4M3)));
            const uint32_t l2 = __nv_cvt_float2_to_fp8x2(make_float2(f.x - r.x, f.y - r.y), __NV_SATFINITE, __NV_E4M3);
            hi[u >> 1] |= c2 << (16 * (u & 1));
            lo[u >> 1] |= l2 << (16 * (u & 1));
          }
          if (c < G * CPR) {
            // 8 codes: half of a 16-byte piece of the swizzled row
            auto put = [&](int n, const uint32_t (&x)[2]) {
              const int piece = C::ROWB == 128 ? (cc >> 1) ^ (n & 7) : (cc >> 1) ^ ((n >> 1) & 3);
              *reinterpret_cast<uint2*>(qs + n * C::ROWB + (piece << 4) + (cc & 1) * 8) = make_uint2(x[0], x[1]);
            };
            put(h, hi);
            put(GP + h, lo);
            if (cc == 0) qfac[(item & 1) * 16 + h] = a.scale_log2 * pow2i(-e);
          }
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (F8 && lane == 0) mbar_arrive(&q_set[item & 1]);
      more = walk.next();
      if (more) fetch(walk.b, walk.kvh());
      for (int j = lo; j < hi; ++j, ++it) {
        const int st = it % C::NS;
        // (a P V does not wait behind a tile that is still on its way)
        if (pend >= 0 && !__all_sync(0xffffffffu, mbar_test(&k_full[st], (it / C::NS) & 1))) issue_pv();
        wait_warp(&k_full[st], (it / C::NS) & 1);
        if (it >= 2) wait_warp(&s_free[it & 1], ((it >> 1) - 1) & 1);
        if (!ok) break;
        if (elect_one()) {
          tc_fence_after();
          const uint64_t k_desc = k_desc0 + (uint32_t)(st * sdesc_step(C::STAGE));
          const uint64_t q_desc = q_desc0 + (uint32_t)((item % C::NQ) * sdesc_step(C::QBUF));
#pragma unroll
          for (int y = 0; y < NK; ++y)
#pragma unroll
            for (int kk = 0; kk < KSTEPS; ++kk)
              tc_mma_any<F8>(tmem + (it & 1) * C::SBUF + y * C::SN,
                             k_desc + sdesc_step(y * C::GRP + (kk >> 2) * C::BOX + (kk & 3) * 32),
                             q_desc + sdesc_step((kk >> 2) * C::QBLK + (kk & 3) * 32), C::IDESC_S, kk > 0 ? 1u : 0u);
          tc_commit(&s_full[it & 1]);
        }
        __syncwarp();
        if (pend >= 0) issue_pv();
        pend = it;
        pend_item = item;
        pend_first = j == lo;
        pend_last = j == hi - 1;
      }
      ++item;
    }
    if (pend >= 0 && ok) issue_pv();
    if (elect_one()) tc_commit(drain);
    __syncwarp();
    drain_wait(drain, 0, a.err);
    __syncwarp();
  } else if (warp >= kFinish) {
    // ------------------------------------------------------------ finishing items
    const int r = threadIdx.x & 127;  // row of O^T
    const uint32_t tl = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    // sequences without a token
    for (int b = p; !CL && b < a.n_seqs; b += gridDim.x)
      if ((few ? __shfl_sync(0xffffffffu, len_reg, b) : mirrored ? lens_s[b] : seq_len(a, b, false)) == 0)
        for (int i = r; i < g.Hq * D / 8; i += 128)
          reinterpret_cast<uint4*>(static_cast<bf16*>(a.out) + (size_t)b * g.Hq * D)[i] = make_uint4(0, 0, 0, 0);
    // clusters: row r's values to the CTA that finishes it, head r's state to all
    const int lg_rows = CL ? (D == 128 ? 7 : 6) - lg_ctas : 0;
    auto push = [&](const float (&o)[GP], float m, float l) {
      if (r < D) {
        const uint32_t dst = cluster_addr(recv + ((rank * G) << lg_rows) + (r & ((1 << lg_rows) - 1)), (uint32_t)(r >> lg_rows));
#pragma unroll
        for (int h = 0; h < GP; ++h)
          if (h < G) cluster_st_f32(dst + (uint32_t)(h << lg_rows) * 4, o[h]);
      }
      if (r < G)
        for (int c = 0; c < 1 << lg_ctas; ++c)
          cluster_st2(cluster_addr(recv_ml + rank * 16 + r, (uint32_t)c), __float_as_uint(m), __float_as_uint(l));
    };
    if constexpr (CL) {
      if (!walk.left) {
        const float none[GP] = {};
        push(none, -INFINITY, 0.f);
      }
    }
    int item = 0;
    bool ok = true;
    while (ok && walk.next()) {
      const int x = item & 1;
      const int f = CL ? 0 : deal.cta_of(walk.off), last = CL ? 0 : deal.cta_of(walk.off + walk.tiles - 1);
      bf16* out = static_cast<bf16*>(a.out) + ((size_t)walk.b * g.Hq + (size_t)walk.kvh() * G) * D;
      ok = wait_bar(&l_full[x], (item >> 1) & 1, a.err, abort_flag);
      ok = wait_bar(&o_full[x], (item >> 1) & 1, a.err, abort_flag) && ok;
      tc_fence_after();
      float o[GP];
      {
        uint32_t part[C::PARTS][cmax(GP, 8)];
#pragma unroll
        for (int q = 0; q < C::PARTS; ++q) tmem_ld(tl + C::OCOL + x * C::NPV + (q * C::MB + r / D) * GP, part[q]);
        tmem_ld_wait();
#pragma unroll
        for (int h = 0; h < GP; ++h) {
          o[h] = __uint_as_float(part[0][h]);
#pragma unroll
          for (int q = 1; q < C::PARTS; ++q) o[h] += __uint_as_float(part[q][h]);
        }
      }
      if (D == 64 && r >= 64) {
#pragma unroll
        for (int h = 0; h < GP; ++h) upper[h * 64 + r - 64] = o[h];
      }
      ok = named_barrier_and(2, 128, ok);
      if (!ok) break;
      if (D == 64 && r < 64) {
#pragma unroll
        for (int h = 0; h < GP; ++h) o[h] += upper[h * 64 + r];
      }
      auto sum_of = [&](int h) {
        float L = 0.f;
#pragma unroll
        for (int u = 0; u < NW; u += 4) {
          const float4 s4 = *reinterpret_cast<const float4*>(lsum + (x * GP + h) * NW + u);
          L += (s4.x + s4.y) + (s4.z + s4.w);
        }
        return L;
      };
      if constexpr (CL) {
        push(o, r < G ? mfin[x * 16 + r] : 0.f, r < G ? sum_of(r) : 0.f);
      } else if (f == last) {
#pragma unroll
        for (int h = 0; h < GP; ++h)
          if (r < D && h < G) out[h * D + r] = __float2bfloat16_rn(__fdividef(o[h], sum_of(h)));
        if (D == 64) named_barrier_sync(2, 128);  // `upper` has been read
      } else {
        float* slot = state_slot(a, p, p == f ? 1 : 0, D);
#pragma unroll
        for (int h = 0; h < GP; ++h)
          if (r < D && h < G) __stcg(slot + h * D + r, o[h]);
        if (r < G) {
          __stcg(slot + G * D + r, mfin[x * 16 + r]);
          __stcg(slot + G * D + G + r, sum_of(r));
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&o_free[x]);
      ++item;
      if (f != last) {
        join_item<D>(a, p, f, last, G, out, flag);
      }
    }
  } else {
    // ------------------------------------------------------------ softmax
    const int t = threadIdx.x;            // key of the tile (and key t + SOFT)
    const int r = t & 127;                // its row in its group (and row r of O^T, threads 0-127)
    const uint32_t tl = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    int it = 0, item = 0;
    // ok: the softmax threads' common verdict, set at a barrier; local_ok: this thread's waits since
    bool ok = true, local_ok = true;
    while (ok && walk.next()) {
      const Seq& w = walk.q;
      const bool strm = walk.streaming();
      float m[GP], l[GP];
      // V powers below this, 90 below the largest of the tiles that moved a maximum: a key of any other whose
      // weight is zero as a float has less than 2^-48 of the weight of the one that is the maximum. (Asking
      // every weight instead costs 2 to 7%, asking so 1 to 4, and 6 on 128 x 1,000 tokens of 64-wide heads.)
      float ev_far = -INFINITY;
#pragma unroll
      for (int h = 0; h < GP; ++h) {
        m[h] = -INFINITY;
        l[h] = 0.f;
      }
      for (int j = walk.lo; j < walk.hi; ++j, ++it) {
        const int x = it & 1, st = it % C::NS;
        const bool first = j == walk.lo;
        bool see[KP];
        int ek[KP], ev[KP];
        if (F8) local_ok = wait_bar(&k_full[st], (it / C::NS) & 1, a.err, abort_flag) && local_ok;
#pragma unroll
        for (int c = 0; c < KP; ++c) {
          const int key = t + c * C::SOFT, y = key >> 7;
          const int slot = (j << (LG - lg)) + (key >> lg);
          const long long pos = ((long long)walk.page_of_slot(slot) << lg) + (key & (a.pool.ps - 1));
          see[c] = pos < w.len && (!strm || pos < g.S || pos >= w.w0);
          const unsigned hidden = __ballot_sync(0xffffffffu, !see[c]);
          ek[c] = ev[c] = 0;
          if constexpr (F8) {
            const int8_t* pw = sPow + st * C::POWB + ((key >> lg) << (lg + 1)) + (key & (a.pool.ps - 1));
            ek[c] = see[c] ? pw[0] : 0;
            ev[c] = see[c] ? pw[a.pool.ps] : 0;
          }
          if (hidden) {
            // V rows that no weight may meet (0 times a NaN is NaN), while S is formed
            constexpr int CH = C::ROWB / 16;
            local_ok = wait_bar(&v_full[st], (it / C::NS) & 1, a.err, abort_flag) && local_ok;
#pragma unroll
            for (int db = 0; db < C::DBLK; ++db) {
              uint4* v4 = reinterpret_cast<uint4*>(smem + st * C::STAGE + C::HALF + y * C::GRP + db * C::BOX +
                                                   (warp & 3) * 32 * C::ROWB);
              for (int i = lane; i < 32 * CH; i += 32)
                if (hidden >> (i / CH) & 1) v4[i] = make_uint4(0, 0, 0, 0);
            }
          }
        }
        if (F8 && first) local_ok = wait_bar(&q_set[item & 1], (item >> 1) & 1, a.err, abort_flag) && local_ok;
        local_ok = wait_bar(&s_full[x], (it >> 1) & 1, a.err, abort_flag) && local_ok;
        tc_fence_after();
        constexpr int SC = F8 ? cmax(2 * GP, 8) : cmax(GP, 8);  // columns read
        uint32_t v[KP][SC];
#pragma unroll
        for (int c = 0; c < KP; ++c) tmem_ld(tl + x * C::SBUF + ((t + c * C::SOFT) >> 7) * C::SN, v[c]);
        tmem_ld_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s_free[x]);
        float s[KP][GP];
#pragma unroll
        for (int c = 0; c < KP; ++c) {
          const float kf = pow2i(ek[c]);
#pragma unroll
          for (int h = 0; h < GP; ++h) {
            if constexpr (F8)
              s[c][h] = fmaf(__uint_as_float(v[c][h]) + __uint_as_float(v[c][GP + h]), kf * qfac[(item & 1) * 16 + h],
                             (float)ev[c]);
            else
              s[c][h] = __uint_as_float(v[c][h]) * a.scale_log2;
            if (!see[c]) s[c][h] = -INFINITY;
          }
        }
        // the running maximum moves only when a key is far above it; all threads agree
        auto top_of = [&](int h) { return warp_max(KP == 2 ? fmaxf(s[0][h], s[KP - 1][h]) : s[0][h]); };
        bool below = local_ok;
        if (!first) {
          float wm[GP];
#pragma unroll
          for (int h = 0; h < GP; ++h) wm[h] = top_of(h);
#pragma unroll
          for (int h = 0; h < GP; ++h) below = below && wm[h] <= m[h] + C::kLag;
        }
        if (first || !named_barrier_and(1, C::SOFT, below)) {
          float* rx = red + x * (C::REDH * NW);
          {
            float wm[GP];
#pragma unroll
            for (int h = 0; h < GP; ++h) wm[h] = top_of(h);
            if (lane == 0) {
#pragma unroll
              for (int h = 0; h < GP; ++h) rx[h * NW + warp] = wm[h];
            }
            if constexpr (F8) {
              const float top = warp_max((float)max(ev[0], ev[KP - 1]));
              if (lane == 0) rx[GP * NW + warp] = top;
            }
          }
          ok = named_barrier_and(1, C::SOFT, local_ok);
          if (!ok) break;
          auto top_in = [&](int h) {
            float top = -INFINITY;
#pragma unroll
            for (int u = 0; u < NW; u += 4) {
              const float4 f = *reinterpret_cast<const float4*>(rx + h * NW + u);
              top = fmaxf(top, fmaxf(fmax3f(f.x, f.y, f.z), f.w));
            }
            return top;
          };
          if (F8) ev_far = fmaxf(ev_far, top_in(GP) - 90.f);
          bool resc = false;
          float alpha[GP];
#pragma unroll
          for (int h = 0; h < GP; ++h) {
            const float top = top_in(h);
            alpha[h] = 1.f;
            if (first) {
              m[h] = top;
            } else if (top > m[h] + C::kLag) {
              alpha[h] = m[h] == -INFINITY ? 0.f : fast_exp2(m[h] - top);
              l[h] = F8 ? scaled(l[h], m[h] - top) : l[h] * alpha[h];
              m[h] = top;
              resc = true;
            }
          }
          if (resc && warp < 4) {
            // row r of O^T, once O += P(it - 1) V has landed
            local_ok = wait_bar(&p_free[x ^ 1], ((it - 1) >> 1) & 1, a.err, abort_flag) && local_ok;
            tc_fence_after();
#pragma unroll
            for (int q = 0; q < C::MB * C::PARTS; ++q) {
              const uint32_t col = tl + C::OCOL + (item & 1) * C::NPV + q * GP;
              uint32_t o[cmax(GP, 8)];
              tmem_ld(col, o);
              tmem_ld_wait();
#pragma unroll
              for (int h = 0; h < GP; ++h) o[h] = __float_as_uint(__uint_as_float(o[h]) * alpha[h]);
              tmem_st_n<GP>(col, o);
            }
            tmem_st_wait();
          }
        }
        if (F8 && fminf((float)ev[0], (float)ev[KP - 1]) < ev_far) {  // a weight that is zero may not be so times 2^-ev
#pragma unroll
          for (int c = 0; c < KP; ++c)
#pragma unroll
            for (int h = 0; h < GP; ++h) {
              const float low = s[c][h] - m[h] + C::kRaise;
              if (see[c] && low < -126.f) {
                l[h] += fast_exp2(low - (float)ev[c]);
                s[c][h] = -INFINITY;
              }
            }
        }
        // the P buffer is free once O += P(it - NPB) V is done
        if (it >= C::NPB)
          local_ok = wait_bar(&p_free[(it - C::NPB) & 1], ((it - C::NPB) >> 1) & 1, a.err, abort_flag) && local_ok;
#pragma unroll
        for (int c = 0; c < KP; ++c) {
          const int y = (t + c * C::SOFT) >> 7;
          float pr[GP];
#pragma unroll
          for (int h = 0; h < GP; ++h) pr[h] = see[c] ? fast_exp2(s[c][h] - m[h] + C::kRaise) : 0.f;
          // weights of key r of group y -> column r of the K-major [NPV][128 keys] buffer of its set
          uint8_t* pb = sP + (it % C::NPB) * C::PBUF + (y / C::MB) * C::PSET;
          const int n0 = (y % C::MB) * GP;
          if constexpr (F8) {
            const float un = pow2i(-ev[c]);
#pragma unroll
            for (int h = 0; h < GP; h += 2) {
              float2 rest = make_float2(pr[h], pr[h + 1]);
              l[h] = fmaf(rest.x, un, l[h]);
              l[h + 1] = fmaf(rest.y, un, l[h + 1]);
#pragma unroll
              for (int q = 0; q < C::PARTS; ++q) {
                const uint32_t c2 = __nv_cvt_float2_to_fp8x2(rest, __NV_SATFINITE, __NV_E5M2);
                const int n = q * C::MB * GP + n0 + h;
                pb[n * 128 + (((r >> 4) ^ (n & 7)) << 4) + (r & 15)] = (uint8_t)c2;
                pb[(n + 1) * 128 + (((r >> 4) ^ ((n + 1) & 7)) << 4) + (r & 15)] = (uint8_t)(c2 >> 8);
                if (q + 1 < C::PARTS) {
                  const float2 f = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)c2, __NV_E5M2)));
                  rest.x -= f.x;
                  rest.y -= f.y;
                }
              }
            }
          } else {
#pragma unroll
            for (int h = 0; h < GP; ++h) {
              l[h] += pr[h];
              const int n = n0 + h;
              *reinterpret_cast<bf16*>(pb + (r >> 6) * C::PBLK + n * 128 + ((((r & 63) >> 3) ^ (n & 7)) << 4) + (r & 7) * 2) =
                  __float2bfloat16_rn(pr[h]);
            }
          }
        }
        fence_proxy_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[x]);
      }
      if (!ok) break;

      // ---- the item's sums and maxima, for the warps that finish it
      if (item >= 2) local_ok = wait_bar(&o_free[item & 1], ((item >> 1) - 1) & 1, a.err, abort_flag) && local_ok;
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) {
#pragma unroll
        for (int h = 0; h < GP; ++h) l[h] += __shfl_xor_sync(0xffffffffu, l[h], o);
      }
      if (lane == 0) {
#pragma unroll
        for (int h = 0; h < GP; ++h) {
          lsum[((item & 1) * GP + h) * NW + warp] = l[h];
          if (warp == 0) mfin[(item & 1) * 16 + h] = m[h];
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&l_full[item & 1]);
      ++item;
    }
  }

  tc_fence_before();
  if constexpr (CL) {
    // the states of all CTAs have arrived (the waits of one that gave up are bounded: it comes
    // here too)
    __syncwarp();
    cluster_arrive();
    cluster_wait();
    if (warp >= kFinish && warp < kFinish + 4) {
      const int lg_rows = (D == 128 ? 7 : 6) - lg_ctas, n = 1 << lg_ctas;
      bf16* out = static_cast<bf16*>(a.out) + ((size_t)walk.b * g.Hq + (size_t)walk.kvh() * G) * D + (rank << lg_rows);
      for (int i = threadIdx.x & 127; i < G << lg_rows; i += 128) {
        const int h = i >> lg_rows;
        float M = -INFINITY, L = 0.f, O = 0.f;
#pragma unroll 4
        for (int c = 0; c < n; ++c) M = fmaxf(M, recv_ml[c * 16 + h].x);
#pragma unroll 4
        for (int c = 0; c < n; ++c) {
          const float2 ml = recv_ml[c * 16 + h];
          const float w = ml.y == 0.f ? 0.f : fast_exp2(ml.x - M);
          L += ml.y == 0.f ? 0.f : scaled(ml.y, ml.x - M);
          O += w * recv[((c * G) << lg_rows) + i];
        }
        // (a sequence without a token: zeros)
        out[(size_t)h * D + (i & ((1 << lg_rows) - 1))] = __float2bfloat16_rn(walk.tiles == 0 ? 0.f : O / L);
      }
    }
  }
  __syncthreads();
  tc_fence_after();
  if (warp == kMma) tmem_dealloc(tmem, C::TMEM_COLS);
}

// cluster: CTAs of a cluster, 0: no clusters.
template <int D, bool F8, int GP, bool CL>
cudaError_t launch(const PagedDecodeArgs& a, int ctas, int cluster, cudaStream_t s) {
  using C = Lay<D, F8, GP, CL>;
  auto kernel = paged_decode_kernel<D, F8, GP, CL>;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = once_per_device(done, [&] {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
    if (e == cudaSuccess && CL) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    return e;
  });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(C::THREADS);
  cfg.dynamicSmemBytes = C::SMEM;
  cfg.stream = s;
  // its start runs under the end of the kernel before it
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = CL ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <int D, bool F8, int GP>
cudaError_t launch_split(const PagedDecodeArgs& a, int num_sms, int cluster, cudaStream_t s) {
  if (cluster > 0) return launch<D, F8, GP, true>(a, a.n_seqs * a.geom.Hkv * cluster, cluster, s);
  return launch<D, F8, GP, false>(a, num_sms, 0, s);
}

template <int D, bool F8>
cudaError_t launch_heads(const PagedDecodeArgs& a, int num_sms, int cluster, cudaStream_t s) {
  const int G = a.geom.G;
  if (G <= 2) return launch_split<D, F8, 2>(a, num_sms, cluster, s);
  if (G <= 4) return launch_split<D, F8, 4>(a, num_sms, cluster, s);
  if (G <= 8) return launch_split<D, F8, 8>(a, num_sms, cluster, s);
  return launch_split<D, F8, 16>(a, num_sms, cluster, s);
}

}  // namespace pdec
}  // namespace aoh
