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
// with m the running maximum of s_j + ev_j, so that w_j is the size of key j's contribution. q
// (8 significant bits) is the sum of two e4m3 numbers (4 bits each): exactly, down to 2^-17 of the
// row's largest. A weight is the sum of three e5m2 numbers (3 bits each, rounded to
// nearest: 2^-9 of it, as good as bf16, at 2^-16 .. 2^15.8, so a key counts down to 2^-28 of
// the heaviest). The parts are columns of the MMAs, which have sixteen at least.
//
// The items, (sequence, KV head), are cut into tiles of 64 KB of K and V; all tiles, item
// after item, are dealt to the CTAs in equal runs, so that every CTA streams as many bytes
// whatever the lengths. A CTA joins the runs of an item that it shares: each stores its
// state (O, max, sum), and the last to arrive adds them up (groups of 16 first).
// A streaming head's tiles are the pages of its sinks and then those of its window.
//
// Warps: 4 NK softmax (a thread a key of the tile), two producers, one MMA issuer.
#pragma once

#include <cuda_fp8.h>
#include <math.h>

#include "common.cuh"
#include "internal.h"
#include "tc.cuh"

namespace aoh {
namespace pdec {

using bf16 = __nv_bfloat16;
constexpr int kNS = 3;              // ring stages
constexpr int kGroup = 16;          // states joined at a time
constexpr int kLensCap = 1024;      // lengths mirrored in shared memory

// Shapes of one head size, format and (padded) number of query heads a KV head.
template <int D_, bool F8_, int GP_>
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
  static constexpr int NK = HALF / GRP;                    // groups of a tile
  static constexpr int KEYS = NK * 128;
  static constexpr int MB = 128 / D;                       // groups side by side in a P V MMA
  static constexpr int SETS = NK / MB;
  static constexpr int PARTS = F8 ? 3 : 1;                 // columns of a weight
  static constexpr int NPV = (MB * PARTS * GP + 15) / 16 * 16;
  static constexpr int SN = F8 ? (2 * GP + 15) / 16 * 16 : 16;
  static constexpr int SBUF = NK * SN;                     // TMEM columns of one tile's S
  static constexpr int OCOL = 2 * SBUF;
  static constexpr int TMEM_COLS = next_pow2(cmax(OCOL + NPV, 32));
  static constexpr int SOFT = 128 * NK;                    // softmax threads
  static constexpr int THREADS = SOFT + 96;
  static constexpr int QBLK = SN * ROWB, QBUF = DBLK * QBLK;
  static constexpr int PBLK = NPV * 128;                   // weights of 128 bytes of keys
  static constexpr int PSET = PBLK * ES;
  static constexpr int PBUF = SETS * PSET;
  static constexpr int POWB = F8 ? 2 * KEYS : 0;           // a stage's powers
  static constexpr int FIXED = kNS * STAGE + 2 * QBUF + kNS * POWB + 8192 + 2048;
  static constexpr int NPB = FIXED + 2 * PBUF <= 225 * 1024 ? 2 : 1;
  static constexpr int OFF_Q = kNS * STAGE;
  static constexpr int OFF_P = OFF_Q + 2 * QBUF;
  static constexpr int OFF_POW = OFF_P + NPB * PBUF;
  static constexpr int OFF_RED = OFF_POW + kNS * POWB;     // [2][GP][4 NK] warp maxima
  static constexpr int OFF_LSUM = OFF_RED + 2 * GP * 4 * NK * 4;  // [4 NK][GP]
  static constexpr int OFF_X = OFF_LSUM + 4 * NK * GP * 4;  // [GP][64] the upper rows of O (d_head 64)
  static constexpr int OFF_QF = OFF_X + (D == 64 ? GP * 64 * 4 : 0);  // [2][16] factors of the scores
  static constexpr int OFF_BAR = OFF_QF + 128;
  static constexpr int NBAR = 3 * kNS + 10 + 2;
  static constexpr int OFF_MISC = OFF_BAR + NBAR * 8;
  static constexpr int OFF_LENS = OFF_MISC + 64 + 8 * 32;
  static constexpr int SMEM = OFF_LENS + kLensCap * 4 + 1024;
  // kind::f16 with bf16, or kind::f8f6f4 with e4m3 (weights: e5m2); V is MN-major
  static constexpr uint32_t IDESC_S = F8 ? idesc_f8(128, SN, false, 0) : idesc_bf16(128, SN, false, false);
  static constexpr uint32_t IDESC_PV = F8 ? idesc_f8(128, NPV, true, 1) : idesc_bf16(128, NPV, false, true);
  static constexpr float kRaise = F8 ? 12.f : 0.f;         // weights are 2^(s - m + kRaise)
  static constexpr float kLag = F8 ? 3.75f : 8.f;          // the maximum follows the keys' once it is so far behind
  static_assert(SMEM <= 232448, "shared memory");
  static_assert(OFF_P % 1024 == 0 && PBLK % 1024 == 0 && QBLK % 1024 == 0, "operand alignment");
  static_assert(TMEM_COLS <= 512, "TMEM columns");
};

// An item: the keys of one KV head of a sequence that its queries see, as tiles.
struct Item {
  int len, kvh, w0, gslot, gap, tiles;
  bool strm;
};
// Head k of a sequence of len tokens, retrieval heads before streaming ones.
// LG: log2 of the keys of a tile.
template <int LG>
__device__ __forceinline__ Item make_item(const PagedDecodeArgs& a, int len, int k) {
  const CacheGeom& g = a.geom;
  Item t;
  t.len = len;
  t.strm = k >= g.n_r;
  t.kvh = t.strm ? g.s_head[k - g.n_r] : g.r_head[k];
  t.w0 = t.gslot = t.gap = 0;
  const int lg = a.pool.lg_ps;
  if (t.strm && len - g.W > g.S) {
    t.w0 = len - g.W;
    t.gslot = (g.S + a.pool.ps - 1) >> lg;
    t.gap = max((t.w0 >> lg) - t.gslot, 0);
  }
  const int slots = (int)(((long long)len + a.pool.ps - 1) >> lg) - t.gap;
  t.tiles = (slots + (1 << (LG - lg)) - 1) >> (LG - lg);
  return t;
}
// Page of the item (a slot) -> page of the sequence.
__device__ __forceinline__ int page_of_slot(const Item& t, int slot) { return slot < t.gslot ? slot : slot + t.gap; }

// The tokens of sequence b, within what its table holds.
__device__ __forceinline__ int seq_len(const PagedDecodeArgs& a, int b, bool report) {
  const int n = __ldcg(a.lens + b), most = a.table_stride << a.pool.lg_ps;
  if (n >= 0 && n <= most) return n;
  if (report) atomicOr(a.err, kErrPages);
  return n < 0 ? 0 : most;
}

// The items of a CTA's run of tiles [start, end), in order.
template <int LG>
struct Walk {
  const PagedDecodeArgs& a;
  const int* lens_s;
  long long start, end, off;  // off: the first tile of the item
  int b, k, lo, hi;
  Item t;
  __device__ __forceinline__ Walk(const PagedDecodeArgs& a_, const int* ls, long long s, long long e, int b0, long long off0)
      : a(a_), lens_s(ls), start(s), end(e), off(off0), b(b0), k(-1) {
    t.tiles = 0;
  }
  __device__ __forceinline__ int len() const { return lens_s ? lens_s[b] : seq_len(a, b, false); }
  __device__ __forceinline__ bool next() {
    while (true) {
      off += t.tiles;
      if (off >= end) return false;
      if (++k == a.geom.Hkv) {
        k = 0;
        ++b;
      }
      t = make_item<LG>(a, len(), k);
      lo = (int)(max(start, off) - off);
      hi = (int)min(end - off, (long long)t.tiles);
      if (lo < hi) return true;
    }
  }
};

__device__ __forceinline__ int cta_of(long long x, long long total, int P) {
  return (int)(((x + 1) * (long long)P - 1) / total);
}

// A state of an item that CTAs share: O [G][D], then the maxima and sums [G] each. Slots of
// a CTA: 0, 1 the state of its first and of its last item, 2, 3 the states joined by the group
// that it heads.
__host__ __device__ constexpr int state_floats(int D) { return 16 * (D + 2); }
__device__ __forceinline__ float* state_slot(const PagedDecodeArgs& a, int cta, int slot, int D) {
  return a.states + ((size_t)cta * 4 + slot) * state_floats(D);
}

// Adds up n states and stores the outputs (out) or the sum (dst); 128 threads.
template <int D, class Part>
__device__ __forceinline__ void join(int n, Part part, int G, bf16* out, float* dst) {
  constexpr int U = 8;
  for (int v = threadIdx.x; v < G * (D / 4); v += 128) {
    const int h = v / (D / 4);
    float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
    float M = -INFINITY, L = 0.f;
    for (int j = 0; j < n; j += U) {
      float4 x[U];
      float mj[U], lj[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float* p = part(min(j + u, n - 1));
        x[u] = __ldcg(reinterpret_cast<const float4*>(p) + v);
        mj[u] = __ldcg(p + G * D + h);
        lj[u] = __ldcg(p + G * D + G + h);
      }
      float top = M;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (j + u < n) top = fmaxf(top, mj[u]);
      const float sc = M == -INFINITY ? 0.f : fast_exp2(M - top);
      O.x *= sc;
      O.y *= sc;
      O.z *= sc;
      O.w *= sc;
      L *= sc;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (j + u >= n || mj[u] == -INFINITY) continue;
        const float w = fast_exp2(mj[u] - top);
        O.x += w * x[u].x;
        O.y += w * x[u].y;
        O.z += w * x[u].z;
        O.w += w * x[u].w;
        L += w * lj[u];
      }
      M = top;
    }
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
  const int p0 = f + (p - f) / kGroup * kGroup;
  const int size = min(kGroup, last - p0 + 1), groups = (last - f) / kGroup + 1;
  const int gslot = p0 == f ? 1 : 0;
  auto arrive = [&](uint32_t* counter, int of) {
    named_barrier_sync(2, 128);
    if (threadIdx.x == 0) {
      const bool done = atom_add_acq_rel_gpu(counter, 1u) == (uint32_t)(of - 1);
      if (done) *counter = 0u;
      *flag = done;
    }
    named_barrier_sync(2, 128);
    return *flag != 0;
  };
  if (!arrive(&a.counters[3 * p0 + gslot], size)) return;
  auto own = [&](int j) { return state_slot(a, p0 + j, p0 + j == f ? 1 : 0, D); };
  if (groups == 1) {
    join<D>(size, own, G, out, nullptr);
    return;
  }
  join<D>(size, own, G, nullptr, state_slot(a, p0, 2 + gslot, D));
  if (!arrive(&a.counters[3 * f + 2], groups)) return;
  join<D>(groups, [&](int j) { return state_slot(a, f + j * kGroup, 2 + (j == 0 ? 1 : 0), D); }, G, out, nullptr);
}

// Powers of two as floats.
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

template <int D, bool F8, int GP>
__global__ void __launch_bounds__(Lay<D, F8, GP>::THREADS, 1)
    paged_decode_kernel(const __grid_constant__ PagedDecodeArgs a) {
  using C = Lay<D, F8, GP>;
  constexpr int NK = C::NK, LG = NK == 1 ? 7 : NK == 2 ? 8 : 9;
  static_assert(1 << LG == C::KEYS, "keys of a tile");
  constexpr int NT = C::THREADS, NW = C::SOFT / 32;
  constexpr int kLoadK = NW, kLoadV = NW + 1, kMma = NW + 2;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  uint8_t* sQ = smem + C::OFF_Q;
  uint8_t* sP = smem + C::OFF_P;
  int8_t* sPow = reinterpret_cast<int8_t*>(smem + C::OFF_POW);
  float* red = reinterpret_cast<float*>(smem + C::OFF_RED);
  float* lsum = reinterpret_cast<float*>(smem + C::OFF_LSUM);
  float* upper = reinterpret_cast<float*>(smem + C::OFF_X);
  float* qfac = reinterpret_cast<float*>(smem + C::OFF_QF);
  uint64_t* k_full = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);  // K and powers of a stage landed
  uint64_t* v_full = k_full + kNS;
  uint64_t* empty = v_full + kNS;
  uint64_t* s_full = empty + kNS;  // [2] S(j) in TMEM
  uint64_t* s_free = s_full + 2;   // [2] S(j) read by the softmax
  uint64_t* p_full = s_free + 2;   // [2] P(j) written
  uint64_t* p_free = p_full + 2;   // [2] O += P(j) V(j) done
  uint64_t* q_set = p_free + 2;    // [2] the item's factors written
  uint64_t* o_free = q_set + 2;    // the item's O read
  uint64_t* drain = o_free + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* flag = reinterpret_cast<volatile int*>(tmem_slot + 2);
  int* first_b = reinterpret_cast<int*>(tmem_slot + 3);
  long long* sh64 = reinterpret_cast<long long*>(smem + C::OFF_MISC + 16);  // total, first offset
  long long* wsum = reinterpret_cast<long long*>(smem + C::OFF_MISC + 64);
  int* lens_s = reinterpret_cast<int*>(smem + C::OFF_LENS);

  const CacheGeom& g = a.geom;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int G = g.G, lg = a.pool.lg_ps;

  // rows of Q and P that no head fills stay zero for the whole launch
  for (int i = threadIdx.x; i < (2 * C::QBUF + C::NPB * C::PBUF) / 16; i += NT)
    reinterpret_cast<uint4*>(sQ)[i] = make_uint4(0, 0, 0, 0);
  fence_proxy_async_smem();
  if (threadIdx.x < 32) qfac[threadIdx.x] = 0.f;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kNS; ++s) {
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
    }
    mbar_init(o_free, 4);
    mbar_init(drain, 1);
    *abort_flag = 0;
    *first_b = 0;
    fence_mbar_init();
  }
  if (warp == kLoadK && lane == 0) prefetch_tmap(&a.pages);
  if (warp == kMma) {
    tmem_alloc(tmem_slot, C::TMEM_COLS);
    tmem_relinquish();
  }
  // everything earlier kernels wrote is visible from here on
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  // ---- this CTA's run: a prefix sum of the sequences' tiles
  auto seq_tiles = [&](int len) {
    long long n = 0;
    if (g.n_r > 0) n += (long long)g.n_r * make_item<LG>(a, len, 0).tiles;
    if (g.n_s > 0) n += (long long)g.n_s * make_item<LG>(a, len, g.n_r).tiles;
    return n;
  };
  const bool mirrored = a.n_seqs <= kLensCap;
  const int per = (a.n_seqs + NT - 1) / NT;
  const int b0 = min(a.n_seqs, (int)threadIdx.x * per), b1 = min(a.n_seqs, b0 + per);
  long long mine = 0;
  for (int b = b0; b < b1; ++b) {
    const int len = seq_len(a, b, blockIdx.x == 0);
    if (mirrored) lens_s[b] = len;
    mine += seq_tiles(len);
  }
  long long inc = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  if (lane == 31) wsum[warp] = inc;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  long long before = inc - mine, total = 0;
  for (int w = 0; w < NT / 32; ++w) {
    if (w < warp) before += wsum[w];
    total += wsum[w];
  }
  const int P = (int)min((long long)gridDim.x, total), p = blockIdx.x;
  const long long start = p < P ? (long long)p * total / P : total, end = p < P ? (long long)(p + 1) * total / P : total;
  if (before <= start && start < before + mine) {
    int b = b0;
    while (true) {
      const long long n = seq_tiles(mirrored ? lens_s[b] : seq_len(a, b, false));
      if (start < before + n) break;
      before += n;
      ++b;
    }
    *first_b = b;
    sh64[0] = before;
  }
  // sequences without a token
  for (int b = p; b < a.n_seqs; b += gridDim.x)
    if ((mirrored ? lens_s[b] : seq_len(a, b, false)) == 0)
      for (int i = threadIdx.x; i < g.Hq * D / 8; i += NT)
        reinterpret_cast<uint4*>(static_cast<bf16*>(a.out) + (size_t)b * g.Hq * D)[i] = make_uint4(0, 0, 0, 0);
  __syncthreads();
  Walk<LG> walk(a, mirrored ? lens_s : nullptr, start, end, *first_b, p < P ? sh64[0] : total);

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
      const Item& t = walk.t;
      const int32_t* row = a.table + (size_t)walk.b * a.table_stride;
      const int slots = (int)(((long long)t.len + a.pool.ps - 1) >> lg) - t.gap;
      for (int j = walk.lo; j < walk.hi; ++j, ++it) {
        const int st = it % kNS;
        const int n = min(spt, slots - j * spt);
        int page = 0;
        if (lane < n) page = __ldg(row + page_of_slot(t, j * spt + lane));
        const bool bad = (unsigned)page >= (unsigned)a.pool.n_pages;
        if (bad && !is_v) atomicOr(a.err, kErrPages);
        if (it >= kNS) ok = __all_sync(0xffffffffu, wait_bar(&empty[st], ((it / kNS) & 1) ^ 1, a.err, abort_flag));
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
                           a.pool.powers + (((size_t)pg * g.Hkv + t.kvh) << (lg + 1)) + (c & ((1 << (lg - 3)) - 1)) * 16);
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
          const int block = bad ? 2 * g.Hkv * a.pool.n_pages : (page * 2 + (is_v ? 1 : 0)) * g.Hkv + t.kvh;
#pragma unroll
          for (int db = 0; db < C::DBLK; ++db) tma_load_3d(dst + db * C::BOX, &a.pages, db * 64, 0, block, &full[st]);
        }
        __syncwarp();
      }
    }
    // every issued copy lands before the CTA can exit
    if (F8) asm volatile("cp.async.wait_all;" ::: "memory");
    if (lane == 0)
      for (int j = it > kNS ? it - kNS : 0; j < it; ++j) drain_wait(&full[j % kNS], (j / kNS) & 1, a.err);
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
    int it = 0, ofw = 0, item = 0;
    bool ok = true;
    auto wait_warp = [&](uint64_t* bar, uint32_t parity) {
      if (ok) ok = __all_sync(0xffffffffu, wait_bar(bar, parity, a.err, abort_flag));
      return ok;
    };
    // the O of the first n items has been read
    auto wait_ofree = [&](int n) {
      for (; ok && ofw < n; ++ofw) wait_warp(o_free, ofw & 1);
    };
    auto issue_pv = [&](int j, bool first, int item) {
      wait_warp(&v_full[j % kNS], (j / kNS) & 1);
      wait_warp(&p_full[j & 1], (j >> 1) & 1);
      if (first) wait_ofree(item);
      if (!ok) return;
      if (elect_one()) {
        tc_fence_after();
        const uint64_t v_desc = v_desc0 + (uint32_t)((j % kNS) * sdesc_step(C::STAGE));
        const uint64_t p_desc = p_desc0 + (uint32_t)((j % C::NPB) * sdesc_step(C::PBUF));
#pragma unroll
        for (int z = 0; z < C::SETS; ++z)
#pragma unroll
          for (int kk = 0; kk < PSTEPS; ++kk)
            tc_mma_any<F8>(tmem + C::OCOL, v_desc + sdesc_step(z * C::MB * C::GRP + kk * (32 / C::ES) * C::ROWB),
                           p_desc + sdesc_step(z * C::PSET + (kk >> 2) * C::PBLK + (kk & 3) * 32), C::IDESC_PV,
                           first && z == 0 && kk == 0 ? 0u : 1u);
        tc_commit(&p_free[j & 1]);
        tc_commit(&empty[j % kNS]);
      }
      __syncwarp();
    };
    constexpr int CPR = D / 8;                    // 16-byte pieces of a query row
    constexpr int QV = (GP * CPR + 31) / 32;
    while (ok && walk.next()) {
      // the item's queries: piece c of the G x D block; CPR neighbouring lanes hold a row
      uint4 qr[QV];
      const bf16* qg = static_cast<const bf16*>(a.q) + (size_t)walk.b * a.q_stride + (size_t)walk.t.kvh * G * D;
#pragma unroll
      for (int i = 0; i < QV; ++i) {
        const int c = lane + 32 * i;
        qr[i] = c < G * CPR ? *reinterpret_cast<const uint4*>(qg + c * 8) : make_uint4(0, 0, 0, 0);
      }
      // buffer item & 1 was last read by the MMAs of item - 2
      wait_ofree(item - 1);
      if (!ok) break;
      uint8_t* qs = sQ + (item & 1) * C::QBUF;
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
      for (int j = walk.lo; j < walk.hi; ++j, ++it) {
        const int st = it % kNS;
        wait_warp(&k_full[st], (it / kNS) & 1);
        if (it >= 2) wait_warp(&s_free[it & 1], ((it >> 1) - 1) & 1);
        if (!ok) break;
        if (elect_one()) {
          tc_fence_after();
          const uint64_t k_desc = k_desc0 + (uint32_t)(st * sdesc_step(C::STAGE));
          const uint64_t q_desc = q_desc0 + (uint32_t)((item & 1) * sdesc_step(C::QBUF));
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
        // P V of the tile before, behind this tile's S
        if (j > walk.lo) issue_pv(it - 1, j - 1 == walk.lo, item);
      }
      if (ok) issue_pv(it - 1, walk.hi - 1 == walk.lo, item);
      ++item;
    }
    if (elect_one()) tc_commit(drain);
    __syncwarp();
    drain_wait(drain, 0, a.err);
    __syncwarp();
  } else {
    // ------------------------------------------------------------ softmax
    const int t = threadIdx.x;            // key of the tile
    const int y = t >> 7, r = t & 127;    // its group, and its row there (and row r of O^T, threads 0-127)
    const uint32_t tl = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    int it = 0, item = 0;
    // ok: the softmax threads' common verdict, set at a barrier; local_ok: this thread's waits since
    bool ok = true, local_ok = true;
    while (ok && walk.next()) {
      const Item& w = walk.t;
      float m[GP], l[GP];
#pragma unroll
      for (int h = 0; h < GP; ++h) {
        m[h] = -INFINITY;
        l[h] = 0.f;
      }
      for (int j = walk.lo; j < walk.hi; ++j, ++it) {
        const int x = it & 1, st = it % kNS;
        const long long vrow = ((long long)j << LG) + t;
        const int slot = (int)(vrow >> lg);
        const long long pos = ((long long)page_of_slot(w, slot) << lg) + (t & (a.pool.ps - 1));
        const bool see = pos < w.len && (!w.strm || pos < g.S || pos >= w.w0);
        const unsigned hidden = __ballot_sync(0xffffffffu, !see);
        if (F8) local_ok = wait_bar(&k_full[st], (it / kNS) & 1, a.err, abort_flag) && local_ok;
        int ek = 0, ev = 0;
        if constexpr (F8) {
          const int8_t* pw = sPow + st * C::POWB + ((t >> lg) << (lg + 1)) + (t & (a.pool.ps - 1));
          ek = see ? pw[0] : 0;
          ev = see ? pw[a.pool.ps] : 0;
        }
        if (hidden) {
          // V rows that no weight may meet (0 times a NaN is NaN), while S is formed
          constexpr int CH = C::ROWB / 16;
          local_ok = wait_bar(&v_full[st], (it / kNS) & 1, a.err, abort_flag) && local_ok;
#pragma unroll
          for (int db = 0; db < C::DBLK; ++db) {
            uint4* v4 = reinterpret_cast<uint4*>(smem + st * C::STAGE + C::HALF + y * C::GRP + db * C::BOX + (warp & 3) * 32 * C::ROWB);
            for (int c = lane; c < 32 * CH; c += 32)
              if (hidden >> (c / CH) & 1) v4[c] = make_uint4(0, 0, 0, 0);
          }
        }
        if (F8 && j == walk.lo)
          local_ok = wait_bar(&q_set[item & 1], (item >> 1) & 1, a.err, abort_flag) && local_ok;
        local_ok = wait_bar(&s_full[x], (it >> 1) & 1, a.err, abort_flag) && local_ok;
        tc_fence_after();
        constexpr int SC = F8 ? cmax(2 * GP, 8) : cmax(GP, 8);  // columns read
        uint32_t v[SC];
        tmem_ld(tl + x * C::SBUF + y * C::SN, v);
        tmem_ld_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s_free[x]);
        float s[GP];
        const float kf = pow2i(ek);
#pragma unroll
        for (int h = 0; h < GP; ++h) {
          if constexpr (F8)
            s[h] = fmaf(__uint_as_float(v[h]) + __uint_as_float(v[GP + h]), kf * qfac[(item & 1) * 16 + h], (float)ev);
          else
            s[h] = __uint_as_float(v[h]) * a.scale_log2;
          if (!see) s[h] = -INFINITY;
        }
        // the running maximum moves only when a key is far above it; all threads agree
        float wm[GP];
        bool below = local_ok;
#pragma unroll
        for (int h = 0; h < GP; ++h) {
          wm[h] = warp_max(s[h]);
          below = below && wm[h] <= m[h] + C::kLag;
        }
        const bool first = j == walk.lo;
        bool resc = false;
        float alpha[GP];
        if (!named_barrier_and(1, C::SOFT, below && !first)) {
          float* rx = red + x * (GP * NW);
          if (lane == 0) {
#pragma unroll
            for (int h = 0; h < GP; ++h) rx[h * NW + warp] = wm[h];
          }
          ok = named_barrier_and(1, C::SOFT, local_ok);
          if (!ok) break;
#pragma unroll
          for (int h = 0; h < GP; ++h) {
            float top = -INFINITY;
#pragma unroll
            for (int u = 0; u < NW; u += 4) {
              const float4 f = *reinterpret_cast<const float4*>(rx + h * NW + u);
              top = fmaxf(top, fmaxf(fmax3f(f.x, f.y, f.z), f.w));
            }
            alpha[h] = 1.f;
            if (first) {
              m[h] = top;
            } else if (top > m[h] + C::kLag) {
              alpha[h] = m[h] == -INFINITY ? 0.f : fast_exp2(m[h] - top);
              m[h] = top;
              l[h] *= alpha[h];
              resc = true;
            }
          }
        }
        // the P buffer is free once O += P(it - NPB) V is done
        if (it >= C::NPB)
          local_ok = wait_bar(&p_free[(it - C::NPB) & 1], ((it - C::NPB) >> 1) & 1, a.err, abort_flag) && local_ok;
        if (resc && y == 0) {
          // row r of O^T, once O += P(it - 1) V has landed
          local_ok = wait_bar(&p_free[x ^ 1], ((it - 1) >> 1) & 1, a.err, abort_flag) && local_ok;
          tc_fence_after();
#pragma unroll
          for (int q = 0; q < C::MB * C::PARTS; ++q) {
            uint32_t o[cmax(GP, 8)];
            tmem_ld(tl + C::OCOL + q * GP, o);
            tmem_ld_wait();
#pragma unroll
            for (int h = 0; h < GP; ++h) o[h] = __float_as_uint(__uint_as_float(o[h]) * alpha[h]);
            tmem_st_n<GP>(tl + C::OCOL + q * GP, o);
          }
          tmem_st_wait();
        }
        float pr[GP];
#pragma unroll
        for (int h = 0; h < GP; ++h) pr[h] = see ? fast_exp2(s[h] - m[h] + C::kRaise) : 0.f;
        // weights of key r of group y -> column r of the K-major [NPV][128 keys] buffer of its set
        uint8_t* pb = sP + (it % C::NPB) * C::PBUF + (y / C::MB) * C::PSET;
        const int n0 = (y % C::MB) * GP;
        if constexpr (F8) {
          const float un = pow2i(-ev);
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
        fence_proxy_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[x]);
      }
      if (!ok) break;

      // ---- the item's state: row r of O^T (threads 0-127), m, and l summed over the keys
#pragma unroll
      for (int h = 0; h < GP; ++h) {
        float sum = l[h];
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) lsum[warp * GP + h] = sum;
      }
      float o[GP];
      if (y == 0) {
        const int last = it - 1;
        local_ok = wait_bar(&p_free[last & 1], (last >> 1) & 1, a.err, abort_flag) && local_ok;
        tc_fence_after();
#pragma unroll
        for (int q = 0; q < C::PARTS; ++q) {
          uint32_t part[cmax(GP, 8)];
          tmem_ld(tl + C::OCOL + (q * C::MB + r / D) * GP, part);
          tmem_ld_wait();
#pragma unroll
          for (int h = 0; h < GP; ++h) o[h] = (q == 0 ? 0.f : o[h]) + __uint_as_float(part[h]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(o_free);
        if (D == 64 && r >= 64) {
#pragma unroll
          for (int h = 0; h < GP; ++h) upper[h * 64 + r - 64] = o[h];
        }
      }
      ok = named_barrier_and(1, C::SOFT, local_ok);
      ++item;
      if (!ok) break;
      if (y != 0) continue;
      if (D == 64 && r < 64) {
#pragma unroll
        for (int h = 0; h < GP; ++h) o[h] += upper[h * 64 + r];
      }
      float L[GP];
#pragma unroll
      for (int h = 0; h < GP; ++h) {
        L[h] = 0.f;
#pragma unroll
        for (int u = 0; u < NW; ++u) L[h] += lsum[u * GP + h];
      }
      bf16* out = static_cast<bf16*>(a.out) + ((size_t)walk.b * g.Hq + (size_t)w.kvh * G) * D;
      const int f = cta_of(walk.off, total, P), lst = cta_of(walk.off + w.tiles - 1, total, P);
      if (f == lst) {
#pragma unroll
        for (int h = 0; h < GP; ++h)
          if (r < D && h < G) out[h * D + r] = __float2bfloat16_rn(o[h] / L[h]);
      } else {
        float* slot = state_slot(a, p, p == f ? 1 : 0, D);
#pragma unroll
        for (int h = 0; h < GP; ++h)
          if (h < G) {
            if (r < D) __stcg(slot + h * D + r, o[h]);
            if (r == h) {
              __stcg(slot + G * D + h, m[h]);
              __stcg(slot + G * D + G + h, L[h]);
            }
          }
        join_item<D>(a, p, f, lst, G, out, flag);
      }
      named_barrier_sync(2, 128);  // `upper` and the flag have been read
    }
  }

  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kMma) tmem_dealloc(tmem, C::TMEM_COLS);
}

template <int D, bool F8, int GP>
cudaError_t launch(const PagedDecodeArgs& a, int num_sms, cudaStream_t s) {
  using C = Lay<D, F8, GP>;
  auto kernel = paged_decode_kernel<D, F8, GP>;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = once_per_device(
      done, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM); });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)num_sms);
  cfg.blockDim = dim3(C::THREADS);
  cfg.dynamicSmemBytes = C::SMEM;
  cfg.stream = s;
  // its start runs under the end of the kernel before it
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <int D, bool F8>
cudaError_t launch_heads(const PagedDecodeArgs& a, int num_sms, cudaStream_t s) {
  const int G = a.geom.G;
  if (G <= 2) return launch<D, F8, 2>(a, num_sms, s);
  if (G <= 4) return launch<D, F8, 4>(a, num_sms, s);
  if (G <= 8) return launch<D, F8, 8>(a, num_sms, s);
  return launch<D, F8, 16>(a, num_sms, s);
}

}  // namespace pdec
}  // namespace aoh
