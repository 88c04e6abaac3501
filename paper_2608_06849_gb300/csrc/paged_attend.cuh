// Attention of a chunk of new tokens of every sequence over a paged cache, on the prefill kernel
// (prefill_tc.cuh; include/aoh.h: aoh_paged_attend). Items are folded ones (prefill_packed.cuh): all
// query heads of a KV head at some neighbouring tokens, so that a KV head's pages are read once for
// all of them; the tokens' own keys lie in the pages already. Lengths and tables are read on the device.
//
// bf16 pages go to the shared tiles by TMA, page by page. Codes of 8 bits come as they lie into a
// ring of units of 64 keys, from which four warps write bf16 tiles (code * 2^power is one exactly, so
// that everything behind is the computation on bf16 pages). With few rows the second query tile's
// place is part of the ring.
#pragma once

#include "paged_rows.cuh"
#include "prefill_packed_launch.cuh"

namespace aoh {
namespace pf {

// F8: pages of 8 bits.
template <bool F8>
struct PagedArgs : PagedAttendArgs {};

// The tokens of sequence b, within what its table holds.
__device__ __forceinline__ int attend_len(const PagedAttendArgs& a, int b) {
  const int n = __ldcg(a.lens + b), most = a.table_stride << a.pool.lg_ps;
  if (n >= 0 && n <= most) return n;
  if (threadIdx.x == 0) atomicOr(a.err, kErrPages);
  return n < 0 ? 0 : most;
}

struct PagedItem : FoldedItem {
  int b;
  __device__ __forceinline__ PagedItem(const PagedAttendArgs& a, uint64_t code)
      : PagedItem(a, code, a.seqs.of((int)(code >> 34))) {}
  __device__ __forceinline__ PagedItem(const PagedAttendArgs& a, uint64_t code, const int4& s)
      : FoldedItem(a, code, make_int4(s.x, s.y, 0, attend_len(a, s.z))), b(s.z) {}
};

template <bool F8>
struct CallOf<PagedArgs<F8>> {
  using ItemT = PagedItem;
  using MaskT = PackedMask;
  static constexpr bool kEmptyRows = true;
  static constexpr bool kRepairs = true;
  static constexpr bool kThirdS = true;
  template <int D>
  static constexpr bool kLaneRows = true;
  static constexpr bool kChained = true;
  static constexpr bool kPaged = true, kF8 = F8;
  // 8 bits: producer and MMA issuer (and two warps that fill up their group), two groups of softmax
  // and one that converts
  static constexpr int kThreads = F8 ? 512 : pf::kThreads, kSoftmax = F8 ? 4 : 2;
};

// Q_A, Q_B, units of codes, K and V tiles, powers of the units, barriers.
template <int D>
struct TcCfg<PagedArgs<true>, D> : PfCfg<D> {
  using C = PfCfg<D>;
  static constexpr int UNIT = 64 * D;                    // codes of 64 keys
  static constexpr int UNITS = 4, LONE = C::QBYTES / UNIT;  // in the ring, and in Q_B's place
  static constexpr int MOST = UNITS + LONE;
  static constexpr int OFF_RAW = C::OFF_Q + 2 * C::QBYTES;
  static constexpr int OFF_KV = OFF_RAW + UNITS * UNIT;
  static constexpr int OFF_POW = OFF_KV + kNS * C::KVBYTES;
  static constexpr int OFF_BAR = OFF_POW + MOST * 64;
  static constexpr int OFF_RING = OFF_BAR + C::NBAR * 8 + 16;  // barriers of the ring, rows without data
  static constexpr int SMEM = OFF_RING + MOST * (8 + 8 + 4) + 1024;
  static_assert(SMEM <= 232448, "shared memory");
};

// A tile's pages in the lanes of the producer: `rows` of a page (all of it, or 64 of 128) at key
// lane * rows of the tile.
template <bool F8, int D>
struct PageWalk<PagedArgs<F8>, D> {
  using C = PfCfg<D>;
  int lane, rows, page, row;  // page: the lane's, or -1: out of range; row: the first in the page
  bool has;                   // whether the lane has a page with keys
  __device__ __forceinline__ PageWalk(const PagedAttendArgs& a, const PagedItem&, int lane_)
      : lane(lane_), rows(min(a.pool.ps, F8 ? 64 : 128)), page(-1), row(0), has(false) {}
  __device__ __forceinline__ int key() const { return lane * rows; }
  // visited tile i of the item
  __device__ __forceinline__ void look(const PagedAttendArgs& a, const PagedItem& t, int i) {
    const int pos = t.chunk_tile(i) * kBN + key();
    has = key() < kBN && pos < t.klen;
    row = pos & (a.pool.ps - 1);
    page = -1;
    if (!has) return;
    page = __ldg(a.table + (size_t)t.b * a.table_stride + (pos >> a.pool.lg_ps));
    if ((unsigned)page >= (unsigned)a.pool.n_pages) {
      page = -1;
      atomicOr(a.err, kErrPages);
    }
  }
  // K (sel 0) or V of the tile: the pages that hold keys; the warp (bf16 pages)
  __device__ __forceinline__ void load(const PagedArgs<F8>& a, const PagedItem& t, int sel, uint8_t* dst, uint64_t* bar) const {
    const int n = __popc(__ballot_sync(0xffffffffu, has));
    if (lane == 0) mbar_arrive_expect_tx(bar, (uint32_t)(n * rows) * (D * 2));
    __syncwarp();
    if (has) {
      // a page out of range reads as zeros (its coordinate is past the map's end)
      const int block = page < 0 ? 2 * a.pool.Hkv * a.pool.n_pages : (page * 2 + sel) * a.pool.Hkv + t.kvh;
#pragma unroll
      for (int db = 0; db < C::DBLK; ++db) tma_load_3d(dst + db * C::BOX + key() * 128, &a.pages, db * 64, 0, block, bar);
    }
    __syncwarp();
  }
};

// The ring of codes: unit n (of the n-th half of a K or V tile) in place n % count.
template <int D>
struct RawRing<PagedArgs<true>, D> {
  using A = PagedArgs<true>;
  using L = TcCfg<A, D>;
  uint8_t* data;
  int8_t* powers;  // [MOST][64]
  uint64_t *full, *empty;
  uint32_t* bad;  // [MOST]: groups of 16 rows whose page is out of range
  int count;
  __device__ __forceinline__ RawRing(uint8_t* smem, bool lone)
      : data(smem + (lone ? L::OFF_Q + L::QBYTES : L::OFF_RAW)),
        powers(reinterpret_cast<int8_t*>(smem + L::OFF_POW)),
        full(reinterpret_cast<uint64_t*>(smem + L::OFF_RING)),
        empty(full + L::MOST),
        bad(reinterpret_cast<uint32_t*>(empty + L::MOST)),
        count(lone ? L::MOST : L::UNITS) {}
  __device__ __forceinline__ void init() {
    for (int i = 0; i < L::MOST; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], kConvert);
    }
  }
  // Unit n: half of K (sel 0) or V of the tile that `pages` looked up; the producer's warp.
  __device__ __forceinline__ bool fill(const A& a, const PagedItem& t, const PageWalk<A, D>& pages, int n, int sel, int half,
                                       int lane, volatile int* abort_flag) {
    const int r = n % count;
    if (n >= count && !__all_sync(0xffffffffu, wait_bar(&empty[r], ((n / count) & 1) ^ 1, a.err, abort_flag))) return false;
    const bool mine = pages.has && (pages.key() >> 6) == half, good = mine && pages.page >= 0;
    const int at = pages.key() & 63, rows = pages.rows;
    const uint32_t groups = mine && !good ? ((1u << (rows >> 4)) - 1u) << (at >> 4) : 0u;
    const uint32_t all_bad = __reduce_or_sync(0xffffffffu, groups);
    const int loads = __popc(__ballot_sync(0xffffffffu, good));
    if (lane == 0) {
      bad[r] = all_bad;
      mbar_arrive_expect_tx(&full[r], (uint32_t)(loads * rows) * (D + 1));
    }
    __syncwarp();
    if (good) {
      const size_t block = ((size_t)pages.page * 2 + sel) * a.pool.Hkv + t.kvh;
      bulk_g2s(data + r * L::UNIT + at * D, static_cast<const uint8_t*>(a.pool.data) + ((block << a.pool.lg_ps) + pages.row) * D,
               (uint32_t)(rows * D), &full[r]);
      const size_t power = (((size_t)pages.page * a.pool.Hkv + t.kvh) * 2 + sel) << a.pool.lg_ps;
      bulk_g2s(powers + r * 64 + at, a.pool.powers + power + pages.row, (uint32_t)rows, &full[r]);
    }
    __syncwarp();
    return true;
  }
  // Every issued copy has landed.
  __device__ __forceinline__ void drain(const A& a, int n, int lane) {
    if (lane == 0)
      for (int u = n > count ? n - count : 0; u < n; ++u) drain_wait(&full[u % count], (u / count) & 1, a.err);
    __syncwarp();
  }
  // Unit n as bf16 rows 64 * half .. of a tile (zeros from row `valid` on): warp w of kConvert writes 16 rows, a
  // lane 16 numbers at a time, as two 16-byte pieces, the lanes of the second box the other one first: the
  // lanes that store at a time touch every bank once.
  __device__ __forceinline__ bool convert(const A& a, int n, uint8_t* tile, int half, int valid, int w, int lane,
                                          volatile int* abort_flag) {
    constexpr int LPR = D / 16, STEP = 32 / LPR;
    const int r = n % count;
    if (!__all_sync(0xffffffffu, wait_bar(&full[r], (n / count) & 1, a.err, abort_flag))) return false;
    const uint32_t lost = bad[r];
    const int c = lane % LPR, flip = (c >> 2) & 1;
    uint4 x[16 / STEP];
    int e[16 / STEP];
#pragma unroll
    for (int i = 0; i < 16 / STEP; ++i) {
      const int row = w * 16 + i * STEP + lane / LPR;
      x[i] = lds128(data + r * L::UNIT + row * D + c * 16);
      e[i] = powers[r * 64 + row];
    }
#pragma unroll
    for (int i = 0; i < 16 / STEP; ++i) {
      const int row = w * 16 + i * STEP + lane / LPR, at = half * 64 + row;
      rows::Sixteen y = rows::decode(x[i], e[i]);
      if (at >= valid || (lost >> (row >> 4) & 1)) y = rows::Sixteen{};
      const uint4 p0 = make_uint4(y.w[0], y.w[1], y.w[2], y.w[3]), p1 = make_uint4(y.w[4], y.w[5], y.w[6], y.w[7]);
      uint8_t* to = tile + (c >> 2) * L::BOX + at * 128;
      const int piece = 2 * c & 7;
      *reinterpret_cast<uint4*>(to + (((piece + flip) ^ (at & 7)) << 4)) = flip ? p1 : p0;
      *reinterpret_cast<uint4*>(to + (((piece + 1 - flip) ^ (at & 7)) << 4)) = flip ? p0 : p1;
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&empty[r]);
    return true;
  }
};

// The lane's numbers of key j of K (sel 0) or V (repair_rows; a page out of range: zeros).
template <int D>
__device__ __forceinline__ void load_key(const PagedAttendArgs& a, const PagedItem& t, int j, int sel, int lane,
                                         float (&to)[D / 32]) {
  const int page = __ldg(a.table + (size_t)t.b * a.table_stride + (j >> a.pool.lg_ps)), row = j & (a.pool.ps - 1);
  if ((unsigned)page >= (unsigned)a.pool.n_pages) {
#pragma unroll
    for (int n = 0; n < D / 32; ++n) to[n] = 0.f;
    return;
  }
  const size_t at = (((((size_t)page * 2 + sel) * a.pool.Hkv + t.kvh) << a.pool.lg_ps) + row) * D + lane * (D / 32);
  if (a.pool.form == 0) {
    load_numbers<D>(static_cast<const bf16*>(a.pool.data) + at, to);
  } else {
    const int e = a.pool.powers[((((size_t)page * a.pool.Hkv + t.kvh) * 2 + sel) << a.pool.lg_ps) + row];
    const float scale = __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
    for (int n = 0; n < D / 32; n += 2) {
      const uint16_t two = *reinterpret_cast<const uint16_t*>(static_cast<const uint8_t*>(a.pool.data) + at + n);
      const float2 f = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2(two, __NV_E4M3)));
      to[n] = f.x * scale;
      to[n + 1] = f.y * scale;
    }
  }
}

// Items of a launch at most: beside the arguments of such a call 3,840 are too many.
constexpr int kAttendByValue = 3200;

// The items of a call: `split` CTAs each (1: one), as launch_prefill_folded has them.
template <bool F8, int D>
cudaError_t launch_attend(const PagedAttendArgs& args, const std::vector<uint64_t>& items, int split, cudaStream_t s) {
  PagedArgs<F8> a;
  static_cast<PagedAttendArgs&>(a) = args;
  if (split > 1)
    return launch_items<PagedArgs<F8>, D, kSplit, kPrefillSplitMost>(a, items.data(), (int)items.size(), split, s);
  const size_t n = items.size();
  if (n <= kTiny) return launch_items<PagedArgs<F8>, D, kWhole, kTiny>(a, items.data(), (int)n, 1, s);
  if (n <= kSmall) return launch_items<PagedArgs<F8>, D, kWhole, kSmall>(a, items.data(), (int)n, 1, s);
  for (size_t i = 0; i < n; i += kAttendByValue) {
    const int m = (int)(n - i < (size_t)kAttendByValue ? n - i : (size_t)kAttendByValue);
    a.follows = i > 0;
    const cudaError_t e = launch_items<PagedArgs<F8>, D, kWhole, kAttendByValue>(a, items.data() + i, m, 1, s);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace pf
}  // namespace aoh
