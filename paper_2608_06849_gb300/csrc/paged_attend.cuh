// Attention of a chunk of new tokens of every sequence over a paged cache, on the prefill kernel
// (prefill_tc.cuh; include/aoh.h: aoh_paged_attend). Items are folded ones (prefill_packed.cuh): all
// query heads of a KV head at some neighbouring tokens, so that a KV head's pages are read once for
// all of them; the tokens' own keys lie in the pages already. Lengths and tables are read on the device.
//
// bf16 pages go to the shared tiles by TMA, page by page. Codes of 8 bits are loaded into registers by seven
// more warps, which write bf16 tiles (code * 2^power is one exactly, so that everything behind is
// the computation on bf16 pages). That takes an item as many instructions as its softmax: where several
// items visit the same tiles, paged_api.cu has them written out as bf16 pages once, for the bf16 kernel;
// sequences that prove longer than the host took them to be are then left to this one.
//
// A chunk's items are few and unlike (a retrieval head's visit the whole prefix, a streaming one's its window), so
// that whole items leave SMs idle at the end: prefill_plan.h has them shared by clusters or cut into parts, whose
// states meet in global memory: 133 KB a part of d_head 128, most of which L2 holds (456 parts of a chunk of 2,048 rows, 61 MB
// of states: 41 MB written to HBM, of which 15 are the outputs).
#pragma once

#include "paged_rows.cuh"
#include "prefill_packed_launch.cuh"

namespace aoh {
namespace pf {

// F8: pages of 8 bits.
template <bool F8>
struct PagedArgs : PagedAttendArgs {};

// The tokens of sequence b, within what its table holds.
__device__ __forceinline__ int attend_len(const PagedAttendArgs& a, int b, bool tells) {
  const int n = __ldcg(a.lens + b);
  if (n >= 0 && n <= a.holds) return n;
  if (tells) atomicOr(a.err, kErrPages);
  return n < 0 ? 0 : a.holds;
}

struct PagedItem : FoldedItem {
  int index, b, first;  // among the sequences with rows, the sequence's number, its first page written out
  // (of the CTA's threads one, or each with tells, reports a length out of range)
  __device__ __forceinline__ PagedItem(const PagedAttendArgs& a, uint64_t code, bool tells = false)
      : PagedItem(a, code, a.seqs.of((int)(code >> 34)), tells || threadIdx.x == 0) {}
  __device__ __forceinline__ PagedItem(const PagedAttendArgs& a, uint64_t code, const int4& s, bool tells)
      : PagedItem(a, code, s, attend_len(a, s.z, tells)) {}
  __device__ __forceinline__ PagedItem(const PagedAttendArgs& a, uint64_t code, const int4& s, int keys)
      : FoldedItem(a, code, make_int4(s.x, s.y, 0, keys)), index((int)(code >> 34)), b(s.z), first(s.w) {}
  // whether another kernel of the call computes it
  __device__ __forceinline__ bool elsewhere(const PagedAttendArgs& a) const {
    if (!a.written) return false;
    return (klen <= (a.seqs.of(index + 1).w - first) * kBN) == (a.table != nullptr);
  }
  // the page with position pos
  __device__ __forceinline__ int page_of(const PagedAttendArgs& a, int pos) const {
    const int slot = pos >> a.pool.lg_ps;
    return a.table ? __ldg(a.table + (size_t)b * a.table_stride + slot) : first + slot;
  }
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
  // 8 bits: MMA issuer (warp 1) and three warps that convert, two groups of softmax, four more that convert
  static constexpr int kThreads = F8 ? 512 : pf::kThreads, kSoftmax = F8 ? 4 : 2;
};

// bf16: a tile's pages in the lanes of the producer.
template <int D>
struct PageWalk<PagedArgs<false>, D> {
  using C = PfCfg<D>;
  int lane, rows, page;  // page: the lane's, at key lane * rows, or -1: out of range
  int ahead;             // the entry of the tile after it, which is on its way meanwhile
  bool has;              // whether the lane has a page with keys
  __device__ __forceinline__ PageWalk(int lane_, const PagedAttendArgs& a)
      : lane(lane_), rows(a.pool.ps), page(-1), ahead(-1), has(false) {}
  __device__ __forceinline__ int key() const { return lane * rows; }
  __device__ __forceinline__ bool position(const PagedItem& t, int i, int* pos) const {
    *pos = t.chunk_tile(i) * kBN + key();
    return key() < kBN && *pos < t.klen;
  }
  // visited tile i of the item, the first that is looked up or the one after the last that was
  __device__ __forceinline__ int entry(const PagedAttendArgs& a, const PagedItem& t, int i) const {
    int pos;
    return position(t, i, &pos) ? t.page_of(a, pos) : -1;
  }
  __device__ __forceinline__ void fetch(const PagedAttendArgs& a, const PagedItem& t, int i) { ahead = entry(a, t, i); }
  __device__ __forceinline__ void look(const PagedAttendArgs& a, const PagedItem& t, int i, bool more) {
    int pos;
    has = position(t, i, &pos);
    page = ahead;
    if (more) fetch(a, t, i + 1);
    if (has && (unsigned)page >= (unsigned)a.pool.n_pages) {
      page = -1;
      atomicOr(a.err, kErrPages);
    }
  }
  // K (sel 0) or V of the tile: the pages that hold keys; the warp
  __device__ __forceinline__ void load(const PagedArgs<false>& a, const PagedItem& t, int sel, uint8_t* dst, uint64_t* bar) const {
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

// 8 bits: a warp's way through the groups of 16 rows of an item's K and V tiles, eight of a tile, every
// kConvert-th its own. A group lies in one page. kAhead groups are in registers or on their way, the entry
// of the table for the one behind them too.
template <int D>
struct CodeWalk<PagedArgs<true>, D> {
  using A = PagedArgs<true>;
  using C = PfCfg<D>;
  static constexpr int kAhead = 3;
  struct Group {
    uint2 x[4][D / 64];  // 8 codes of every fourth row, in both boxes
    int power;           // of row lane % 16
    int rows;            // rows that hold keys (others are zeros)
  };
  Group group[kAhead];
  int page;  // of the next group to be loaded
  // Group n: K or V of visited tile first + n / 16, rows 16 (n % 8) on.
  __device__ __forceinline__ static int position(const PagedItem& t, int first, int n) {
    return t.chunk_tile(first + (n >> 4)) * kBN + (n & 7) * 16;
  }
  __device__ __forceinline__ void look(const A& a, const PagedItem& t, int first, int n, int all) {
    page = -1;
    if (n >= all) return;
    const int pos = position(t, first, n);
    if (pos < t.klen) page = t.page_of(a, pos);
  }
  // A lane 8 codes of a row at a time, 8 lanes a row of a box, so that the lanes that store a row
  // of a tile touch every bank once.
  __device__ __forceinline__ void load(const A& a, const PagedItem& t, int first, int n, int all, int lane, Group& g) {
    g.rows = 0;
    if (n >= all) return;
    const int pos = position(t, first, n), sel = n >> 3 & 1, lg = a.pool.lg_ps;
    if (pos >= t.klen) return;
    if ((unsigned)page >= (unsigned)a.pool.n_pages) {
      if (lane == 0) atomicOr(a.err, kErrPages);
      return;
    }
    g.rows = t.klen - pos;
    const int row = pos & (a.pool.ps - 1);
    const uint8_t* from = static_cast<const uint8_t*>(a.pool.data) +
                          (((((size_t)page * 2 + sel) * a.pool.Hkv + t.kvh) << lg) + row + (lane >> 3)) * D + (lane & 7) * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int k = 0; k < D / 64; ++k) g.x[i][k] = __ldg(reinterpret_cast<const uint2*>(from + i * 4 * D + k * 64));
    g.power = __ldg(a.pool.powers + (((((size_t)page * a.pool.Hkv + t.kvh) * 2 + sel) << lg) + row + (lane & 15)));
  }
  // Group n as bf16 rows of its tile.
  __device__ __forceinline__ static void put(const Group& g, int n, uint8_t* tile, int lane) {
    const int sub = lane >> 3, c = lane & 7, row0 = (n & 7) * 16;
    // row at of the tile: its pieces c ^ (at & 7)
    uint8_t* to = tile + (row0 + sub) * 128 + ((c ^ sub) << 4);
    const int other = (c ^ sub ^ 4) * 16 - (c ^ sub) * 16;  // rows 4 on
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float scale = __uint_as_float((uint32_t)(127 + __shfl_sync(0xffffffffu, g.power, i * 4 + sub)) << 23);
      const float2 f2 = make_float2(scale, scale);
#pragma unroll
      for (int k = 0; k < D / 64; ++k) {
        uint32_t y[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint32_t word = u < 2 ? g.x[i][k].x : g.x[i][k].y, two = u & 1 ? word >> 16 : word & 0xffffu;
          const float2 f = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3)));
          const float2 z = __fmul2_rn(f, f2);
          y[u] = float2_to_bf16x2(z.x, z.y);
        }
        if (g.rows < 16 && i * 4 + sub >= g.rows) y[0] = y[1] = y[2] = y[3] = 0;
        *reinterpret_cast<uint4*>(to + i * 4 * 128 + (i & 1 ? other : 0) + k * C::BOX) = make_uint4(y[0], y[1], y[2], y[3]);
      }
    }
  }
  // All groups of the warp, the w-th of kConvert, into the ring of tiles.
  __device__ __forceinline__ void run(const A& a, const PagedItem& t, int first, int n_tiles, int w, uint8_t* ring,
                                      uint64_t* kv_full, uint64_t* kv_empty, int lane, volatile int* abort_flag) {
    const int all = 16 * n_tiles;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      look(a, t, first, w + k * kConvert, all);
      load(a, t, first, w + k * kConvert, all, lane, group[k]);
    }
    look(a, t, first, w + kAhead * kConvert, all);
    int n = w;
    while (true) {
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (n >= all) return;
        const int it = n >> 3, st = it % kNS;
        if (it >= kNS && !__all_sync(0xffffffffu, wait_bar(&kv_empty[st], ((it / kNS) & 1) ^ 1, a.err, abort_flag))) return;
        put(group[k], n, ring + st * C::KVBYTES, lane);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&kv_full[st]);
        load(a, t, first, n + kAhead * kConvert, all, lane, group[k]);
        n += kConvert;
        look(a, t, first, n + kAhead * kConvert, all);
      }
    }
  }
};

// The lane's numbers of key j of K (sel 0) or V (repair_rows).
template <int D>
__device__ __forceinline__ void load_key(const PagedAttendArgs& a, const PagedItem& t, int j, int sel, int lane,
                                         float (&to)[D / 32]) {
  // (of written-out pages the table is their numbers, one after the other)
  if (a.table) {
    rows::load_key<D>(a.pool, a.table + (size_t)t.b * a.table_stride, t.kvh, j, sel, lane, to);
  } else {
    const size_t at = ((((size_t)t.page_of(a, j) * 2 + sel) * a.pool.Hkv + t.kvh) * kBN + (j & (kBN - 1))) * D;
    load_numbers<D>(static_cast<const bf16*>(a.pool.data) + at + lane * (D / 32), to);
  }
}

// Items of a launch at most: beside the arguments of such a call 3,840 are too many.
constexpr int kAttendByValue = 3200;

// The items of a call: `split` CTAs each (1: one), as launch_prefill_folded has them.
template <bool F8, int D>
cudaError_t launch_attend(const PagedAttendArgs& args, const std::vector<uint64_t>& items, int split, bool is_short, int num_sms,
                          cudaStream_t s) {
  PagedArgs<F8> a;
  static_cast<PagedAttendArgs&>(a) = args;
  if (split > 1)
    return launch_items<PagedArgs<F8>, D, kSplit, kPrefillSplitMost>(a, items.data(), (int)items.size(), split, s);
  const size_t n = items.size();
  if (a.states) return launch_items<PagedArgs<F8>, D, kJoined, kJoinedEntries>(a, items.data(), (int)n, 1, s);
  // (a CTA holds the sequences of kShortItems items)
  if (n > (size_t)kShortItems * num_sms && kAttendByValue > kShortItems * num_sms) is_short = false;
  if constexpr (!F8)
    for (size_t i = 0; is_short && i < n; i += kAttendByValue) {
      const int m = (int)(n - i < (size_t)kAttendByValue ? n - i : (size_t)kAttendByValue);
      a.follows = i > 0;
      const cudaError_t e = launch_short<PagedArgs<F8>, D, kAttendByValue>(a, items.data() + i, m, num_sms, s);
      if (e != cudaSuccess || i + m == n) return e;
    }
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
