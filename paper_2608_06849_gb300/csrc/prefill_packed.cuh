// Packed prompts on the prefill kernels (prefill_tc.cuh, prefill_short.cuh): the rows
// of all sequences lie one behind the other, queries in one tensor, keys and values in
// others, and row i of a sequence of q_len rows and k_len keys sits at position
// k_len - q_len + i among its keys. There is no cache: every KV tile is 128 keys of the
// sequence from its first key on, whatever row of the tensor that is, so a tile's first
// key is always the tile's first row. Rows past a sequence's last key belong to the
// next one; they are hidden by the mask and, as V rows, zeroed.
//
// Two kinds of items (packed_folds chooses): 128 rows of two heads, or 256 of one, as in a
// cache's prefill (PackedArgs); or a few rows of all heads of a KV head (FoldedArgs).
#pragma once

#include "prefill_tile.cuh"

namespace aoh {
namespace pf {

struct PackedItem {
  static constexpr int n_c = 0;  // no cached tiles
  int h, kvh, q0, len, qrow, krow, klen, off, a_end, c_begin, c_end;
  bool streaming, two_heads;
  __device__ __forceinline__ PackedItem(const PackedArgs& a, uint64_t code) {
    const CacheGeom& g = a.geom;
    two_heads = (code & kPrefillTwoHeads) != 0;
    code &= ~kPrefillTwoHeads;
    h = (int)(code >> 24) & 1023;
    q0 = (int)(code & 0xffffffu) * (two_heads ? kBM : 2 * kBM);
    kvh = h / g.G;
    streaming = g.kind[kvh] != 0;
    const int4 s = a.seqs.of((int)(code >> 34));
    qrow = s.x;
    len = s.y;
    krow = s.z;
    klen = s.w;
    off = klen - len;
    const int end = max(off + min(q0 + (two_heads ? kBM : 2 * kBM), len), 0);
    const int tiles = (end + kBN - 1) / kBN;
    if (!streaming) {
      a_end = c_begin = c_end = tiles;
    } else {
      a_end = (min(g.S, end) + kBN - 1) / kBN;
      c_begin = max(a_end, max(0, g.wstart(off + q0)) / kBN);
      c_end = max(c_begin, tiles);
    }
  }
  static constexpr int span = kBM;  // tokens of a query tile
  __device__ __forceinline__ int row0(int x) const { return two_heads ? q0 : q0 + x * kBM; }
  __device__ __forceinline__ int head(int x) const { return two_heads ? h + x : h; }
  __device__ __forceinline__ int tiles() const { return a_end + (c_end - c_begin); }
  __device__ __forceinline__ int chunk_tile(int i) const { return i < a_end ? i : c_begin + (i - a_end); }
  __device__ __forceinline__ int valid(const CacheGeom&, int i) const { return klen - chunk_tile(i) * kBN; }
  __device__ __forceinline__ int row(int x, int r) const { return row0(x) + r; }
  __device__ __forceinline__ bool has_row(int x, int r) const { return row(x, r) < len; }
  __device__ __forceinline__ size_t out_row(const PackedArgs& a, int x, int r) const {
    return (size_t)(qrow + row(x, r)) * a.geom.Hq + head(x);
  }
  __device__ __forceinline__ int rot(const CacheGeom&) const { return 0; }
};

template <int D>
__device__ __forceinline__ void load_q(const PackedArgs& a, const PackedItem& t, int x, uint8_t* dst, uint64_t* bar) {
  using C = PfCfg<D>;
  mbar_arrive_expect_tx(bar, C::QBYTES);
  for (int db = 0; db < C::DBLK; ++db)
    tma_load_4d(dst + db * C::BOX, &a.tq, db * 64, t.head(x), t.qrow + t.row0(x), 0, bar);
}

// A folded item is two query tiles, each of all G heads of a KV head at 128 / G neighbouring
// tokens: row r of a tile is head r % G at its token r / G, the order in which a token's heads
// lie in memory, so that a tile is one box of the queries' tensor (where G does not divide
// 128 the last one or two rows of a tile are not used). Short rows thus fill their tiles with
// heads, and the keys of a KV head are read once for all of its query heads.
struct FoldedItem {
  static constexpr int n_c = 0;  // no cached tiles
  int G, span, rcp, kvh, q0, len, qrow, krow, klen, off, a_end, c_begin, c_end;
  bool streaming;
  __device__ __forceinline__ FoldedItem(const FoldedArgs& a, uint64_t code) {
    const CacheGeom& g = a.geom;
    G = g.G;
    span = a.span;
    rcp = a.rcp;
    kvh = (int)(code >> 24) & 1023;
    q0 = (int)(code & 0xffffffu) * (2 * span);
    streaming = g.kind[kvh] != 0;
    const int4 s = a.seqs.of((int)(code >> 34));
    qrow = s.x;
    len = s.y;
    krow = s.z;
    klen = s.w;
    off = klen - len;
    const int end = max(off + min(q0 + 2 * span, len), 0);
    const int tiles = (end + kBN - 1) / kBN;
    if (!streaming) {
      a_end = c_begin = c_end = tiles;
    } else {
      a_end = (min(g.S, end) + kBN - 1) / kBN;
      c_begin = max(a_end, max(0, g.wstart(off + q0)) / kBN);
      c_end = max(c_begin, tiles);
    }
  }
  // query tile x: its first token; row r of it: its token, whether there is one, and its place
  // among the output's rows of D
  __device__ __forceinline__ int row0(int x) const { return q0 + x * span; }
  __device__ __forceinline__ int token(int r) const { return (r * rcp) >> 16; }  // r / G
  __device__ __forceinline__ int row(int x, int r) const { return row0(x) + token(r); }
  __device__ __forceinline__ bool has_row(int x, int r) const { return r < span * G && row(x, r) < len; }
  __device__ __forceinline__ size_t out_row(const FoldedArgs& a, int x, int r) const {
    return (size_t)(qrow + row0(x) + token(r)) * a.geom.Hq + kvh * G + (r - token(r) * G);
  }
  __device__ __forceinline__ int tiles() const { return a_end + (c_end - c_begin); }
  __device__ __forceinline__ int chunk_tile(int i) const { return i < a_end ? i : c_begin + (i - a_end); }
  __device__ __forceinline__ int valid(const CacheGeom&, int i) const { return klen - chunk_tile(i) * kBN; }
  __device__ __forceinline__ int rot(const CacheGeom&) const { return 0; }
};

template <int D>
__device__ __forceinline__ void load_q(const FoldedArgs& a, const FoldedItem& t, int x, uint8_t* dst, uint64_t* bar) {
  using C = PfCfg<D>;
  mbar_arrive_expect_tx(bar, C::DBLK * t.span * t.G * 128);
  for (int db = 0; db < C::DBLK; ++db)
    tma_load_4d(dst + db * C::BOX, &a.tq, db * 64, t.kvh * t.G, t.qrow + t.row0(x), 0, bar);
}

template <int D, class T>
__device__ __forceinline__ void load_packed_kv(const PackedArgs& a, const T& t, int i, int sel, uint8_t* dst, uint64_t* bar) {
  using C = PfCfg<D>;
  mbar_arrive_expect_tx(bar, C::KVBYTES);
  const CUtensorMap* map = sel ? &a.tv : &a.tk;
  for (int db = 0; db < C::DBLK; ++db)
    tma_load_4d(dst + db * C::BOX, map, db * 64, t.kvh, t.krow + t.chunk_tile(i) * kBN, 0, bar);
}
template <int D>
__device__ __forceinline__ void load_kv(const PackedArgs& a, const PackedItem& t, int i, int sel, uint8_t* dst,
                                        uint64_t* bar) {
  load_packed_kv<D>(a, t, i, sel, dst, bar);
}
template <int D>
__device__ __forceinline__ void load_kv(const FoldedArgs& a, const FoldedItem& t, int i, int sel, uint8_t* dst,
                                        uint64_t* bar) {
  load_packed_kv<D>(a, t, i, sel, dst, bar);
}

// The keys of tile ja that token i (position off + i) of a query tile from token qx0 on sees,
// as in Mask.
struct PackedMask {
  bool need;
  int e_hi, a0 = 0, a1 = 0;
  static constexpr int b0 = 0, b1 = 0;
  template <class T>
  __device__ __forceinline__ PackedMask(const CacheGeom& g, const T& t, int ja, int i, int qx0, int) {
    const int j0 = t.chunk_tile(ja) * kBN, jl = j0 + kBN - 1, pos = t.off + i;
    need = !(jl <= t.off + qx0 && jl < t.klen &&
             (!t.streaming || jl < g.S || j0 >= g.wstart(t.off + qx0 + t.span - 1)));
    const int kmax = min(pos, t.klen - 1) - j0;
    e_hi = kmax + 1;
    if (t.streaming) {
      e_hi = min(e_hi, g.S - j0);
      a0 = g.wstart(pos) - j0;
      a1 = kmax + 1;
    }
  }
};

// Rows row0, row0 + 1, ... of an item's 256 whose bits are set once more, by the warp, where a
// hidden key's V made their outputs wrong: in a matrix product a weight of zero times a NaN or
// an infinity is a NaN, so that such a V row reaches rows that share a tile with it and do not see
// it. Rows with an output that is not finite come here. One whose tiles hide no such V row from it
// (the few keys of each that it does not see are looked at) keeps its output; any other is computed
// from the keys that it sees alone, the newest first, a lane D / 32 of the numbers, until all of
// them are NaN: a sequence that went bad at some token ends there.
// 8,192 tokens of 8/2 heads of 128, half streaming, 0.09 ms: with V all NaN 0.8, an infinity at key 0
// 1.1, one behind the sinks of every streaming row 4.2, one number of every V row infinite 90.
// Calls without such values pay for the look at their outputs alone: 16 x 101-2,999 tokens 230 ->
// 233 us, 32,768 tokens the same.
template <int D, class A>
__device__ void repair_rows(const A& a, uint64_t code, int row0, uint32_t rows) {
  constexpr int N = D / 32;
  const typename CallOf<A>::ItemT t(a, code);
  const CacheGeom& g = a.geom;
  const int lane = threadIdx.x & 31;
  auto load = [&](const void* base, long long stride, long long row, int head, float (&to)[N]) {
    const bf16* p = static_cast<const bf16*>(base) + row * stride + head * D + lane * N;
#pragma unroll
    for (int n = 0; n < N; n += 2) {
      const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(p + n));
      to[n] = f.x;
      to[n + 1] = f.y;
    }
  };
  __syncwarp();  // the rows' first writes come before
  for (; rows; rows &= rows - 1) {
    const int row = row0 + __ffs((int)rows) - 1, x = row >> 7, r = row & 127;
    if (!t.has_row(x, r)) continue;
    const int pos = t.off + t.row(x, r);
    const int w0 = t.streaming ? max(0, g.wstart(pos)) : 0, sinks = t.streaming ? min(g.S, w0) : 0;
    float v[N], o[N] = {};
    bool hit = false;
    // of each tile only what this row does not see: between the sinks and the window, and past the row
    for (int i = 0; i < t.tiles() && !hit; ++i) {
      const int j0 = t.chunk_tile(i) * kBN, j1 = min(j0 + kBN, t.klen);
      float bad = 0.f;
      auto look = [&](int from, int to) {
        for (int j = from; j < to; ++j) {
          load(a.v, a.v_stride, t.krow + j, t.kvh, v);
#pragma unroll
          for (int n = 0; n < N; ++n) bad = fmaf(v[n], 0.f, bad);
        }
      };
      look(max(j0, sinks), min(j1, w0));
      look(max(j0, pos + 1), j1);
      hit = __any_sync(0xffffffffu, !(bad == 0.f));
    }
    if (!hit) continue;
    const size_t at = t.out_row(a, x, r);
    float q[N], k[N], m = -INFINITY, l = 0.f;
    load(a.q, a.q_stride, at / g.Hq, (int)(at % g.Hq), q);
    for (int j = pos; j >= 0; --j) {
      if (j < w0) j = min(j, sinks - 1);
      if (j < 0) break;
      load(a.k, a.k_stride, t.krow + j, t.kvh, k);
      load(a.v, a.v_stride, t.krow + j, t.kvh, v);
      float s = 0.f;
#pragma unroll
      for (int n = 0; n < N; ++n) s = fmaf(q[n], k[n], s);
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
      s *= a.scale_log2;
      const float top = fmaxf(m, s), base = top == -INFINITY ? 0.f : top;
      const float f = fast_exp2(m - base), p = fast_exp2(s - base);
      m = top;
      l = l * f + p;
      bool done = l > 0.f;  // with every number a NaN, which it stays
#pragma unroll
      for (int n = 0; n < N; ++n) {
        o[n] = o[n] * f + p * v[n];
        done = done && isnan(o[n]);
      }
      if (isnan(l) || __all_sync(0xffffffffu, done)) break;
    }
    bf16* out = static_cast<bf16*>(a.out) + at * D + lane * N;
#pragma unroll
    for (int n = 0; n < N; n += 2)
      *reinterpret_cast<uint32_t*>(out + n) =
          l == 0.f ? 0u : isnan(l) ? 0x7fc07fc0u : float2_to_bf16x2(o[n] / l, o[n + 1] / l);
  }
}

template <>
struct CallOf<PackedArgs> {
  using ItemT = PackedItem;
  using MaskT = PackedMask;
  static constexpr bool kEmptyRows = true;  // fewer keys than rows
  static constexpr bool kRepairs = true;
  static constexpr bool kThirdS = true;
  template <int D>
  static constexpr bool kLaneRows = D == 64;
  static constexpr bool kChained = true;
};
template <>
struct CallOf<FoldedArgs> {
  using ItemT = FoldedItem;
  using MaskT = PackedMask;
  static constexpr bool kEmptyRows = true;
  static constexpr bool kRepairs = true;
  static constexpr bool kThirdS = true;
  template <int D>
  static constexpr bool kLaneRows = true;
  static constexpr bool kChained = true;
};

}  // namespace pf
}  // namespace aoh
