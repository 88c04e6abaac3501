// Prefill of many short work items (prefill_tc.cuh describes the computation and
// the warps' roles): one CTA an SM goes through its items in one pipeline. A CTA an
// item spends 4 us of its life on its start (barriers, TMEM, Q and the first tile
// from memory, the first S and its softmax) and its end (the last P V, O to
// memory) with idle tensor cores, as much as three KV tiles of work. Here the next
// item's K, V and Q load while the last tiles of this one run, and a query tile's
// rows are written while the other's MMAs and the next item's first S go on.
//
// Barrier phases run on across items (counters instead of tile indexes); q_empty
// tells the producer that the item's last S is done. O needs no barrier: the warps
// that read O_X are those whose weights the next item's first P V into it waits
// for. The items are dealt in a fixed order, heaviest first, forth and back (CTA c
// takes items c, 2 P - 1 - c, 2 P + c, ...), which evens out their cost.
//
// 8 ragged sequences of up to 2,999 tokens, 32/8 heads of 128 of which half stream (S =
// 64, W = 512): 276 us with a CTA an item, 244 so; heads of 64 230 -> 210; 16 sequences
// of up to 700 tokens 89 -> 71. What is left of an item's start and end is the chain
// from its last S to the next item's first P V: Q's buffer, S and its softmax.
//
// Over pages (of bf16; paged_attend.cuh) the items' sequences are read before the roles begin, and the first
// entries of the table of the next item are on their way while this one's tiles are: 128 sequences of 2-5 rows
// after 20-36 tokens, 32/8 heads of 64, 45 -> 38 us, 64 of 100-300 rows after up to 1,000 145 -> 130, 16 of 300-700 after up
// to 500, heads of 128, 99 -> 85.
#pragma once

#include <string.h>

#include "prefill_tile.cuh"

namespace aoh {
namespace pf {

// Items of a CTA over pages at most: their sequences are read once, before the roles begin.
constexpr int kShortItems = 32;

template <int D>
struct ShortCfg {
  using C = PfCfg<D>;
  static constexpr int COLS = 64;                // columns of O staged at a time
  static constexpr int STAGE = 32 * COLS * 2;    // a warp's
  static constexpr int OFF_STAGE = C::OFF_BAR;   // 8 warps
  static constexpr int OFF_BAR = OFF_STAGE + 8 * STAGE;
  static constexpr int NBAR = 2 + 2 * kNS + 4 + 8 + 4 + 2 + 1;
  static constexpr int OFF_ITEMS = OFF_BAR + (NBAR * 8 + 15) / 16 * 16 + 16;  // pages: sequences of the CTA's items
  static constexpr int SMEM = OFF_ITEMS + kShortItems * 20 + 1024;
  static_assert(SMEM <= 232448, "shared memory");
};

template <class A, int D, int CAP>
__global__ void __launch_bounds__(kThreads, 1)
    prefill_short_kernel(const __grid_constant__ A a, const __grid_constant__ WorkList<CAP> wl, int n_items) {
  using C = PfCfg<D>;
  using X = ShortCfg<D>;
  using Call = CallOf<A>;
  using SB = SBuf<A, D>;
  constexpr bool PAGED = Call::kPaged;
  static_assert(!Call::kF8, "pages of bf16");
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  uint8_t* sQ = smem + C::OFF_Q;
  uint8_t* sKV = smem + C::OFF_KV;
  uint64_t* q_full = reinterpret_cast<uint64_t*>(smem + X::OFF_BAR);
  uint64_t* q_empty = q_full + 1;
  uint64_t* kv_full = q_empty + 1;
  uint64_t* kv_empty = kv_full + kNS;
  uint64_t* s_full = kv_empty + kNS;   // [SB::bar]: S_A, S_B ready
  uint64_t* p_full = s_full + 4;       // [SB::bar][2]: P_A, P_B written, keys 0-63 and 64-127
  uint64_t* pv_done = p_full + 8;      // [SB::bar]: O_A, O_B updated
  uint64_t* v_zeroed = pv_done + 4;    // [2]: padding rows of every other partial V tile are zeroed
  uint64_t* drain = v_zeroed + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  uint32_t* spoilt = tmem_slot + 2;  // this CTA's items with a value that is not finite: bit k mod 32
  int4* seq_s = reinterpret_cast<int4*>(smem + X::OFF_ITEMS);  // pages: the k-th item's sequence
  int* klen_s = reinterpret_cast<int*>(seq_s + kShortItems);   // and its keys, or -1: another kernel's

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const CacheGeom& g = a.geom;
  const int P = gridDim.x, cta = blockIdx.x;
  if constexpr (Call::kChained)
    if (threadIdx.x == 0) prefetch_maps(a);
  // this CTA's k-th item
  auto item_index = [&](int k) { return k * P + ((k & 1) ? P - 1 - cta : cta); };
  auto item_code = [&](int i) { return CAP > 0 ? wl.item[i] : a.work[i]; };
  auto item = [&](int k) {
    if constexpr (PAGED)
      return typename Call::ItemT(a, item_code(item_index(k)), seq_s[k], klen_s[k]);
    else
      return typename Call::ItemT(a, item_code(item_index(k)));
  };
  auto elsewhere = [&](int k) { return PAGED && klen_s[k] < 0; };
  if (threadIdx.x == 0) {
    mbar_init(q_full, 2);
    mbar_init(q_empty, 1);
    for (int s = 0; s < kNS; ++s) {
      mbar_init(&kv_full[s], 1);
      mbar_init(&kv_empty[s], 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&p_full[2 * i], 4);
      mbar_init(&p_full[2 * i + 1], 4);
      mbar_init(&pv_done[i], 1);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(&v_zeroed[x], 1);
    }
    mbar_init(drain, 1);
    *abort_flag = 0;
    *spoilt = 0;
    fence_mbar_init();
  }
  if constexpr (PAGED) {
    if (warp == 2 && item_index(lane) < n_items) {
      wait_to_start(a);
      const typename Call::ItemT t(a, item_code(item_index(lane)), true);
      seq_s[lane] = make_int4(t.qrow, t.len, t.b, t.first);
      klen_s[lane] = t.elsewhere(a) ? -1 : t.klen;
    }
  }
  if (warp == 1) {
    tmem_alloc(tmem_slot, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  if constexpr (Call::kChained) wait_to_start(a);

  if (warp == 0) {
    // ------------------------------------------------------------ producer
    int it = 0;         // copies of the KV ring so far (K, V, K, V, ...)
    int n_partial = 0;  // partial V tiles so far
    int issued = 0, nq = 0;  // nq: items whose Q was loaded
    bool ok = true;
    PageWalk<A, D> pages(lane, a);
    int early = -1, entry = -1;  // pages: the item whose first entry of the table is on its way, and that
    for (int k = 0; ok; ++k) {
      const int ii = item_index(k);
      if (ii >= n_items) break;
      // the append may start once every CTA is at its last item (append.cu)
      if (item_index(k + 1) >= n_items) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
      if (elsewhere(k)) continue;
      const auto t = item(k);
      const int n = t.tiles();
      if constexpr (PAGED) {
        if (early == k)
          pages.ahead = entry;
        else if (n > 0)
          pages.fetch(a, t, 0);
      }
      for (int jj = 0; jj < n && ok; ++jj) {
        if constexpr (PAGED) {
          pages.look(a, t, jj, jj + 1 < n);
          if (jj == 0 && item_index(k + 1) < n_items && !elsewhere(k + 1)) {
            early = k + 1;
            entry = pages.entry(a, item(k + 1), 0);
          }
        }
        for (int sel = 0; sel < 2; ++sel, ++it) {
          const int st = it % kNS;
          if constexpr (PAGED) {
            if (it >= kNS) ok = __all_sync(0xffffffffu, wait_bar(&kv_empty[st], ((it / kNS) & 1) ^ 1, a.err, abort_flag));
            if (ok) {
              pages.load(a, t, sel, sKV + st * C::KVBYTES, &kv_full[st]);
              issued = it + 1;
            }
            if (lane == 0 && ok && jj == 0 && sel == 0) {
              if (nq >= 1) ok = wait_bar(q_empty, (nq - 1) & 1, a.err, abort_flag);
              if (ok) {
                load_q<D>(a, t, 0, sQ, q_full);
                load_q<D>(a, t, 1, sQ + C::QBYTES, q_full);
              }
            }
            if (jj == 0 && sel == 0 && __all_sync(0xffffffffu, ok)) ++nq;
          } else if (lane == 0) {
            if (it >= kNS) ok = wait_bar(&kv_empty[st], ((it / kNS) & 1) ^ 1, a.err, abort_flag);
            if (ok) {
              load_kv<D>(a, t, jj, sel, sKV + st * C::KVBYTES, &kv_full[st]);
              issued = it + 1;
            }
            if (ok && jj == 0 && sel == 0) {
              // Q after the first K tile: its buffer is free once the last
              // item's last S is done
              if (k >= 1) ok = wait_bar(q_empty, (k - 1) & 1, a.err, abort_flag);
              if (ok) {
                load_q<D>(a, t, 0, sQ, q_full);
                load_q<D>(a, t, 1, sQ + C::QBYTES, q_full);
                nq = k + 1;
              }
            }
          }
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          const int valid = t.valid(g, jj);
          if (sel == 1 && valid < kBN) {
            ok = __all_sync(0xffffffffu, wait_bar(&kv_full[st], (it / kNS) & 1, a.err, abort_flag));
            if (!ok) break;
            zero_tail<D>(sKV + st * C::KVBYTES, valid, lane);
            if (lane == 0) mbar_arrive(&v_zeroed[n_partial & 1]);
            ++n_partial;
          }
        }
      }
    }
    // every issued copy lands before the CTA can exit
    if (lane == 0) {
      if (nq > 0) drain_wait(q_full, (nq - 1) & 1, a.err);
      for (int j = issued > kNS ? issued - kNS : 0; j < issued; ++j)
        drain_wait(&kv_full[j % kNS], (j / kNS) & 1, a.err);
    }
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer
    const uint64_t q_desc = sdesc_sw128(smem_u32(sQ), 16, 1024);
    const uint64_t k_desc0 = sdesc_sw128(smem_u32(sKV), 16, 1024);
    const uint64_t v_desc0 = sdesc_sw128(smem_u32(sKV), C::BOX, 1024);
    int kt = 0;         // KV tiles before this one, over all items
    int n_partial = 0;  // partial V tiles so far
    int nq = 0;         // items with tiles so far
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      if (ok) ok = __all_sync(0xffffffffu, wait_bar(bar, parity, a.err, abort_flag));
      return ok;
    };
    auto commit = [&](uint64_t* bar) {
      if (elect_one()) tc_commit(bar);
    };
    auto s_at = [&](int x, int kt, int b) {
      const uint64_t k_desc = k_desc0 + (uint32_t)(((2 * kt) % kNS) * sdesc_step(C::KVBYTES));
      if (elect_one()) {
        issue_s<D>(tmem + b * 128, q_desc + sdesc_step(x * C::QBYTES), k_desc);
        tc_commit(&s_full[SB::bar(x, kt)]);
      }
    };
    auto s_of = [&](int x, int kt) { s_at(x, kt, x); };
    auto pv_at = [&](int x, bool first, int b) {
      const uint64_t v_desc = v_desc0 + (uint32_t)(((2 * kt + 1) % kNS) * sdesc_step(C::KVBYTES));
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if (!wait(&p_full[2 * SB::bar(x, kt) + half], SB::phase(kt))) return false;
        tc_fence_after();
        if (elect_one()) {
          issue_pv<D>(tmem + SB::O + x * D, tmem + b * 128, v_desc, half, first);
          if (half) tc_commit(&pv_done[SB::bar(x, kt)]);
        }
      }
      return true;
    };
    auto pv_of = [&](int x, bool first) { return pv_at(x, first, x); };
    int b = 0;  // three buffers: that of tile kt's S_A
    auto wait_k = [&](int kt) { return wait(&kv_full[(2 * kt) % kNS], ((2 * kt) / kNS) & 1); };
    for (int k = 0; ok; ++k) {
      const int ii = item_index(k);
      if (ii >= n_items) break;
      if (elsewhere(k)) continue;
      const auto t = item(k);
      const int n = t.tiles();
      if (PAGED && n == 0) continue;
      const int part0 = t.n_c > 0 && t.valid(g, t.n_c - 1) < kBN ? t.n_c - 1 : -1;
      const int part1 = t.valid(g, n - 1) < kBN ? n - 1 : -1;
      if (!wait(q_full, nq & 1) || !wait_k(kt)) break;
      ++nq;
      tc_fence_after();
      if constexpr (SB::N == 3) {
        auto on = [](int b) { return b == 2 ? 0 : b + 1; };
        s_at(0, kt, b);
        s_at(1, kt, on(b));
        commit(&kv_empty[(2 * kt) % kNS]);
        if (n == 1) {
          commit(q_empty);
        } else {
          if (!wait_k(kt + 1)) break;
          tc_fence_after();
          s_at(0, kt + 1, on(on(b)));
        }
        // after the P V of an S comes the third S after it
        for (int jj = 0; jj < n && ok; ++jj, ++kt) {
          if (!wait(&kv_full[(2 * kt + 1) % kNS], ((2 * kt + 1) / kNS) & 1)) break;
          if (jj == part0 || jj == part1) {
            if (!wait(&v_zeroed[n_partial & 1], (n_partial >> 1) & 1)) break;
            ++n_partial;
          }
          if (!pv_at(0, jj == 0, b)) break;
          if (jj + 1 < n) {
            s_at(1, kt + 1, b);
            commit(&kv_empty[(2 * (kt + 1)) % kNS]);
            if (jj + 2 == n) commit(q_empty);
          }
          b = on(b);
          if (!pv_at(1, jj == 0, b)) break;
          commit(&kv_empty[(2 * kt + 1) % kNS]);
          if (jj + 2 < n) {
            if (!wait_k(kt + 2)) break;
            tc_fence_after();
            s_at(0, kt + 2, b);
          }
          b = on(b);
        }
        continue;
      }
      s_of(0, kt);
      s_of(1, kt);
      commit(&kv_empty[(2 * kt) % kNS]);
      if (n == 1) commit(q_empty);
      for (int jj = 0; jj < n && ok; ++jj, ++kt) {
        const bool more = jj + 1 < n;
        if (!wait(&kv_full[(2 * kt + 1) % kNS], ((2 * kt + 1) / kNS) & 1)) break;
        if (jj == part0 || jj == part1) {
          if (!wait(&v_zeroed[n_partial & 1], (n_partial >> 1) & 1)) break;
          ++n_partial;
        }
        if (!pv_of(0, jj == 0)) break;
        if (more) {
          if (!wait_k(kt + 1)) break;
          tc_fence_after();
          s_of(0, kt + 1);
        }
        if (!pv_of(1, jj == 0)) break;
        commit(&kv_empty[(2 * kt + 1) % kNS]);
        if (more) {
          s_of(1, kt + 1);
          commit(&kv_empty[(2 * (kt + 1)) % kNS]);
          if (jj + 2 == n) commit(q_empty);
        }
      }
    }
    commit(drain);
    __syncwarp();
    drain_wait(drain, 0, a.err);
    __syncwarp();
  } else {
    // ------------------------------------------------------------ softmax
    const int x = (warp - 2) >> 2;  // 0: tile A (warps 2-5), 1: tile B (warps 6-9)
    const int q4 = warp & 3;        // TMEM lane quarter this warp may access
    const int r = q4 * 32 + lane;
    const uint32_t tl = tmem + ((uint32_t)(q4 * 32) << 16);
    const uint32_t o_col = SB::O + x * D;
    uint32_t s_col = x * 128;
    uint8_t* stage = smem + X::OFF_STAGE + (warp - 2) * X::STAGE;
    uint32_t kt = 0;  // KV tiles so far, over all items
    bool ok = true;
    for (int k = 0; ok; ++k) {
      const int ii = item_index(k);
      if (ii >= n_items) break;
      if (elsewhere(k)) continue;
      const auto t = item(k);
      const int qx0 = t.row0(x), i = t.row(x, r), n = t.tiles();
      const int rot = t.rot(g);
      float m = -INFINITY, l = 0.f;
      for (int jj = 0; jj < n && ok; ++jj, ++kt) {
        const typename Call::MaskT mask(g, t, jj, i, qx0, rot);
        ok = __all_sync(0xffffffffu, wait_bar(&s_full[SB::bar(x, kt)], SB::phase(kt), a.err, abort_flag));
        if (!ok) break;
        tc_fence_after();
        ok = softmax_tile<D>(a, mask, tl, s_col, o_col, jj == 0, m, l, &pv_done[SB::bar(x, kt - 1)], SB::phase(kt - 1),
                             &p_full[2 * SB::bar(x, kt)], abort_flag);
        if (SB::N == 3) s_col = s_col >= 128 ? s_col - 128 : 256;  // two buffers on
      }
      if (!ok) break;
      // (without a tile: zeros)
      if (!PAGED || n > 0)
        ok = __all_sync(0xffffffffu, wait_bar(&pv_done[SB::bar(x, kt - 1)], SB::phase(kt - 1), a.err, abort_flag));
      if (!ok) break;
      tc_fence_after();
      if (store_o<D, X::COLS>(a, t, x, q4 * 32, tl + o_col, l, stage, lane) && lane == 0)
        atomicOr(spoilt, 1u << (k & 31));
      tc_fence_before();
    }
    // after the loop, which a call would slow down; rows that need none come out the same
    if constexpr (Call::kRepairs) {
      __syncwarp();
      const uint32_t which = *spoilt;
      for (int k = 0; which && item_index(k) < n_items; ++k)
        if (which >> (k & 31) & 1) repair_rows<D>(a, item_code(item_index(k)), x * 128 + q4 * 32, ~0u);
    }
  }

  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, kTmemCols);
  if constexpr (Call::kChained) wait_to_end(a);
}

}  // namespace pf
}  // namespace aoh
