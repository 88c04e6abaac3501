// Causal prefill attention on tcgen05 tensor cores (Sec. 5, "Chunked-Prefill
// Stage", with the per-token sink + window rule for streaming heads). A call
// processes one chunk of every sequence: rows at positions Lb .. Lb + len - 1
// after Lb cached tokens (Lb = 0 for a first prefill). Cached keys are read
// from the KV cache itself (retrieval rows, or the streaming sink + ring
// slots) before the chunk's own keys; the cache is appended after this
// kernel, so the ring still holds the positions the chunk's rows need.
//
// One CTA computes two 128-row query tiles (A, B) against the same stream of
// 128-key K/V tiles: the same rows of two heads of a group, or two consecutive
// tiles of one head. The KV tiles visited come from a per-head schedule: a
// retrieval head visits tiles 0 .. causal end; a streaming head only the
// tiles holding its S sinks and the tiles that intersect the W-token window
// of some row, so its cost is O(S + W) per row instead of O(T). Consecutive
// tiles visit the union of their tile sets; a tile hidden from every row of
// one query tile contributes zero weights there. Tiles fully visible to every
// row of a query tile skip the mask.
//
// Warp roles (320 threads):
//   warp 0      TMA producer: Q_A, Q_B once, then K_j / V_j tiles into a
//               4-stage ring (4D tensor maps over [B][T][H][D], 128-byte swizzle).
//   warp 1      TMEM owner and MMA issuer. S_X(j) = Q_X K_j^T reads both
//               operands from shared memory; O_X += P_X(j) V_j reads P_X from
//               TMEM, where the softmax wrote it over the first 64 columns of
//               S_X. Per KV tile the issue order is O_A += P_A V, S_A(j+1),
//               O_B += P_B V, S_B(j+1): a tile's next S overwrites its P only
//               after the P.V that reads it (MMAs of one thread run in order),
//               and while one query tile's softmax runs the tensor pipe works
//               on the other's MMAs, hiding the commit -> softmax -> issue
//               latency of each tile.
//   warps 2-5   softmax of tile A, warps 6-9 softmax of tile B (of 8-bit pages warps 4-11,
//               behind them four that turn codes into bf16 tiles: paged_attend.cuh): thread r owns
//               row r (TMEM lane r). One tcgen05.ld pass reads its S row, a
//               two-range integer mask hides keys, max and sum reduce in 8
//               independent chains, p = 2^(s*scale - m) costs one FFMA and one
//               EX2, the running max moves only when it grows by more than
//               2^8 (O rarely rescaled), and bf16 P pairs go back to TMEM with
//               tcgen05.st (key k in column k/2, even k in the low half),
//               announced in two halves of 64 keys.
// TMEM columns: S_A / P_A [0,128), S_B / P_B [128,256), O_A [256, 256+D),
// O_B [256+D, 256+2D); with three buffers for S (SBuf) O comes 128 columns later.
#pragma once

#include <string.h>

#include "cluster.cuh"
#include "prefill_tile.cuh"

namespace aoh {
namespace pf {

// kPairs: clusters of two CTAs, each with its entry of the list. Where both have the
// same item's halves, each visits half of its KV tiles; then each finishes one of
// the two query tiles: it receives the other
// CTA's state of that tile (O, running max and sum) in shared memory that the
// main loop no longer needs, adds its own and writes the rows.
// kSplit: clusters of C = 2 .. 16 CTAs, an item each: every CTA visits a C-th of its KV
// tiles and finishes a C-th of its 256 rows, whose states it receives from all (its own among
// them). An item whose second query tile has no row is a lone one: both halves of the
// pipeline work on its first tile, A on the even KV tiles and B on the odd ones, and their states
// count as those of two CTAs.
// kJoined: CTAs of their own, one for each part of an item's KV tiles (an entry has the part, the parts
// and a number of the item's: joined_entry). Each stores its state in global memory, and the last to
// arrive adds them up.
constexpr int kWhole = 0, kPairs = 1, kSplit = 2, kJoined = 3;

// Whether a part of an item saw no key of a row. A part whose visible scores are all NaN has a
// maximum of -inf as well, no NaN being the greater of two numbers, but its sum is NaN.
__device__ __forceinline__ bool empty_state(float m, float l) { return m == -INFINITY && l == 0.f; }

// The state of part `rank` of `parts` of an item to global memory ([D / 4][256 rows] float4, then (m, l) of
// each row); the last CTA to arrive adds up the parts' and writes the rows. All threads; w: the warp among the
// softmax warps (others: outside 0-7). The copies and MMAs of the CTA are done with its shared memory.
template <int D, int O, class A, class T>
__device__ __forceinline__ void join_parts(const A& a, const T& t, uint64_t code, int slot, int rank, int parts, int n_tiles,
                                           float m, float l, bool ok, uint32_t tmem, uint8_t* smem, volatile int* last, int w) {
  const int lane = threadIdx.x & 31, x = w >> 2, q4 = (threadIdx.x >> 5) & 3, r = q4 * 32 + lane, row = x * 128 + r;
  const bool soft = w >= 0 && w < 8 && t.has_row(x, q4 * 32);  // alike in a warp
  auto state = [&](int part) { return a.states + (size_t)(slot * a.most_parts + part) * (64 * D + 128); };
  auto ends = [&](int part) { return reinterpret_cast<float2*>(state(part) + 64 * D); };
  if (soft) {
    float4* to = state(rank) + row;
    __stcg(ends(rank) + row, make_float2(ok ? m : -INFINITY, l));
    if (n_tiles > 0) {
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        uint32_t v[32];
        tmem_ld32(tmem + ((uint32_t)(q4 * 32) << 16) + O + x * D + c * 32, v);
        tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 32; e += 4)
          __stcg(to + (c * 8 + e / 4) * 256, make_float4(__uint_as_float(v[e]), __uint_as_float(v[e + 1]),
                                                         __uint_as_float(v[e + 2]), __uint_as_float(v[e + 3])));
      }
    }
    tc_fence_before();
    __threadfence();
  }
  __syncthreads();
  if (threadIdx.x == 0) *last = atomicAdd(a.arrived + slot, 1) == parts - 1;
  __syncthreads();
  if (!*last) return;
  __threadfence();
  if (!soft) return;
  float M = -INFINITY, L = 0.f, f[kJoinedMost];
#pragma unroll
  for (int p = 0; p < kJoinedMost; ++p)
    if (p < parts) M = fmaxf(M, __ldcg(ends(p) + row).x);
#pragma unroll
  for (int p = 0; p < kJoinedMost; ++p) {
    f[p] = -1.f;  // a state that saw no key, whose numbers may never have been written
    if (p < parts) {
      const float2 ml = __ldcg(ends(p) + row);
      if (!empty_state(ml.x, ml.y)) {
        f[p] = fast_exp2(ml.x - M);
        L += f[p] * ml.y;
      }
    }
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  uint8_t* stage = smem + w * (32 * D * 2);
  Spoilt spoilt;
#pragma unroll 1
  for (int c = 0; c < D / 32; ++c) {
    float4 o[8] = {};
#pragma unroll
    for (int p = 0; p < kJoinedMost; ++p) {
      if (p >= parts) break;
      float4 z[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = __ldcg(state(p) + (c * 8 + e) * 256 + row);
      if (f[p] < 0.f) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        o[e].x += f[p] * z[e].x;
        o[e].y += f[p] * z[e].y;
        o[e].z += f[p] * z[e].z;
        o[e].w += f[p] * z[e].w;
      }
    }
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const float y[8] = {o[e].x * inv,     o[e].y * inv,     o[e].z * inv,     o[e].w * inv,
                          o[e + 1].x * inv, o[e + 1].y * inv, o[e + 1].z * inv, o[e + 1].w * inv};
      spoilt.add(put_row<D>(stage, lane, c * 4 + e / 2, y));
    }
  }
  write_rows<D, D>(a, t, x, q4 * 32, 0, stage, lane);
  const uint32_t rows = spoilt.rows(t.has_row(x, r));
  if (rows) repair_rows<D>(a, code, x * 128 + q4 * 32, rows);
}

template <class A, int D, int MODE, int CAP>
__global__ void __launch_bounds__(CallOf<A>::kThreads, 1)
    prefill_tc_kernel(const __grid_constant__ A a, const __grid_constant__ WorkList<CAP> wl) {
  using C = PfCfg<D>;
  using Call = CallOf<A>;
  using SB = SBuf<A, D>;
  constexpr bool PAGED = Call::kPaged, F8 = Call::kF8;
  constexpr int S0 = Call::kSoftmax;  // the first of the 8 softmax warps
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  uint8_t* sQ = smem + C::OFF_Q;
  uint8_t* sKV = smem + C::OFF_KV;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);
  uint64_t* q_full = bars;
  uint64_t* kv_full = bars + 1;
  uint64_t* kv_empty = kv_full + kNS;
  uint64_t* s_full = kv_empty + kNS;  // [SB::bar]: S_A, S_B ready
  uint64_t* p_full = s_full + 4;      // [SB::bar][2]: P_A, P_B written, keys 0-63 and 64-127
  uint64_t* pv_done = p_full + 8;     // [SB::bar]: O_A, O_B updated (P buffer free)
  uint64_t* drain = pv_done + 4;
  // [2]: padding rows of the item's first / second partial V tile are zeroed.
  // Only the last cache tile and the chunk tile holding row len - 1 can be
  // partial, so each barrier completes at most once per item.
  uint64_t* v_zeroed = drain + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(v_zeroed + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // the append may start once the last CTAs of this grid run (append.cu)
  if constexpr (!PAGED) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if constexpr (Call::kChained) {
    if (threadIdx.x == 0) prefetch_maps(a);
    if (PAGED || a.seqs.table != nullptr) wait_to_start(a);  // the item is read from device memory
  }
  // (a launch of the same call that follows finds what this one has waited for)
  if constexpr (PAGED) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  constexpr bool PAIRS = MODE == kPairs, SPLIT = MODE == kSplit, JOINED = MODE == kJoined;
  const int entry = SPLIT ? blockIdx.x / cluster_ctas() : blockIdx.x;
  const uint64_t given = CAP > 0 ? wl.item[entry] : a.work[entry], code = JOINED ? given & (kJoinedPart - 1) : given;
  if (PAIRS && code == kPrefillNone) return;
  const int ctas = SPLIT ? (int)cluster_ctas() : JOINED ? joined_parts(given) : 2;
  const bool half = SPLIT || (JOINED && ctas > 1) || (PAIRS && code >= kPrefillHalf);  // alike in all CTAs of a cluster
  const typename Call::ItemT t(a, code & ~kPrefillHalf);
  if constexpr (PAGED) {
    if (t.elsewhere(a)) {  // alike in all CTAs of a cluster
      wait_to_end(a);
      return;
    }
  }
  const CacheGeom& g = a.geom;
  const int n_all = t.tiles();
  // this CTA visits tiles t0 .. t0 + n_tiles - 1 of the item's n_all
  const int rank = JOINED ? joined_part(given) : half ? (int)cluster_rank() : 0;
  const int per = SPLIT || JOINED ? (n_all + ctas - 1) / ctas : (n_all + 1) / 2;
  const int t0 = rank * per;
  const int n_tiles = !half ? n_all : SPLIT || JOINED ? max(0, min(per, n_all - t0)) : rank == 0 ? (n_all + 1) / 2 : n_all / 2;
  const bool lone = SPLIT && !t.has_row(1, 0);
  PageWalk<A, D> pages(warp == 0 ? lane : -1, a);
  if (threadIdx.x == 0) {
    mbar_init(q_full, 2);
    for (int s = 0; s < kNS; ++s) {
      mbar_init(&kv_full[s], F8 ? 8 : 1);  // (eight groups of rows)
      mbar_init(&kv_empty[s], 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&p_full[2 * i], 4);
      mbar_init(&p_full[2 * i + 1], 4);
      mbar_init(&pv_done[i], 1);
    }
    mbar_init(drain, 1);
    mbar_init(&v_zeroed[0], 1);
    mbar_init(&v_zeroed[1], 1);
    *abort_flag = 0;
    fence_mbar_init();
    fence_proxy_async_smem();
    if constexpr (Call::kChained) wait_to_start(a);
    // the first loads need no other warp
    load_q<D>(a, t, 0, sQ, q_full);
    load_q<D>(a, t, 1, sQ + C::QBYTES, q_full);
    if constexpr (!PAGED)
      if (n_tiles > 0) load_kv<D>(a, t, t0, 0, sKV, &kv_full[0]);
  }
  if constexpr (PAGED && !F8) {
    if (warp == 0 && n_tiles > 0) {
      __syncwarp();
      pages.fetch(a, t, t0);
      pages.look(a, t, t0, n_tiles > 1);
      pages.load(a, t, 0, sKV, &kv_full[0]);
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

  // a half: a row's final softmax state (softmax warps)
  float end_m = -INFINITY, end_l = 0.f;
  bool end_ok = true;
  if (warp < S0 || warp >= S0 + 8) {
    if constexpr (F8) {
      // The softmax warps have their registers before any of these takes its own back below: a
      // role may end at once, and then there would be none left for them to wait for.
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
      __syncthreads();
    }
    if (F8 && warp != 1) {
      if constexpr (F8) {
        // ---------------------------------------------------------- codes to bf16 tiles
        CodeWalk<A, D> walk;
        walk.run(a, t, t0, n_tiles, warp == 0 ? 0 : warp < S0 ? warp - 1 : warp - (S0 + 8) + S0 - 1, sKV, kv_full, kv_empty,
                 lane, abort_flag);
        if (warp == 0) {
          if (lane == 0) drain_wait(q_full, 0, a.err);
          __syncwarp();
        }
      }
    } else if (warp == 0) {
      // ------------------------------------------------------------ producer
      // Lane 0 issues the copies. Rows of a V tile past its valid keys may hold
      // anything (cache rows not yet written, chunk padding) and a zero weight
      // times a NaN is still NaN, so for a partial V tile the whole warp waits
      // for the copy, zeroes those rows and signals v_zeroed before the MMA
      // issuer may read the tile.
      int issued = min(n_tiles, 1), n_partial = 0;  // the first K tile is on its way
      bool ok = true;
      for (int jj = 0; jj < n_tiles && ok; ++jj) {
        if constexpr (PAGED && !F8)
          if (jj > 0) pages.look(a, t, t0 + jj, jj + 1 < n_tiles);
        for (int sel = 0; sel < 2; ++sel) {
          const int it = 2 * jj + sel;
          const int st = it % kNS;
          if constexpr (PAGED && !F8) {
            if (it >= kNS) ok = __all_sync(0xffffffffu, wait_bar(&kv_empty[st], ((it / kNS) & 1) ^ 1, a.err, abort_flag));
            if (ok && it > 0) {
              pages.load(a, t, sel, sKV + st * C::KVBYTES, &kv_full[st]);
              issued = it + 1;
            }
          } else if (lane == 0) {
            if (it >= kNS) ok = wait_bar(&kv_empty[st], ((it / kNS) & 1) ^ 1, a.err, abort_flag);
            if (ok && it > 0) {
              load_kv<D>(a, t, t0 + jj, sel, sKV + st * C::KVBYTES, &kv_full[st]);
              issued = it + 1;
            }
          }
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          const int valid = t.valid(g, t0 + jj);
          if (sel == 1 && valid < kBN && n_partial < 2) {
            ok = __all_sync(0xffffffffu, wait_bar(&kv_full[st], (it / kNS) & 1, a.err, abort_flag));
            if (!ok) break;
            zero_tail<D>(sKV + st * C::KVBYTES, valid, lane);
            if (lane == 0) mbar_arrive(&v_zeroed[n_partial]);
            ++n_partial;
          }
        }
      }
      // every issued copy lands before the CTA can exit
      if (lane == 0) {
        drain_wait(q_full, 0, a.err);
        for (int it = issued > kNS ? issued - kNS : 0; it < issued; ++it)
          drain_wait(&kv_full[it % kNS], (it / kNS) & 1, a.err);
      }
      __syncwarp();
    } else {
      // ------------------------------------------------------------ MMA issuer
      // The whole warp runs the loop (its values stay warp-uniform); one elected
      // lane, the same each time, issues.
      const uint64_t q_desc = sdesc_sw128(smem_u32(sQ), 16, 1024);
      const uint64_t k_desc0 = sdesc_sw128(smem_u32(sKV), 16, 1024);
      const uint64_t v_desc0 = sdesc_sw128(smem_u32(sKV), C::BOX, 1024);
      // S_X of the step, against K_jj, to buffer b
      auto s_at = [&](int x, int step, int jj, int b) {
        const uint64_t k_desc = k_desc0 + (uint32_t)(((2 * jj) % kNS) * sdesc_step(C::KVBYTES));
        if (elect_one()) {
          issue_s<D>(tmem + b * 128, q_desc + (lone ? 0u : sdesc_step(x * C::QBYTES)), k_desc);
          tc_commit(&s_full[SB::bar(x, step)]);
        }
      };
      auto s_of = [&](int x, int jj) { s_at(x, jj, jj, x); };
      auto commit = [&](uint64_t* bar) {
        if (elect_one()) tc_commit(bar);
      };
      bool ok = n_tiles > 0;
      auto wait = [&](uint64_t* bar, uint32_t parity) {
        if (ok) ok = __all_sync(0xffffffffu, wait_bar(bar, parity, a.err, abort_flag));
        return ok;
      };
      // O_X += P_X(step) V_jj, P in buffer b: the first half of the keys while the softmax forms the
      // second half's weights
      auto pv_at = [&](int x, int step, int jj, int b) {
        const uint64_t v_desc = v_desc0 + (uint32_t)(((2 * jj + 1) % kNS) * sdesc_step(C::KVBYTES));
  #pragma unroll
        for (int half = 0; half < 2; ++half) {
          if (!wait(&p_full[2 * SB::bar(x, step) + half], SB::phase(step))) return false;
          tc_fence_after();
          if (elect_one()) {
            issue_pv<D>(tmem + SB::O + x * D, tmem + b * 128, v_desc, half, step == 0);
            if (half) tc_commit(&pv_done[SB::bar(x, step)]);
          }
        }
        return true;
      };
      auto pv_of = [&](int x, int jj) { return pv_at(x, jj, jj, x); };
      auto wait_k = [&](int jj) { return wait(&kv_full[(2 * jj) % kNS], ((2 * jj) / kNS) & 1); };
      // only the last cached tile and the last chunk tile can be partial
      int n_partial = 0;  // partial V tiles seen so far (index into v_zeroed)
      const int part0 = t.n_c > 0 && t.valid(g, t.n_c - 1) < kBN ? t.n_c - 1 - t0 : -1;
      const int part1 = t.valid(g, n_all - 1) < kBN ? n_all - 1 - t0 : -1;
      auto wait_v = [&](int jj) {
        if (!wait(&kv_full[(2 * jj + 1) % kNS], ((2 * jj + 1) / kNS) & 1)) return false;
        if (!F8 && (jj == part0 || jj == part1)) {
          if (!wait(&v_zeroed[n_partial], 0)) return false;
          ++n_partial;
        }
        return true;
      };
      if (SPLIT && lone) {
        // S_X of tile j, whose K is then free
        auto lone_s = [&](int x, int j) {
          if (j >= n_tiles) return true;
          if (!wait_k(j)) return false;
          tc_fence_after();
          s_at(x, j >> 1, j, j % SB::N);
          commit(&kv_empty[(2 * j) % kNS]);
          return true;
        };
        if (wait(q_full, 0) && lone_s(0, 0)) lone_s(1, 1);
        for (int j = 0; j < n_tiles && ok; ++j) {
          const int x = j & 1;
          if (!wait_v(j) || !pv_at(x, j >> 1, j, j % SB::N)) break;
          commit(&kv_empty[(2 * j + 1) % kNS]);
          if (!lone_s(x, j + 2)) break;
        }
      } else if (SB::N == 3) {
        if (wait(q_full, 0) && wait_k(0)) {
          tc_fence_after();
          s_at(0, 0, 0, 0);
          s_at(1, 0, 0, 1);
          commit(&kv_empty[0]);
          if (n_tiles > 1 && wait_k(1)) {
            tc_fence_after();
            s_at(0, 1, 1, 2);
          }
        }
        // after the P V of the n-th S comes the n + 3rd S
        int b = 0;
        for (int jj = 0; jj < n_tiles && ok; ++jj) {
          if (!wait_v(jj) || !pv_at(0, jj, jj, b)) break;
          if (jj + 1 < n_tiles) {
            s_at(1, jj + 1, jj + 1, b);
            commit(&kv_empty[(2 * (jj + 1)) % kNS]);
          }
          b = b == 2 ? 0 : b + 1;
          if (!pv_at(1, jj, jj, b)) break;
          commit(&kv_empty[(2 * jj + 1) % kNS]);
          if (jj + 2 < n_tiles) {
            if (!wait_k(jj + 2)) break;
            tc_fence_after();
            s_at(0, jj + 2, jj + 2, b);
          }
          b = b == 2 ? 0 : b + 1;
        }
      } else if (wait(q_full, 0) && wait_k(0)) {
        tc_fence_after();
        s_of(0, 0);
        s_of(1, 0);
        commit(&kv_empty[0]);
      }
      for (int jj = 0; SB::N == 2 && jj < n_tiles && ok && !lone; ++jj) {
        const bool more = jj + 1 < n_tiles;
        // tile A: P_A(jj) sits in S_A's columns; S_A(jj+1) may overwrite them
        // only after O_A += P_A(jj) V_jj is issued (same-thread MMAs run in order)
        if (!wait_v(jj) || !pv_of(0, jj)) break;
        if (more) {
          if (!wait_k(jj + 1)) break;
          tc_fence_after();
          s_of(0, jj + 1);
        }
        if (!pv_of(1, jj)) break;
        commit(&kv_empty[(2 * jj + 1) % kNS]);
        if (more) {
          s_of(1, jj + 1);
          commit(&kv_empty[(2 * (jj + 1)) % kNS]);
        }
      }
      commit(drain);
      __syncwarp();
      drain_wait(drain, 0, a.err);
      __syncwarp();
    }
    if constexpr (F8) {
      __syncwarp();
      asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kExchanged));
    }
  } else {
    if constexpr (F8) {
      asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
      __syncthreads();
    }
    // ------------------------------------------------------------ softmax
    const int x = (warp - S0) >> 2;       // 0: tile A (the first four warps), 1: tile B
    const int q4 = warp & 3;              // TMEM lane quarter this warp may access
    const int r = q4 * 32 + lane;
    const int qt = lone ? 0 : x;          // the query tile
    const int qx0 = t.row0(qt);           // its first row
    const int i = t.row(qt, r);           // of the sequence
    const int steps = lone ? (n_tiles + 1 - x) >> 1 : n_tiles;
    const uint32_t tl = tmem + ((uint32_t)(q4 * 32) << 16);
    const uint32_t o_col = SB::O + x * D;
    uint32_t s_col = x * 128;
    const int rot = t.rot(g);
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    for (int jj = 0; jj < steps && ok; ++jj) {
      const typename Call::MaskT mask(g, t, t0 + (lone ? 2 * jj + x : jj), i, qx0, rot);
      ok = __all_sync(0xffffffffu, wait_bar(&s_full[SB::bar(x, jj)], SB::phase(jj), a.err, abort_flag));
      if (!ok) break;
      tc_fence_after();
      ok = softmax_tile<D>(a, mask, tl, s_col, o_col, jj == 0, m, l, &pv_done[SB::bar(x, jj - 1)], SB::phase(jj - 1),
                           &p_full[2 * SB::bar(x, jj)], abort_flag);
      if (SB::N == 3) s_col = s_col >= 128 ? s_col - 128 : 256;  // two buffers on
    }
    if (half) {
      end_m = m;
      end_l = l;
      end_ok = ok && (steps == 0 ||
                      __all_sync(0xffffffffu, wait_bar(&pv_done[SB::bar(x, steps - 1)], SB::phase(steps - 1), a.err, abort_flag)));
    } else if (ok && (Call::kEmptyRows && n_tiles == 0
                          ? __all_sync(0xffffffffu, wait_bar(q_full, 0, a.err, abort_flag))
                          : __all_sync(0xffffffffu, wait_bar(&pv_done[SB::bar(x, n_tiles - 1)], SB::phase(n_tiles - 1), a.err,
                                                             abort_flag)))) {
      tc_fence_after();
      // Q_X is free: the last S_X was done before the last P V, or it came and none reads it
      const uint32_t spoilt =
          store_o<D, D>(a, t, x, q4 * 32, tl + o_col, l, sQ + x * C::QBYTES + q4 * (C::QBYTES / 4), lane);
      if constexpr (Call::kRepairs)
        if (spoilt) repair_rows<D>(a, code, x * 128 + q4 * 32, spoilt);
    }
    if constexpr (F8) {
      __syncwarp();
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kExchanged));
    }
  }

  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if constexpr (SPLIT) {
    // all CTAs' copies and MMAs are done with their shared memory
    cluster_arrive();
    cluster_wait();
    // The rows that there are, rounded up, are dealt to the CTAs in runs, and only those travel.
    // n states of each of this CTA's rows. Receive buffer: [n][D / 4][rows] float4, then [n][rows]
    // (m, l)
    const int all = !lone ? 256 : t.has_row(0, 64) ? 128 : t.has_row(0, 32) ? 64 : 32;
    const int rows = (all + ctas - 1) / ctas, n = lone ? 2 * ctas : ctas;
    constexpr int kMostStates = 288;  // n * rows at any C
    float4* recv = reinterpret_cast<float4*>(smem);
    float2* recv_ml = reinterpret_cast<float2*>(recv + D / 4 * kMostStates);
    uint32_t* spoilt = reinterpret_cast<uint32_t*>(recv_ml + kMostStates);  // [4]: rows with a value that is not finite
    const int x = (warp - S0) >> 2, q4 = warp & 3, r = q4 * 32 + lane;
    const bool soft = warp >= S0 && warp < S0 + 8;
    if (soft) {
      const int row = lone ? r : x * 128 + r, from = lone ? 2 * rank + x : rank;
      const int dst = min(row / rows, ctas - 1), at = row - dst * rows;
      const uint32_t tl = tmem + ((uint32_t)(q4 * 32) << 16) + SB::O + x * D;
      const uint32_t to = cluster_addr(recv + from * (D / 4) * rows + at, (uint32_t)dst);
      if (row < all)
        cluster_st2(cluster_addr(recv_ml + from * rows + at, (uint32_t)dst), __float_as_uint(end_m),
                    __float_as_uint(end_l));
      if (n_tiles > (lone ? x : 0) && t.has_row(lone ? 0 : x, q4 * 32)) {
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          uint32_t v[32];
          tmem_ld32(tl + c * 32, v);
          tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 32; e += 4)
            cluster_st4(to + (uint32_t)((c * 8 + e / 4) * rows * 16), v[e], v[e + 1], v[e + 2], v[e + 3]);
        }
      }
      tc_fence_before();
    }
    cluster_arrive();
    cluster_wait();
    if (soft) {
      const int tid = threadIdx.x - S0 * 32;  // of the 256 softmax threads
      // (m, l) -> the state's weight, negative for an empty state, whose CTA may have had no tile
      // (unwritten values); any other counts
      if (tid < 4) spoilt[tid] = 0;
      if (tid < rows) {
        float M = -INFINITY, L = 0.f;
        for (int c = 0; c < n; ++c) M = fmaxf(M, recv_ml[c * rows + tid].x);
        for (int c = 0; c < n; ++c) {
          const float2 ml = recv_ml[c * rows + tid];
          if (!empty_state(ml.x, ml.y)) L += fast_exp2(ml.x - M) * ml.y;
        }
        const float inv = L == 0.f ? 0.f : 1.f / L;
        for (int c = 0; c < n; ++c) {
          const float2 ml = recv_ml[c * rows + tid];
          recv_ml[c * rows + tid].x = empty_state(ml.x, ml.y) ? -1.f : fast_exp2(ml.x - M) * inv;
        }
      }
      named_barrier_sync(3, 256);
      for (int u = tid; u < D / 4 * rows; u += 256) {
        const int k = u / rows, at = u - k * rows, row = rank * rows + at, ox = row >> 7, orow = row & 127;
        if (!end_ok || row >= all || !t.has_row(ox, orow)) continue;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int c = 0; c < n; ++c) {
          const float f = recv_ml[c * rows + at].x;
          const float4 z = recv[(c * (D / 4) + k) * rows + at];
          if (f < 0.f) continue;
          o.x += f * z.x;
          o.y += f * z.y;
          o.z += f * z.z;
          o.w += f * z.w;
        }
        *reinterpret_cast<uint2*>(static_cast<bf16*>(a.out) + t.out_row(a, ox, orow) * D + k * 4) =
            make_uint2(float2_to_bf16x2(o.x, o.y), float2_to_bf16x2(o.z, o.w));
        if (!(o.x * 0.f + o.y * 0.f + o.z * 0.f + o.w * 0.f == 0.f)) atomicOr(spoilt + (at >> 5), 1u << (at & 31));
      }
      named_barrier_sync(3, 256);
      if (warp < S0 + 4 && spoilt[warp - S0])
        repair_rows<D>(a, code, rank * rows + (warp - S0) * 32, spoilt[warp - S0]);
    }
    __syncthreads();
    tc_fence_after();
  } else if constexpr (JOINED) {
    if (half) join_parts<D, SB::O>(a, t, code, joined_slot(given), rank, ctas, n_tiles, end_m, end_ok ? end_l : 0.f, end_ok, tmem, smem,
                                   reinterpret_cast<volatile int*>(tmem_slot + 2), warp - S0);
  } else if (half) {
    // both CTAs' copies and MMAs are done with their shared memory
    cluster_arrive();
    cluster_wait();
    const int x = (warp - S0) >> 2, q4 = warp & 3, r = q4 * 32 + lane;
    const bool soft = warp >= S0 && warp < S0 + 8;
    const uint32_t tl = tmem + ((uint32_t)(q4 * 32) << 16) + SB::O + x * D;
    float4* recv = reinterpret_cast<float4*>(smem);  // [D / 4][128 rows], then (m, l) per row
    float2* recv_ml = reinterpret_cast<float2*>(recv + D / 4 * 128);
    if (soft && x != rank) {
      const uint32_t dst = cluster_addr(recv + r, (uint32_t)(rank ^ 1));
      cluster_st2(cluster_addr(recv_ml + r, (uint32_t)(rank ^ 1)), __float_as_uint(end_m), __float_as_uint(end_l));
      if (n_tiles > 0) {
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          uint32_t v[32];
          tmem_ld32(tl + c * 32, v);
          tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 32; e += 4)
            cluster_st4(dst + (uint32_t)((c * 8 + e / 4) * 128 * 16), v[e], v[e + 1], v[e + 2], v[e + 3]);
        }
      }
      tc_fence_before();
    }
    cluster_arrive();
    cluster_wait();
    if (soft && x == rank && end_ok) {
      const float2 o_ml = recv_ml[r];
      const float M = fmaxf(end_m, o_ml.x);
      // an empty state's CTA may have had no tile at all (unwritten values); any other state
      // counts, also with a weight that rounds to zero, whose NaN is one in a single CTA as well
      const bool mine = !empty_state(end_m, end_l), other = !empty_state(o_ml.x, o_ml.y);
      const float w0 = mine ? fast_exp2(end_m - M) : 0.f, w1 = other ? fast_exp2(o_ml.x - M) : 0.f;
      const float inv = 1.f / (end_l * w0 + o_ml.y * w1);
      const float f0 = w0 * inv, f1 = w1 * inv;
      uint8_t* stage = smem + C::OFF_BAR - C::QBYTES + q4 * (C::QBYTES / 4);  // past the receive buffer
      Spoilt spoilt;
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        uint32_t v[32];
        tmem_ld32(tl + c * 32, v);
        tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 32; e += 8) {
          float y[8];
#pragma unroll
          for (int k = 0; k < 8; k += 4) {
            const float4 z = recv[(c * 8 + (e + k) / 4) * 128 + r];
            y[k + 0] = (mine ? __uint_as_float(v[e + k + 0]) * f0 : 0.f) + (other ? z.x * f1 : 0.f);
            y[k + 1] = (mine ? __uint_as_float(v[e + k + 1]) * f0 : 0.f) + (other ? z.y * f1 : 0.f);
            y[k + 2] = (mine ? __uint_as_float(v[e + k + 2]) * f0 : 0.f) + (other ? z.z * f1 : 0.f);
            y[k + 3] = (mine ? __uint_as_float(v[e + k + 3]) * f0 : 0.f) + (other ? z.w * f1 : 0.f);
          }
          const uint4 w = put_row<D>(stage, lane, c * 4 + e / 8, y);
          if (Call::kRepairs) spoilt.add(w);
        }
      }
      write_rows<D, D>(a, t, x, q4 * 32, 0, stage, lane);
      if constexpr (Call::kRepairs) {
        const uint32_t rows = spoilt.rows(t.has_row(x, r));
        if (rows) repair_rows<D>(a, code & ~kPrefillHalf, x * 128 + q4 * 32, rows);
      }
      tc_fence_before();
    }
    __syncthreads();
    tc_fence_after();
  }
  if (warp == 1) tmem_dealloc(tmem, kTmemCols);
  if constexpr (Call::kChained) wait_to_end(a);
}

}  // namespace pf
}  // namespace aoh
