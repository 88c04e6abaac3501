// The host's plan of a prefill call: its work items, how clusters share them, and the
// kernel that runs them. Host code alone.
#pragma once

#include <algorithm>
#include <functional>
#include <vector>

#include "internal.h"

namespace aoh {

// Prefill work: items of two 128-row query tiles, heaviest first so the
// hardware block scheduler fills the machine longest-processing-time first. An
// item is one query tile of two heads of a group, or, for the last head of an
// odd group, two consecutive tiles of that head. Two heads see the same keys;
// two tiles visit the union of their KV tiles, so that each pair of tiles has one
// KV tile that the first does not see, and a sequence's last pair may lack the
// second: 8 ragged sequences of up to 2,999 tokens, 32/8 heads of 128 of which
// half stream (S = 64, W = 512), 298 -> 277 us; 32K tokens of 28/4 streaming heads
// (S = 128, W = 1024) 517 -> 480, 32K with half of them retrieval 2504 -> 2468.
// The cost, the number of KV tiles visited, is the same for all items of a kind,
// so (b, index, kind) entries are sorted and then expanded. *costs receives each
// item's cost; rows_of(b) is sequence b's number of rows, cost(b, q0, q_end, streaming) that
// of the KV tiles that rows q0 .. q_end - 1 visit.
template <class Rows, class Cost>
std::vector<uint64_t> prefill_items(const CacheGeom& g, int B, Rows rows_of, Cost cost, std::vector<int>* costs) {
  constexpr int BM = 128;
  struct Entry {
    int cost, b, index;
    bool streaming, two_heads;
  };
  std::vector<Entry> entries;
  for (int b = 0; b < B; ++b) {
    const int len = rows_of(b);
    for (int streaming = 0; streaming < 2; ++streaming) {
      if ((streaming ? g.n_s : g.n_r) == 0) continue;
      for (int two_heads = 0; two_heads < 2; ++two_heads) {
        if ((two_heads ? g.G / 2 : g.G % 2) == 0) continue;
        const int rows = two_heads ? BM : 2 * BM;
        for (int q0 = 0; q0 < len; q0 += rows)
          entries.push_back({cost(b, q0, std::min(q0 + rows, len), streaming != 0), b, q0 / rows, streaming != 0,
                             two_heads != 0});
      }
    }
  }
  std::stable_sort(entries.begin(), entries.end(), [](const Entry& x, const Entry& y) { return x.cost > y.cost; });
  std::vector<uint64_t> items;
  size_t most = 0;
  for (const Entry& e : entries) most += (size_t)(e.streaming ? g.n_s : g.n_r) * (e.two_heads ? g.G / 2 : 1);
  items.reserve(most);
  costs->reserve(most);
  for (const Entry& e : entries)
    for (int i = 0; i < (e.streaming ? g.n_s : g.n_r); ++i) {
      const int kvh = e.streaming ? g.s_head[i] : g.r_head[i];
      const int first = e.two_heads ? 0 : g.G - 1, step = e.two_heads ? 2 : 1;
      for (int h = first; h + step <= g.G; h += step) {
        items.push_back(prefill_item(e.b, kvh * g.G + h, e.index) | (e.two_heads ? kPrefillTwoHeads : 0));
        costs->push_back(e.cost);
      }
    }
  return items;
}

// A cache's chunk: the cached tiles, then those of the chunk itself.
inline std::vector<uint64_t> prefill_schedule(const CacheGeom& g, const std::vector<int32_t>& base,
                                              const std::vector<int32_t>& lens, std::vector<int>* costs) {
  constexpr int BN = 128;
  return prefill_items(
      g, g.B, [&](int b) { return (int)lens[b]; },
      [&](int b, int q0, int q_end, bool streaming) {
        const int Lb = base[b];
        const int n_c = Lb == 0 ? 0 : ((streaming ? std::min(Lb, g.S + g.W) : Lb) + BN - 1) / BN;
        if (!streaming) return n_c + (q_end + BN - 1) / BN;
        const int a_end = (std::min(std::max(g.S - Lb, 0), q_end) + BN - 1) / BN;
        const int c_begin = std::max(a_end, std::max(0, g.wstart(q0)) / BN);
        const int c_end = std::max(c_begin, (q_end + BN - 1) / BN);
        return n_c + a_end + (c_end - c_begin);
      },
      costs);
}

// Packed prompts (PackedSeqs): row i of a sequence is the last but q_len - 1 - i of its
// k_len positions. The KV tiles that rows q0 .. q_end - 1 visit; none where every row lies before
// the first key.
inline int packed_tiles(const CacheGeom& g, const int4& seq, int q0, int q_end, bool streaming) {
  constexpr int BN = 128;
  const int off = seq.w - seq.y, tiles = (std::max(off + q_end, 0) + BN - 1) / BN;
  if (!streaming) return tiles;
  const int a_end = std::min((g.S + BN - 1) / BN, tiles);
  return a_end + std::max(0, tiles - std::max(a_end, std::max(0, g.wstart(off + q0)) / BN));
}

inline std::vector<uint64_t> packed_schedule(const CacheGeom& g, const std::vector<int4>& seqs, std::vector<int>* costs) {
  return prefill_items(
      g, (int)seqs.size(), [&](int b) { return seqs[b].y; },
      [&](int b, int q0, int q_end, bool streaming) { return packed_tiles(g, seqs[b], q0, q_end, streaming); }, costs);
}

// Folded items: 2 * span rows of all heads of a KV head, heaviest first.
inline std::vector<uint64_t> folded_schedule(const CacheGeom& g, const std::vector<int4>& seqs, int span,
                                             std::vector<int>* costs) {
  struct Entry {
    int cost, b, index;
    bool streaming;
  };
  std::vector<Entry> entries;
  size_t most = 0;
  for (int b = 0; b < (int)seqs.size(); ++b)
    for (int streaming = 0; streaming < 2; ++streaming) {
      if ((streaming ? g.n_s : g.n_r) == 0) continue;
      for (int q0 = 0; q0 < seqs[b].y; q0 += 2 * span) {
        entries.push_back({packed_tiles(g, seqs[b], q0, std::min(q0 + 2 * span, seqs[b].y), streaming != 0), b,
                           q0 / (2 * span), streaming != 0});
        most += streaming ? g.n_s : g.n_r;
      }
    }
  std::stable_sort(entries.begin(), entries.end(), [](const Entry& x, const Entry& y) { return x.cost > y.cost; });
  std::vector<uint64_t> items;
  items.reserve(most);
  costs->reserve(most);
  for (const Entry& e : entries)
    for (int i = 0; i < (e.streaming ? g.n_s : g.n_r); ++i) {
      items.push_back(prefill_item(e.b, e.streaming ? g.s_head[i] : g.r_head[i], e.index));
      costs->push_back(e.cost);
    }
  return items;
}

// Whether folded items end well before plain ones, by the work that each leaves an SM and the
// longest item, in visited tiles, with 4 tiles' time added to an item and 8 to a part of one.
// Rows of more than a few hundred tokens fill plain items, which waste no row where G does not
// divide 128 and are some percent faster then. Measured, us of a call in plain / folded items:
// 33 x 7-34 tokens, 40/8 heads of 128: 28.4 / 14.9; 4 x 17 rows after 20,000, 32/8 heads of 64:
// 100 / 48; 100 rows after 100,000, 28/4 heads of 128: 557 / 124; 4,000 tokens of 32/8 heads 94 /
// 93, of 40/8 heads 122 / 132, of 24/8 heads 77 / 81; 16 x 101-2,999, 32/8 heads, half
// streaming: 236 / 243.
inline bool packed_folds(const CacheGeom& g, const std::vector<int4>& seqs, int span, int num_sms) {
  struct Load {
    long long work = 0, items = 0;
    int longest = 0;
  };
  if (g.G == 1) return false;  // the same items: folded_split alone decides
  auto load_of = [&](auto parts) {  // parts(add): add(rows of an item, items a KV head and such rows)
    Load l;
    for (const int4& seq : seqs)
      for (int streaming = 0; streaming < 2; ++streaming) {
        const int heads = streaming ? g.n_s : g.n_r;
        if (heads == 0) continue;
        parts([&](int rows, int times) {
          for (int q0 = 0; times > 0 && q0 < seq.y; q0 += rows) {
            const int c = packed_tiles(g, seq, q0, std::min(q0 + rows, seq.y), streaming != 0);
            l.work += (long long)heads * times * c;
            l.items += heads * times;
            l.longest = std::max(l.longest, c);
          }
        });
      }
    return l;
  };
  // tiles' time to the end on clusters of c CTAs an item
  auto end_of = [&](const Load& l, int c) {
    const long long extra = c == 1 ? 4 : 8;
    return std::max((double)(l.work + l.items * c * extra) / num_sms, (double)((l.longest + c - 1) / c + extra));
  };
  const Load plain = load_of([&](auto add) { add(128, g.G / 2), add(256, g.G % 2); });
  const Load folded = load_of([&](auto add) { add(2 * span, 1); });
  double p = end_of(plain, 1), f = end_of(folded, 1);
  if (plain.longest >= 7 && plain.items <= num_sms / 2) p = std::min(p, end_of(plain, 2));
  for (int c = 2; c <= 16 && folded.longest >= 7 && folded.items * c <= 2 * num_sms; ++c)
    f = std::min(f, end_of(folded, c));
  return f < 0.9 * p;
}

// CTAs that share each folded item (clusters of 2 to 16), or 1, by the end of longest-first
// schedules in visited tiles, with 4 tiles' time added to an item and 8 to a part of one. lone:
// every item has one query tile alone, whose KV tiles the two halves of a split item's pipeline
// share (a pair of tiles takes 1.3 times one; in several waves the reads take as long either
// way). most(c): clusters of c CTAs that run at once. Measured, 16 rows, us of a call with clusters of 8 whose second query tile is empty / of 16
// whose halves share the tiles: after 50,000, 7/1 heads of 128 78 / 35, 8/1 heads of 64 64 / 26; in
// four waves, 32 sequences' rows after 8,000, unshared / shared 192 / 206. The same pipeline in
// single CTAs gained 4% there and lost 7% on 16 sequences' rows after 4,000: not used. With powers of two
// alone / these sizes: 300 rows of 32/8 heads after 20,000 111 / 83, 256 of 16/2 after 5,000 34 / 22,
// 100 of 28/4 after 100,000 148 / 124.
template <class F>
int folded_split(const std::vector<int>& costs, bool lone, F most, int num_sms, double* its_end = nullptr) {
  const int n = (int)costs.size();
  if (its_end) *its_end = 0;
  if (n > kPrefillSplitMost || n > 4 * num_sms || costs[0] < 7) return 1;
  std::vector<double> free_at;  // a min-heap
  auto end_of = [&](int slots, auto time) {
    free_at.assign(std::max(1, slots), 0.0);
    double end = 0;
    for (int cost : costs) {
      std::pop_heap(free_at.begin(), free_at.end(), std::greater<double>());
      end = std::max(end, free_at.back() += time(cost));
      std::push_heap(free_at.begin(), free_at.end(), std::greater<double>());
    }
    return end;
  };
  double best = end_of(num_sms, [](int cost) { return cost + 4.0; });
  int pick = 1;
  double work = 0;
  for (int cost : costs) work += cost;
  for (int c : {2, 3, 4, 5, 6, 8, 10, 12, 16}) {
    const int slots = most(c);
    // what the parts cost together, and a longest one, may be too much already
    const double pace = lone && n <= slots ? 0.65 : 1.0;
    if (slots < 1 || best <= std::max((work * pace + 8.0 * n * c) / (slots * c), (costs[0] + c - 1) / c * pace + 8.0)) continue;
    const double end = end_of(slots, [&](int cost) { return (cost + c - 1) / c * pace + 8.0; });
    if (end < best) {
      best = end;
      pick = c;
    }
  }
  if (its_end) *its_end = best;
  return pick;
}

// The entries of folded items in parts that CTAs of their own take, longest first, or none: where a longest-first
// schedule of them ends well before `end`, that of the items or of clusters that share them (folded_split), in
// visited tiles, with 4 tiles' time added to an item or part of one and 0.9 for each state that the last to arrive reads (133
// KB at the rate of an SM; measured up to 456 parts, 61 MB, most of which L2 holds: there is no term for states that go to HBM). Where many items are lone ones (lone: how many; folded_split) clusters are left to them,
// whose halves share such an item. Clusters begin and end together, and leave the SMs of a GPC that make no whole
// cluster idle. most_parts: of an item, 2 to kJoinedMost. Measured, us of a chunk without / with (28/4 heads of 128, half streaming with a window of 2,048, after 30,001): 2,048 rows (114
// items of 250 tiles, 114 of 18) 342 / 316 (with inputs that change from call to call 351 / 333), 8 bits 354 / 327, 4,096 651 / 642,
// 8 bits 654 / 619; close to even, 1,024 182 / 186, 512 101 / 102, 8 bits 194 / 197, 113 / 115;
// 32/8 heads, windows of 512: 600 rows after 6,000, half streaming, 52 / 49, 8 bits 60 / 53; 8 bits, 4 x 120 after 9,000, 5 heads
// streaming, 75 / 68. Not cut by this rule: 38 and 42 rows after 2,148-9,831, 40/8 heads, 31 / 40; 32/8 heads of
// 64, 8 bits, 15 x 17-21 after 17,202-28,739 (lone ones) 246 / 298, 17 x 19-59 after 6,000-12,000 (half of them) 128 / 139.
inline std::vector<uint64_t> joined_plan(const std::vector<uint64_t>& items, const std::vector<int>& costs, int lone, int num_sms,
                                         double end, int* most_parts, int* slots) {
  std::vector<uint64_t> best;
  const int n = (int)costs.size();
  if (lone > n / 5 || end <= 0 || n > kPrefillSplitMost || costs[0] < 16) return best;
  constexpr double join = 0.9;
  double limit = 0.97 * end - 2;  // (the launch that clears the counts)
  struct Entry {
    double cost;
    uint64_t entry;
  };
  std::vector<Entry> entries;
  std::vector<double> free_at;
  for (int k = 2; k <= kJoinedMost; ++k) {
    const int longest = (costs[0] + k - 1) / k;
    auto parts_of = [&](int i) { return costs[i] <= longest ? 1 : (costs[i] + longest - 1) / longest; };
    auto cost_of = [&](int i, int parts) { return parts > 1 ? (costs[i] + parts - 1) / parts + 4.0 + join : costs[i] + 4.0; };
    int all = 0, cut = 0;
    double work = 0;
    for (int i = 0; i < n; ++i) {
      const int parts = parts_of(i);
      all += parts;
      cut += parts > 1;
      work += parts * cost_of(i, parts);
    }
    if (all > kJoinedEntries || cut > kJoinedSlots || std::max(work / num_sms, longest + 4.0) + join * k >= limit) continue;
    entries.clear();
    int slot = 0;
    for (int i = 0; i < n; ++i) {
      const int parts = parts_of(i);
      for (int p = 0; p < parts; ++p)
        entries.push_back({cost_of(i, parts), joined_entry(items[i], p, parts, parts > 1 ? slot : 0)});
      slot += parts > 1;
    }
    std::stable_sort(entries.begin(), entries.end(), [](const Entry& x, const Entry& y) { return x.cost > y.cost; });
    free_at.assign(num_sms, 0.0);
    double last = 0;
    for (const Entry& e : entries) {
      std::pop_heap(free_at.begin(), free_at.end(), std::greater<double>());
      last = std::max(last, free_at.back() += e.cost);
      std::push_heap(free_at.begin(), free_at.end(), std::greater<double>());
    }
    if (last + join * k >= limit) continue;
    limit = last + join * k;
    *most_parts = k;
    *slots = slot;
    best.clear();
    for (const Entry& e : entries) best.push_back(e.entry);
  }
  return best;
}

// The work of clusters of two CTAs, two entries a cluster: two items, or one item
// twice, with kPrefillHalf, that its CTAs share (kPrefillNone fills the last
// cluster). Nothing when one CTA an item is as good.
//
// When every item's cluster runs at once, the call lasts as long as its longest
// item, and sharing all halves that. Measured (8 heads of 128, one sequence, us of
// a call without / with): 512 rows (4 tiles) 17 / 18, 640 19 / 20, 1024 22 / 21, 2048
// 33 / 26; heads of 64: 512 16 / 16, 1024 20 / 18, 2048 30 / 22.
//
// In a few waves, as in a chunk after a long prefix whose heavy items all read it,
// a last wave of heavy items that leaves many SMs idle is shared, while the
// lighter items behind it are not. k + 1 of the first k * num_sms + 1 items meet
// on one SM; where that ends a tenth later than the work spread evenly, the ends
// of longest-first schedules decide, in visited tiles, with 4 tiles' time added
// to an item and 8 to a half: nothing shared, or half a wave or a whole one from
// item k * num_sms on (from the even one below, with an odd count of SMs). Past four items an SM the last wave matters little. 28
// heads of 128, half of them streaming (S = 128, W = 2048), us of a call without /
// with: 4096 rows after 16K tokens 388 / 388 (not shared), 20K 471 / 461, 24K 555 /
// 526, 28K 638 / 585; 1024 rows after 24K 272 / 151.
inline std::vector<uint64_t> prefill_pairs(const std::vector<uint64_t>& items, const std::vector<int>& costs, int num_sms) {
  const int n = (int)items.size(), slots = num_sms / 2;
  int first = 0, last = 0;  // items [first, last) are shared
  if (n <= slots) {
    if (n > 0 && costs[0] >= 7) last = n;
  } else if (n <= std::min(4 * num_sms, kPrefillSplitMost)) {
    long long work = 0, meet = 0;
    for (int c : costs) work += c + 4;
    for (int a = 0; a < n; a += num_sms)
      if ((a / num_sms + 1) * (long long)(costs[a] + 4) > meet) {
        meet = (a / num_sms + 1) * (long long)(costs[a] + 4);
        first = a;
      }
    first &= ~1;  // the halves of an item are entries 2 i and 2 i + 1 at any count of SMs
    if (meet * num_sms * 10 > work * 11) {
      std::vector<int> free_at;  // a min-heap
      auto end_of = [&](int count, int shared_end) {
        free_at.assign(count, 0);
        int end = 0;
        for (int i = 0; i < n;) {
          const bool half = i >= first && i < shared_end;
          std::pop_heap(free_at.begin(), free_at.end(), std::greater<int>());
          end = std::max(end, free_at.back() += half ? (costs[i] + 1) / 2 + 8 : costs[i] + 4);
          std::push_heap(free_at.begin(), free_at.end(), std::greater<int>());
          i += count == num_sms || half ? 1 : 2;
        }
        return end;
      };
      int best = end_of(num_sms, 0);
      for (int window = slots; window <= 2 * slots; window += slots) {
        const int end = end_of(slots, first + window);
        if (end < best) {
          best = end;
          last = std::min(first + window, n);
        }
      }
    }
  }
  std::vector<uint64_t> pairs;
  if (last == 0) return pairs;
  pairs.reserve(n + last - first + 2);
  for (int i = 0; i < n; ++i) {
    const bool half = i >= first && i < last;
    if (half) pairs.push_back(items[i] | kPrefillHalf);
    pairs.push_back(items[i] | (half ? kPrefillHalf : 0));
  }
  if (pairs.size() & 1) pairs.push_back(kPrefillNone);
  return pairs;
}

// Whether one CTA an SM goes through all items in one pipeline instead of a CTA an
// item: many short items, whose starts and ends it overlaps. It deals them out
// beforehand, which needs several for an SM to even out, and its loop over KV tiles
// is a few percent slower. Measured, us of a call with a CTA an item / so (32/8 heads
// of 128, half streaming, S = 64, W = 512; items an SM, tiles an item): 8 x 512 (3.4,
// 2.5) 41 / 38, 16 x 512 (6.7, 2.5) 78 / 62, 8 x 1024 (6.7, 4.3) 94 / 79, 2 x 2048
// (3.4, 6.8) 60 / 62, 8 x 2048 (13.5, 6.8) 220 / 191, 1 x 4096 (3.4, 11) 80 / 87, 2 x 4096
// (6.7, 11) 154 / 146, 1 x 8192 (6.7, 19) 224 / 238, 2 x 8192 (13.5, 19) 439 / 433; 4 x 512
// (1.7, 2.5) 24 / 25; 32K tokens of 28/4 heads (24, 73) 2469 / 2609.
inline bool prefill_is_short(const std::vector<int>& costs, int num_sms) {
  const long long n = (long long)costs.size();
  long long tiles = 0;
  for (int c : costs) tiles += c;
  return n >= 3 * num_sms && tiles <= 20 * n && tiles * num_sms * 10 <= 19 * n * n;
}

}  // namespace aoh
