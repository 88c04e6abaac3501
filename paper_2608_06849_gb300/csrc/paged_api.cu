// Host runtime of the paged cache (include/aoh.h): argument validation, the plan of
// packed prompts and kernel launches on the caller's stream.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <new>
#include <vector>

#include "../../include/aoh.h"
#include "internal.h"
#include "prefill_plan.h"

using namespace aoh;

struct aoh_paged {
  aoh_paged_config cfg;
  CacheGeom geom;  // heads, S and W
  PagePool pool;
  int device = 0, num_sms = 0;
  void* meta = nullptr;  // the device arrays below
  int4* d_seqs = nullptr;
  uint32_t* d_err = nullptr;
  uint32_t* d_counters = nullptr;  // decode: arrivals, zero between calls
  float* d_states = nullptr;       // decode: states of items that CTAs share
  CUtensorMap pages;               // of the pool, which does not move
};

namespace {

aoh_status fail(aoh_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  record_error(buf);
  return st;
}

aoh_status cuda_fail(cudaError_t e, const char* what) {
  return fail(AOH_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

aoh_status check_config(const aoh_paged_config* cfg) {
  if (!cfg) return fail(AOH_ERR_INVALID, "cfg is NULL");
  const aoh_paged_config& c = *cfg;
  if (c.n_q_heads < 1 || c.n_kv_heads < 1) return fail(AOH_ERR_INVALID, "n_q_heads and n_kv_heads must be >= 1");
  if (c.n_kv_heads > kMaxKvHeads) return fail(AOH_ERR_UNSUPPORTED, "n_kv_heads > %d", kMaxKvHeads);
  if (c.n_q_heads % c.n_kv_heads) return fail(AOH_ERR_INVALID, "n_q_heads must be a multiple of n_kv_heads");
  if (c.n_q_heads / c.n_kv_heads > 16) return fail(AOH_ERR_UNSUPPORTED, "more than 16 query heads a KV head");
  if (c.d_head != 64 && c.d_head != 128) return fail(AOH_ERR_UNSUPPORTED, "d_head must be 64 or 128");
  if (c.page_size != 16 && c.page_size != 32 && c.page_size != 64 && c.page_size != 128)
    return fail(AOH_ERR_UNSUPPORTED, "page_size must be 16, 32, 64 or 128");
  if (c.n_pages < 1 || (int64_t)c.n_pages * 2 * c.n_kv_heads > (1 << 30))
    return fail(AOH_ERR_INVALID, "n_pages must be >= 1, and at most 2^29 / n_kv_heads");
  if (c.form != AOH_PAGES_BF16 && c.form != AOH_PAGES_E4M3)
    return fail(AOH_ERR_INVALID, "form %d is neither bf16 (0) nor e4m3 (1)", c.form);
  if (c.max_seqs < 1 || c.max_seqs > 65535) return fail(AOH_ERR_INVALID, "max_seqs must be in [1, 65535]");
  if (c.sink < 0 || c.window < 1 || c.sink > (1 << 30) || c.window > (1 << 30))
    return fail(AOH_ERR_INVALID, "need sink in [0, 2^30] and window in [1, 2^30]");
  return AOH_OK;
}

size_t data_bytes(const aoh_paged_config& c) {
  return (size_t)c.n_pages * 2 * c.n_kv_heads * c.page_size * c.d_head * (c.form == AOH_PAGES_BF16 ? 2 : 1);
}

size_t bytes_for(const aoh_paged_config& c) {
  const size_t rows = (size_t)c.n_pages * 2 * c.n_kv_heads * c.page_size;
  return data_bytes(c) + (c.form == AOH_PAGES_E4M3 ? rows : 0);
}

// What every call on a handle checks: the handle and the current device.
aoh_status check_handle(const aoh_paged* h) {
  if (!h) return fail(AOH_ERR_INVALID, "the paged cache is NULL");
  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
  if (dev != h->device)
    return fail(AOH_ERR_INVALID, "the paged cache belongs to device %d; the current device is %d", h->device, dev);
  return AOH_OK;
}

aoh_status check_seqs(const aoh_paged* h, int32_t n_seqs) {
  if (n_seqs < 0 || n_seqs > h->cfg.max_seqs)
    return fail(AOH_ERR_INVALID, "n_seqs = %d is outside [0, max_seqs = %d]", n_seqs, h->cfg.max_seqs);
  return AOH_OK;
}

// A tensor of rows [heads][d_head]: pointer and token stride.
aoh_status check_rows(const char* name, const void* p, int64_t stride, int heads, int d) {
  if (!p) return fail(AOH_ERR_INVALID, "%s must not be NULL", name);
  if (!aligned(p, 16)) return fail(AOH_ERR_INVALID, "%s must be 16-byte aligned", name);
  if (stride < (int64_t)heads * d || stride % 8 || stride >= (int64_t)1 << 38)
    return fail(AOH_ERR_INVALID, "the token stride of %s, %lld elements, must be a multiple of 8 and at least %d", name,
                (long long)stride, heads * d);
  return AOH_OK;
}

aoh_status check_table(const aoh_paged* h, const int32_t* table, int32_t table_stride) {
  if (!table || !aligned(table, 4)) return fail(AOH_ERR_INVALID, "table must be a 4-byte aligned device pointer");
  if (table_stride < 1 || (int64_t)table_stride * h->cfg.page_size > INT32_MAX)
    return fail(AOH_ERR_INVALID, "table_stride must be >= 1 and its pages hold less than 2^31 tokens");
  return AOH_OK;
}

PageRows page_rows(const int32_t* cu, int32_t n_seqs, int32_t n_rows, const int32_t* table, int32_t table_stride) {
  PageRows r;
  r.cu = cu;
  r.table = table;
  r.table_stride = table_stride;
  r.n_seqs = n_seqs;
  r.n_rows = n_rows;
  return r;
}

aoh_status check_cu(const int32_t* cu, int32_t n_seqs, int32_t n_rows) {
  if (n_rows < 0) return fail(AOH_ERR_INVALID, "n_rows must be >= 0");
  if (!cu && n_rows != n_seqs) return fail(AOH_ERR_INVALID, "without cu_rows, n_rows must be n_seqs");
  if (n_seqs == 0 && n_rows > 0) return fail(AOH_ERR_INVALID, "rows without a sequence");
  return AOH_OK;
}

}  // namespace

extern "C" {

size_t aoh_paged_bytes(const aoh_paged_config* cfg) {
  if (check_config(cfg) != AOH_OK) return 0;
  return bytes_for(*cfg);
}

aoh_status aoh_paged_init(const aoh_paged_config* cfg, const uint8_t* head_labels, void* pool, size_t pool_bytes,
                          aoh_paged** out) {
  if (!out) return fail(AOH_ERR_INVALID, "out is NULL");
  *out = nullptr;
  const aoh_status st = check_config(cfg);
  if (st != AOH_OK) return st;
  const aoh_paged_config& c = *cfg;
  if (!head_labels) return fail(AOH_ERR_INVALID, "head_labels is NULL");
  for (int h = 0; h < c.n_kv_heads; ++h)
    if (head_labels[h] != AOH_RETRIEVAL && head_labels[h] != AOH_STREAMING)
      return fail(AOH_ERR_INVALID, "head_labels[%d] = %d is neither retrieval (0) nor streaming (1)", h,
                  (int)head_labels[h]);
  if (!pool) return fail(AOH_ERR_INVALID, "pool is NULL");
  if (!aligned(pool, 256)) return fail(AOH_ERR_INVALID, "pool must be 256-byte aligned");
  if (pool_bytes < bytes_for(c))
    return fail(AOH_ERR_CAPACITY, "pool has %zu bytes, the pages need %zu", pool_bytes, bytes_for(c));

  aoh_paged* h = new (std::nothrow) aoh_paged();
  if (!h) return fail(AOH_ERR_CUDA, "out of host memory");
  h->cfg = c;
  CacheGeom& g = h->geom;
  memset(&g, 0, sizeof(g));
  g.Hq = c.n_q_heads;
  g.Hkv = c.n_kv_heads;
  g.D = c.d_head;
  g.G = c.n_q_heads / c.n_kv_heads;
  g.S = c.sink;
  g.W = c.window;
  for (int k = 0; k < c.n_kv_heads; ++k) {
    g.kind[k] = head_labels[k];
    if (head_labels[k] == AOH_RETRIEVAL) {
      g.idx[k] = (uint8_t)g.n_r;
      g.r_head[g.n_r++] = (uint8_t)k;
    } else {
      g.idx[k] = (uint8_t)g.n_s;
      g.s_head[g.n_s++] = (uint8_t)k;
    }
  }
  PagePool& p = h->pool;
  p.data = pool;
  p.powers = c.form == AOH_PAGES_E4M3 ? static_cast<int8_t*>(pool) + data_bytes(c) : nullptr;
  p.n_pages = c.n_pages;
  p.ps = c.page_size;
  while ((1 << p.lg_ps) < p.ps) ++p.lg_ps;
  p.form = c.form;
  p.Hkv = c.n_kv_heads;
  p.D = c.d_head;

  cudaError_t e = cudaGetDevice(&h->device);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&h->num_sms, cudaDevAttrMultiProcessorCount, h->device);
  const size_t counters = ((size_t)h->num_sms * 3 * 4 + 255) / 256 * 256;
  const size_t seqs = ((size_t)c.max_seqs * sizeof(int4) + 255) / 256 * 256;
  const size_t meta = 256 + counters + seqs + paged_state_floats(h->num_sms, c.d_head) * 4;
  if (e == cudaSuccess) e = cudaMalloc(&h->meta, meta);
  if (e == cudaSuccess) e = cudaMemset(h->meta, 0, meta);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e != cudaSuccess) {
    if (h->meta) cudaFree(h->meta);
    delete h;
    return cuda_fail(e, "metadata allocation");
  }
  uint8_t* base = static_cast<uint8_t*>(h->meta);
  h->d_err = reinterpret_cast<uint32_t*>(base);
  h->d_counters = reinterpret_cast<uint32_t*>(base + 256);
  h->d_seqs = reinterpret_cast<int4*>(base + 256 + counters);
  h->d_states = reinterpret_cast<float*>(base + 256 + counters + seqs);
  if (!make_pages_map(&h->pages, h->pool)) {
    cudaFree(h->meta);
    delete h;
    return fail(AOH_ERR_CUDA, "cuTensorMapEncodeTiled failed for the pages");
  }
  *out = h;
  return AOH_OK;
}

aoh_status aoh_paged_append(aoh_paged* cache, const void* k, const void* v, int64_t k_stride, int64_t v_stride,
                            const int32_t* cu_rows, const int32_t* lens, int32_t n_seqs, int32_t n_rows,
                            const int32_t* table, int32_t table_stride, void* stream) {
  aoh_status st = check_handle(cache);
  if (st == AOH_OK) st = check_seqs(cache, n_seqs);
  if (st == AOH_OK) st = check_cu(cu_rows, n_seqs, n_rows);
  if (st != AOH_OK || n_rows == 0) return st;
  const aoh_paged_config& c = cache->cfg;
  st = check_rows("k", k, k_stride, c.n_kv_heads, c.d_head);
  if (st == AOH_OK) st = check_rows("v", v, v_stride, c.n_kv_heads, c.d_head);
  if (st == AOH_OK) st = check_table(cache, table, table_stride);
  if (st != AOH_OK) return st;
  if (!lens) return fail(AOH_ERR_INVALID, "lens must not be NULL");
  PagedAppendArgs a;
  a.pool = cache->pool;
  a.rows = page_rows(cu_rows, n_seqs, n_rows, table, table_stride);
  a.k = k;
  a.v = v;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.lens = lens;
  a.err = cache->d_err;
  const cudaError_t e = launch_paged_append(a, cache->num_sms, (cudaStream_t)stream);
  return e == cudaSuccess ? AOH_OK : cuda_fail(e, "paged append launch");
}

aoh_status aoh_paged_read(aoh_paged* cache, const int32_t* cu_rows, const int32_t* first, int32_t n_seqs,
                          int32_t n_rows, const int32_t* table, int32_t table_stride, void* k_out, void* v_out,
                          void* stream) {
  aoh_status st = check_handle(cache);
  if (st == AOH_OK) st = check_seqs(cache, n_seqs);
  if (st == AOH_OK) st = check_cu(cu_rows, n_seqs, n_rows);
  if (st != AOH_OK || n_rows == 0) return st;
  const aoh_paged_config& c = cache->cfg;
  const int64_t dense = (int64_t)c.n_kv_heads * c.d_head;
  st = check_rows("k_out", k_out, dense, c.n_kv_heads, c.d_head);
  if (st == AOH_OK) st = check_rows("v_out", v_out, dense, c.n_kv_heads, c.d_head);
  if (st == AOH_OK) st = check_table(cache, table, table_stride);
  if (st != AOH_OK) return st;
  PagedReadArgs a;
  a.pool = cache->pool;
  a.rows = page_rows(cu_rows, n_seqs, n_rows, table, table_stride);
  a.k = k_out;
  a.v = v_out;
  a.first = first;
  a.err = cache->d_err;
  const cudaError_t e = launch_paged_read(a, cache->num_sms, (cudaStream_t)stream);
  return e == cudaSuccess ? AOH_OK : cuda_fail(e, "paged read launch");
}

aoh_status aoh_paged_decode(aoh_paged* cache, const void* q, int64_t q_stride, const int32_t* lens, int32_t n_seqs,
                            int32_t max_len, const int32_t* table, int32_t table_stride, void* out, void* stream) {
  aoh_status st = check_handle(cache);
  if (st == AOH_OK) st = check_seqs(cache, n_seqs);
  if (st != AOH_OK || n_seqs == 0) return st;
  const aoh_paged_config& c = cache->cfg;
  st = check_rows("q", q, q_stride, c.n_q_heads, c.d_head);
  if (st == AOH_OK) st = check_rows("out", out, (int64_t)c.n_q_heads * c.d_head, c.n_q_heads, c.d_head);
  if (st == AOH_OK) st = check_table(cache, table, table_stride);
  if (st != AOH_OK) return st;
  if (!lens) return fail(AOH_ERR_INVALID, "lens must not be NULL");
  if (max_len < 0) return fail(AOH_ERR_INVALID, "max_len must be >= 0");
  // the split counts tiles of at least 128 keys in 32 bits
  if ((int64_t)n_seqs * c.n_kv_heads * (((int64_t)table_stride * c.page_size + 127) / 128) > INT32_MAX)
    return fail(AOH_ERR_INVALID, "%d sequences of up to %lld tokens are too many for one call", n_seqs,
                (long long)table_stride * c.page_size);
  PagedDecodeArgs a;
  a.pages = cache->pages;
  a.states = cache->d_states;
  a.counters = cache->d_counters;
  a.pool = cache->pool;
  a.geom = cache->geom;
  a.q = q;
  a.q_stride = q_stride;
  a.out = out;
  a.lens = lens;
  a.table = table;
  a.table_stride = table_stride;
  a.n_seqs = n_seqs;
  const int32_t holds = table_stride * c.page_size;
  a.max_len = max_len > 0 && max_len < holds ? max_len : holds;
  a.err = cache->d_err;
  a.scale_log2 = (float)(1.4426950408889634 / sqrt((double)c.d_head));
  const cudaError_t e = launch_paged_decode(a, cache->num_sms, (cudaStream_t)stream);
  return e == cudaSuccess ? AOH_OK : cuda_fail(e, "paged decode launch");
}

aoh_status aoh_paged_prefill(aoh_paged* cache, const void* q, const void* k, const void* v, int64_t q_stride,
                             int64_t k_stride, int64_t v_stride, const int32_t* q_lens, const int32_t* k_lens,
                             int32_t n_seqs, void* out, void* stream) try {
  aoh_status st = check_handle(cache);
  if (st == AOH_OK) st = check_seqs(cache, n_seqs);
  if (st != AOH_OK || n_seqs == 0) return st;
  if (!q_lens) return fail(AOH_ERR_INVALID, "q_lens must not be NULL");
  std::vector<int4> seqs;
  seqs.reserve(n_seqs);
  long long n_q = 0, n_k = 0;
  for (int b = 0; b < n_seqs; ++b) {
    const int nq = q_lens[b], nk = k_lens ? k_lens[b] : nq;
    if (nq < 0 || nk < 0) return fail(AOH_ERR_INVALID, "sequence %d has %d rows and %d keys", b, nq, nk);
    if (nq > 0) seqs.push_back(make_int4((int)n_q, nq, (int)n_k, nk));
    n_q += nq;
    n_k += nk;
    if (n_q > (1 << 30) || n_k > (1 << 30)) return fail(AOH_ERR_INVALID, "more than 2^30 rows or keys in one call");
  }
  if (n_q == 0) return AOH_OK;
  const aoh_paged_config& c = cache->cfg;
  st = check_rows("q", q, q_stride, c.n_q_heads, c.d_head);
  if (st == AOH_OK) st = check_rows("out", out, (int64_t)c.n_q_heads * c.d_head, c.n_q_heads, c.d_head);
  if (st == AOH_OK && n_k > 0) st = check_rows("k", k, k_stride, c.n_kv_heads, c.d_head);
  if (st == AOH_OK && n_k > 0) st = check_rows("v", v, v_stride, c.n_kv_heads, c.d_head);
  if (st != AOH_OK) return st;

  FoldedArgs a;
  memset(&a, 0, sizeof(a));
  a.geom = cache->geom;
  a.out = out;
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.err = cache->d_err;
  a.scale_log2 = (float)(1.4426950408889634 / sqrt((double)c.d_head));
  a.span = 128 / a.geom.G;
  a.rcp = 65536 / a.geom.G + 1;
  const bool folds = packed_folds(a.geom, seqs, a.span, cache->num_sms);
  // without any key there is nothing to load, and the maps stand for the queries
  const bool keys = n_k > 0;
  if (!make_rows_map(&a.tq, q, 1, n_q, c.n_q_heads, c.d_head, q_stride, folds ? a.span : 128, folds ? a.geom.G : 1) ||
      !make_rows_map(&a.tk, keys ? k : q, 1, keys ? n_k : n_q, c.n_kv_heads, c.d_head, keys ? k_stride : q_stride) ||
      !make_rows_map(&a.tv, keys ? v : q, 1, keys ? n_k : n_q, c.n_kv_heads, c.d_head, keys ? v_stride : q_stride))
    return fail(AOH_ERR_CUDA, "cuTensorMapEncodeTiled failed for q/k/v");
  cudaStream_t s = (cudaStream_t)stream;
  if (seqs.size() <= (size_t)PackedSeqs::kMost) {
    std::copy(seqs.begin(), seqs.end(), a.seqs.by_value);
  } else {
    a.seqs.table = cache->d_seqs;
    const cudaError_t e = launch_packed_seqs(cache->d_seqs, seqs, s);
    if (e != cudaSuccess) return cuda_fail(e, "sequence upload launch");
  }
  std::vector<int> costs;
  // the pipeline over short items takes no item without a tile
  auto is_short = [&] { return costs.back() > 0 && prefill_is_short(costs, cache->num_sms); };
  cudaError_t e;
  std::vector<uint64_t> items;
  int split = 1;
  bool lone = true;
  if (folds || a.geom.G == 1) {
    items = folded_schedule(a.geom, seqs, a.span, &costs);
    for (const int4& b : seqs) lone = lone && b.y <= a.span;
    split = folded_split(costs, lone, decode_tc_max_clusters, cache->num_sms);
  }
  // With one query head a KV head both kinds are the same items, and two CTAs share a plain one at
  // less cost; more than two share folded ones alone, which is worth it from some tiles on. 8/8 heads,
  // plain / folded: 1,100 rows (9 tiles) 14.7 / 16.4 us, 300 after 5,000 (42) 36.5 / 22.2, 17 after
  // 2,000 18.7 / 8.8, after 20,000 110 / 23.
  if (folds || (lone ? split > 1 : split > 2 && costs[0] >= 16)) {
    e = launch_prefill_folded(a, items, split, split == 1 && is_short(), cache->num_sms, s);
  } else {
    costs.clear();
    items = packed_schedule(a.geom, seqs, &costs);
    const std::vector<uint64_t> pairs = prefill_pairs(items, costs, cache->num_sms);
    e = launch_prefill_packed(a, items, pairs, pairs.empty() && is_short(), cache->num_sms, s);
  }
  return e == cudaSuccess ? AOH_OK : cuda_fail(e, "packed prefill launch");
} catch (const std::exception& x) {
  return fail(AOH_ERR_CUDA, "packed prefill: %s", x.what());
}

aoh_status aoh_paged_check(aoh_paged* cache, void* stream) {
  const aoh_status st = check_handle(cache);
  if (st != AOH_OK) return st;
  cudaError_t e = cudaStreamSynchronize((cudaStream_t)stream);
  if (e != cudaSuccess) return cuda_fail(e, "cudaStreamSynchronize");
  uint32_t err = 0;
  e = cudaMemcpy(&err, cache->d_err, sizeof(err), cudaMemcpyDeviceToHost);
  // a launch that gave up may have left arrivals behind
  if (e == cudaSuccess && (err & kErrTimeout)) e = cudaMemset(cache->d_counters, 0, (size_t)cache->num_sms * 3 * 4);
  if (e == cudaSuccess && err) e = cudaMemset(cache->d_err, 0, sizeof(err));
  if (e != cudaSuccess) return cuda_fail(e, "error word");
  if (err & kErrTimeout) return fail(AOH_ERR_TIMEOUT, "a kernel's bounded wait ran out (error word 0x%x)", err);
  if (err) return fail(AOH_ERR_INVALID, "a length or a page of a call's tables was out of range (error word 0x%x)", err);
  return AOH_OK;
}

void aoh_paged_destroy(aoh_paged* cache) {
  if (!cache) return;
  if (cache->meta) cudaFree(cache->meta);
  delete cache;
}

}  // extern "C"
