// Host runtime of the paged cache (include/aoh.h): argument validation, the plan of
// packed prompts and kernel launches on the caller's stream.
#include <limits.h>
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <mutex>
#include <new>
#include <vector>

#include "../../include/aoh.h"
#include "internal.h"
#include "prefill_plan.h"

using namespace aoh;

constexpr int kPartsASeq = 4;

struct aoh_paged {
  aoh_paged_config cfg;
  CacheGeom geom;  // heads, S and W
  PagePool pool;
  int device = 0, num_sms = 0;
  void* meta = nullptr;  // the device arrays below
  int4* d_seqs = nullptr;  // lists of sequences, or of up to kPartsASeq parts each
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

// The rope and the norms of a rotation of heads of d numbers.
aoh_status check_rotation(const aoh_rope* rope, const aoh_norms* norms, int d) {
  if (!rope) return fail(AOH_ERR_INVALID, "rope is NULL");
  if (rope->n_pairs < 0 || rope->n_pairs % 8 || 2 * rope->n_pairs > d || (rope->interleaved != 0 && rope->interleaved != 1))
    return fail(AOH_ERR_INVALID, "rope turns %d pairs; heads of %d take a multiple of 8, at most %d (aoh_rope_init fills it)",
                rope->n_pairs, d, d / 2);
  if (!(rope->scale >= -1e30f && rope->scale <= 1e30f))
    return fail(AOH_ERR_INVALID, "the rope's scale must be within [-1e30, 1e30]");
  if (!norms || (!norms->q && !norms->k)) return AOH_OK;
  if (norms->type != AOH_NORM_BF16 && norms->type != AOH_NORM_F32)
    return fail(AOH_ERR_INVALID, "norm type %d is neither bf16 (0) nor fp32 (1)", norms->type);
  const size_t align = norms->type == AOH_NORM_F32 ? 4 : 2;
  if (!aligned(norms->q, align) || !aligned(norms->k, align))
    return fail(AOH_ERR_INVALID, "norm weights must be aligned to their numbers");
  if (!(norms->eps >= 0.f && norms->eps <= 1e30f)) return fail(AOH_ERR_INVALID, "eps must be a number >= 0");
  return AOH_OK;
}

// Rows of a rotation: their strides are 32 bits of bytes.
aoh_status check_turned_rows(const char* name, const void* p, int64_t stride, int heads, int d) {
  const aoh_status st = check_rows(name, p, stride, heads, d);
  if (st == AOH_OK && stride >= (int64_t)1 << 31)
    return fail(AOH_ERR_INVALID, "the token stride of %s, %lld elements, must be below 2^31", name, (long long)stride);
  return st;
}

// Rows written where others are read: in place alone, with the same stride.
aoh_status check_in_place(const char* name, const void* in, int64_t in_stride, const void* out, int64_t out_stride) {
  if (in == out && in_stride != out_stride)
    return fail(AOH_ERR_INVALID, "%s in place must keep its token stride", name);
  return AOH_OK;
}

void set_rotation(RotateArgs* a, const aoh_rope* rope, const aoh_norms* norms) {
  memset(a, 0, sizeof(*a));
  a->rope.n_pairs = rope->n_pairs;
  a->rope.interleaved = rope->interleaved;
  a->rope.scale = rope->scale;
  memcpy(a->rope.turns, rope->turns, sizeof(a->rope.turns));
  if (!norms) return;
  a->q_norm = norms->q;
  a->k_norm = norms->k;
  a->norm_f32 = norms->type;
  a->eps = norms->eps;
}

// SMs of the current device.
cudaError_t sm_count(int* n) {
  static std::atomic<int> known[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  *n = dev < 64 ? known[dev].load(std::memory_order_relaxed) : 0;
  if (*n > 0) return cudaSuccess;
  e = cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev);
  if (e == cudaSuccess && dev < 64) known[dev].store(*n, std::memory_order_relaxed);
  return e;
}

// Memory of calls, for pages written out as bf16 and states of items in parts: a pool of each device, which keeps
// it from call to call for all handles (a model's layers use the same), and gives it back with the last handle.
struct ExpandPools {
  static constexpr int kMost = 64;
  std::mutex lock;
  cudaMemPool_t pool[kMost] = {};
  int handles[kMost] = {};
};
ExpandPools& expand_pools() {
  static ExpandPools pools;
  return pools;
}

// One handle more or less on a device. With the last one its pool goes: what calls in flight still use follows
// once they end (a pool that is trimmed instead keeps what the host has not seen freed, for good).
void expand_memories(int device, int handles) {
  ExpandPools& p = expand_pools();
  if (device < 0 || device >= ExpandPools::kMost) return;
  std::lock_guard<std::mutex> hold(p.lock);
  p.handles[device] += handles;
  if (p.handles[device] == 0 && p.pool[device]) {
    if (cudaMemPoolDestroy(p.pool[device]) != cudaSuccess) cudaGetLastError();
    p.pool[device] = nullptr;
  }
}

// While it lives, calls of this thread that take memory or give it back are allowed beside other streams' captures,
// which they would end otherwise.
struct BesideCaptures {
  cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
  BesideCaptures() { cudaThreadExchangeStreamCaptureMode(&mode); }
  ~BesideCaptures() { cudaThreadExchangeStreamCaptureMode(&mode); }
};

// Device memory of a call that is not captured, ordered on its stream; null if there is none to be had.
void* expand_memory(int device, size_t bytes, cudaStream_t s) {
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  void* p = nullptr;
  if (device >= ExpandPools::kMost) return nullptr;
  if (cudaStreamIsCapturing(s, &capture) != cudaSuccess || capture != cudaStreamCaptureStatusNone) {
    cudaGetLastError();
    return nullptr;
  }
  const BesideCaptures relaxed;
  cudaMemPool_t pool = nullptr;
  {
    ExpandPools& pools = expand_pools();
    std::lock_guard<std::mutex> hold(pools.lock);
    if (!pools.pool[device]) {
      cudaMemPoolProps props;
      memset(&props, 0, sizeof(props));
      props.allocType = cudaMemAllocationTypePinned;
      props.location.type = cudaMemLocationTypeDevice;
      props.location.id = device;
      uint64_t keep = UINT64_MAX;
      if (cudaMemPoolCreate(&pools.pool[device], &props) != cudaSuccess) {
        pools.pool[device] = nullptr;
        cudaGetLastError();
        return nullptr;
      }
      cudaMemPoolSetAttribute(pools.pool[device], cudaMemPoolAttrReleaseThreshold, &keep);
    }
    pool = pools.pool[device];
  }
  if (cudaMallocFromPoolAsync(&p, bytes, pool, s) != cudaSuccess) {
    cudaGetLastError();
    return nullptr;
  }
  return p;
}

cudaError_t expand_free(void* p, cudaStream_t s) {
  const BesideCaptures relaxed;
  return cudaFreeAsync(p, s);
}

// Groups of `per` tiles of 128 keys that n rows at the end of `keys` positions see, `most` of a KV head at most, of all
// KV heads.
long long seen_tiles(const CacheGeom& g, int n, int keys, int per = 1, long long most = LLONG_MAX) {
  const long long all = ((long long)keys + 127) / 128, window = ((long long)g.S + g.W + n + 255) / 128;
  auto of = [&](long long tiles) { return std::min((tiles + per - 1) / per, most); };
  return g.n_r * of(all) + g.n_s * of(std::min(all, window));
}

// Calls of a few rows a sequence as parts on the decode kernel, of at most 16 columns each (query heads of a KV
// head times tokens), which reads a sequence's pages once for each part but as they lie, at the rate of HBM. What it
// takes against the tiles of 256 rows, in nanoseconds of the GPU: 10.6 a tile of 128 keys of d_head 128 and part (8
// bits: 5.5, but 8 with more than 8 columns, whose softmax takes longer than the tile's transfer) against 14 (18), and a
// start of 6 us against 10. A short item is a chain of waits on its SM: the first two tiles of the decode kernel's, of 32 KB
// of K, of each part and KV head cost 31 more (28, 38), one of the latter's 25 more, 20 in one pipeline an SM (in_line).
// work: tiles that these `items` visit. Measured, us of a call in tiles / parts: 32 x 2-5 rows after 1,000-16,000, 32/8
// heads, 8 bits 198 / 121, bf16 154 / 144; 4 rows each, 8 bits - / 98, 2 - / 69; 5 rows after 4,096, 28/4 heads, bf16 12.3 /
// 9.4; 32/8 heads, 128 x 2 rows after 20-36, 8 bits 59 / 42, 2-5 after 200-500 111 / 145, 10-15 after 9-16 61 / 181, 64 x
// 2-5 after 20-100 31 / 44, bf16 26 / 31, 256 x 2-4 after 100-300 165 / 160.
bool parts_of(const aoh_paged* h, const std::vector<int4>& seqs, const std::vector<int4>& planned, size_t items,
              long long work, bool in_line, std::vector<int4>* parts, int* tokens) {
  const CacheGeom& g = h->geom;
  const int most = 16 / g.G;
  const double scale = g.D / 128.0 * 0.001;
  const bool f8 = h->cfg.form == AOH_PAGES_E4M3;
  *tokens = 1;
  for (const int4& s : planned) {
    const int count = (s.y + most - 1) / most;
    if (count > 16) return false;
    *tokens = std::max(*tokens, (s.y + count - 1) / count);
  }
  const bool narrow = g.G * *tokens <= 8;
  const int per = !f8 ? 128 / g.D : narrow ? 256 / g.D : 2;
  long long visits = 0, waits = 0, n = 0;
  for (const int4& s : planned) {
    const int count = (s.y + most - 1) / most;
    visits += count * seen_tiles(g, s.y, s.w);
    waits += count * std::max(seen_tiles(g, s.y, s.w, per, 2), (long long)g.Hkv);
    n += count;
  }
  const double tile_ns = !f8 ? 10.6 : narrow ? 5.5 : 8, wait_ns = !f8 ? 31 : narrow ? 28 : 38, item_ns = in_line ? 20 : 25;
  if (6 + waits * wait_ns * 0.001 + visits * tile_ns * scale > 10 + items * item_ns * 0.001 + work * (f8 ? 18 : 14) * scale)
    return false;
  if (n > PackedSeqs::kMost && n > (long long)kPartsASeq * h->cfg.max_seqs) return false;  // more than the device's list holds
  parts->reserve(n);
  for (const int4& s : seqs) {
    const int count = (s.y + most - 1) / most, each = (s.y + count - 1) / count;
    for (int t = 0; t < s.y; t += each) {
      const int m = std::min(each, s.y - t);
      parts->push_back(make_int4(s.x + t, m, s.z, s.y - t - m));
    }
  }
  return true;
}

// Whether to write a call's 8-bit pages out as bf16 ones first, of as many tokens as the plan takes its sequences
// (planned) to have, and which pages they are of each (seqs; the entry behind them has their end): where its items visit the same tiles often enough. work: tiles that they visit in all.
// An item's visit costs an SM 1.1 us more with codes (d_head 128; 2,824 us of 8,192 rows after 16,384 of
// 32/8 heads, 1,626 over bf16 pages), a tile's writing 98 KB of traffic, and the two launches some 8 us.
bool expand_plan(const aoh_paged* h, const std::vector<int4>& planned, long long work, std::vector<int4>* seqs) {
  if (h->cfg.form != AOH_PAGES_E4M3) return false;
  const CacheGeom& g = h->geom;
  long long pages = 0, tiles = 0;
  for (const int4& s : planned) {
    pages += ((long long)s.w + 127) / 128;
    tiles += seen_tiles(g, s.y, s.w);
  }
  const double visit = 7.2 * g.D / 128, write = 16.4 * g.D / 128;
  if (pages == 0 || pages > (4ll << 30) / (2 * g.Hkv * 128 * g.D * 2) || work * visit < tiles * write * 1.2 + 8000) return false;
  pages = 0;
  for (size_t i = 0; i < planned.size(); ++i) {
    (*seqs)[i].w = (int)pages;
    pages += ((long long)planned[i].w + 127) / 128;
  }
  seqs->push_back(make_int4(0, 0, 0, (int)pages));
  return true;
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
  const size_t seqs = ((size_t)c.max_seqs * kPartsASeq * sizeof(int4) + 255) / 256 * 256;
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
  expand_memories(h->device, 1);
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

aoh_status aoh_rope_init(const double* inv_freq, int32_t n_pairs, int32_t interleaved, aoh_rope* out) {
  if (!out) return fail(AOH_ERR_INVALID, "out is NULL");
  memset(out, 0, sizeof(*out));
  if (n_pairs < 0 || n_pairs > 64 || n_pairs % 8)
    return fail(AOH_ERR_INVALID, "n_pairs = %d must be a multiple of 8 in [0, 64]", n_pairs);
  if (interleaved != 0 && interleaved != 1) return fail(AOH_ERR_INVALID, "interleaved must be 0 or 1");
  if (n_pairs > 0 && !inv_freq) return fail(AOH_ERR_INVALID, "inv_freq is NULL");
  for (int i = 0; i < n_pairs; ++i)
    if (!(inv_freq[i] >= -1e6 && inv_freq[i] <= 1e6))
      return fail(AOH_ERR_INVALID, "inv_freq[%d] = %g must be a number within [-1e6, 1e6]", i, inv_freq[i]);
  out->n_pairs = n_pairs;
  out->interleaved = interleaved;
  out->scale = 1.f;
  // inv_freq / 2 pi in two doubles, its whole turns dropped: whole + part, part in [-1/2, 1/2]
  constexpr double kHi = 0.15915494309189535, kLo = -9.839338337591243e-18;  // 1 / (2 pi)
  for (int i = 0; i < n_pairs; ++i) {
    const double f = inv_freq[i], p = f * kHi, rest = fma(f, kHi, -p) + f * kLo, part = p - rint(p);
    const uint64_t head = part >= 0.5 ? 1ull << 63 : (uint64_t)llrint(ldexp(part, 64));
    out->turns[i] = head + (uint64_t)llrint(ldexp(rest, 64));
  }
  return AOH_OK;
}

aoh_status aoh_norm_rotate(const aoh_rope* rope, const aoh_norms* norms, const void* q, const void* k, int64_t q_stride,
                           int64_t k_stride, const int32_t* positions, int32_t n_rows, int32_t n_q_heads,
                           int32_t n_kv_heads, int32_t d_head, void* q_out, void* k_out, int64_t q_out_stride,
                           int64_t k_out_stride, void* stream) {
  if (d_head != 64 && d_head != 128) return fail(AOH_ERR_UNSUPPORTED, "d_head must be 64 or 128");
  if (n_rows < 0) return fail(AOH_ERR_INVALID, "n_rows must be >= 0");
  if (n_q_heads < 0 || n_kv_heads < 0 || n_q_heads > 1024 || n_kv_heads > 1024)
    return fail(AOH_ERR_INVALID, "n_q_heads and n_kv_heads must be in [0, 1024]");
  aoh_status st = check_rotation(rope, norms, d_head);
  if (st != AOH_OK || n_rows == 0 || n_q_heads + n_kv_heads == 0) return st;
  if (n_q_heads > 0) {
    st = check_turned_rows("q", q, q_stride, n_q_heads, d_head);
    if (st == AOH_OK) st = check_turned_rows("q_out", q_out, q_out_stride, n_q_heads, d_head);
    if (st == AOH_OK) st = check_in_place("q", q, q_stride, q_out, q_out_stride);
  }
  if (st == AOH_OK && n_kv_heads > 0) {
    st = check_turned_rows("k", k, k_stride, n_kv_heads, d_head);
    if (st == AOH_OK) st = check_turned_rows("k_out", k_out, k_out_stride, n_kv_heads, d_head);
    if (st == AOH_OK) st = check_in_place("k", k, k_stride, k_out, k_out_stride);
  }
  if (st != AOH_OK) return st;
  if (!positions || !aligned(positions, 4)) return fail(AOH_ERR_INVALID, "positions must be a 4-byte aligned device pointer");
  RotateArgs a;
  set_rotation(&a, rope, norms);
  a.Hq = n_q_heads;
  a.Hkv = n_kv_heads;
  a.q = q;
  a.k = k;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.q_out = q_out;
  a.k_out = k_out;
  a.q_out_stride = q_out_stride;
  a.k_out_stride = k_out_stride;
  a.positions = positions;
  a.rows.n_rows = n_rows;
  int sms = 0;
  cudaError_t e = sm_count(&sms);
  if (e != cudaSuccess) return cuda_fail(e, "cudaDeviceGetAttribute");
  e = launch_rotate(a, d_head, sms, (cudaStream_t)stream);
  return e == cudaSuccess ? AOH_OK : cuda_fail(e, "rotation launch");
}

aoh_status aoh_paged_append_rotated(aoh_paged* cache, const aoh_rope* rope, const aoh_norms* norms, const void* q,
                                    const void* k, const void* v, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                                    const int32_t* positions, const int32_t* cu_rows, const int32_t* lens, int32_t n_seqs,
                                    int32_t n_rows, const int32_t* table, int32_t table_stride, void* q_out,
                                    int64_t q_out_stride, void* stream) {
  aoh_status st = check_handle(cache);
  if (st == AOH_OK) st = check_rotation(rope, norms, cache->cfg.d_head);
  if (st == AOH_OK) st = check_seqs(cache, n_seqs);
  if (st == AOH_OK) st = check_cu(cu_rows, n_seqs, n_rows);
  if (st != AOH_OK || n_rows == 0) return st;
  const aoh_paged_config& c = cache->cfg;
  st = check_turned_rows("q", q, q_stride, c.n_q_heads, c.d_head);
  if (st == AOH_OK) st = check_turned_rows("k", k, k_stride, c.n_kv_heads, c.d_head);
  if (st == AOH_OK) st = check_turned_rows("v", v, v_stride, c.n_kv_heads, c.d_head);
  if (st == AOH_OK) st = check_turned_rows("q_out", q_out, q_out_stride, c.n_q_heads, c.d_head);
  if (st == AOH_OK) st = check_in_place("q", q, q_stride, q_out, q_out_stride);
  if (st == AOH_OK) st = check_table(cache, table, table_stride);
  if (st != AOH_OK) return st;
  if (!lens || !aligned(lens, 4) || !aligned(cu_rows, 4) || !aligned(positions, 4))
    return fail(AOH_ERR_INVALID, "lens, cu_rows and positions must be 4-byte aligned device pointers, lens not NULL");
  RotateArgs a;
  set_rotation(&a, rope, norms);
  a.Hq = c.n_q_heads;
  a.Hkv = c.n_kv_heads;
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_out = q_out;
  a.q_out_stride = q_out_stride;
  a.positions = positions;
  a.rows = page_rows(cu_rows, n_seqs, n_rows, table, table_stride);
  a.pool = cache->pool;
  a.lens = lens;
  a.err = cache->d_err;
  const cudaError_t e = launch_rotate(a, c.d_head, cache->num_sms, (cudaStream_t)stream);
  return e == cudaSuccess ? AOH_OK : cuda_fail(e, "rotated append launch");
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

aoh_status aoh_paged_attend(aoh_paged* cache, const void* q, int64_t q_stride, const int32_t* q_lens, const int32_t* lens,
                            const int32_t* k_lens, int32_t n_seqs, const int32_t* table, int32_t table_stride, void* out,
                            void* stream) try {
  aoh_status st = check_handle(cache);
  if (st == AOH_OK) st = check_seqs(cache, n_seqs);
  if (st != AOH_OK || n_seqs == 0) return st;
  if (!q_lens) return fail(AOH_ERR_INVALID, "q_lens must not be NULL");
  const aoh_paged_config& c = cache->cfg;
  // what the kernel reads of the sequences that have rows, and what the plan takes them to be
  std::vector<int4> seqs, planned;
  seqs.reserve(n_seqs);
  planned.reserve(n_seqs);
  const long long holds = (long long)table_stride * c.page_size;
  long long n_q = 0;
  for (int b = 0; b < n_seqs; ++b) {
    if (q_lens[b] < 0 || (k_lens && k_lens[b] < 0))
      return fail(AOH_ERR_INVALID, "sequence %d has %d rows and %d keys", b, q_lens[b], k_lens ? k_lens[b] : 0);
    if (q_lens[b] > 0) {
      seqs.push_back(make_int4((int)n_q, q_lens[b], b, 0));
      planned.push_back(make_int4((int)n_q, q_lens[b], 0, (int)std::min(k_lens ? (long long)k_lens[b] : holds, holds)));
    }
    n_q += q_lens[b];
    if (n_q > (1 << 30)) return fail(AOH_ERR_INVALID, "more than 2^30 rows in one call");
  }
  if (n_q == 0) return AOH_OK;
  st = check_rows("q", q, q_stride, c.n_q_heads, c.d_head);
  if (st == AOH_OK) st = check_rows("out", out, (int64_t)c.n_q_heads * c.d_head, c.n_q_heads, c.d_head);
  if (st == AOH_OK) st = check_table(cache, table, table_stride);
  if (st != AOH_OK) return st;
  if (!lens || !aligned(lens, 4)) return fail(AOH_ERR_INVALID, "lens must be a 4-byte aligned device pointer");
  if (holds > (1 << 30)) return fail(AOH_ERR_INVALID, "a table's row must hold at most 2^30 tokens");
  // (rows beside a value that is not finite read their queries once more, behind their outputs)
  const __int128 row = (__int128)c.n_q_heads * c.d_head * 2, apart = (__int128)((uintptr_t)out) - (uintptr_t)q;
  if (apart < (n_q - 1) * (__int128)q_stride * 2 + row && -apart < n_q * row)
    return fail(AOH_ERR_INVALID, "out must not overlap the queries");

  cudaStream_t s = (cudaStream_t)stream;
  const int span = 128 / cache->geom.G;
  std::vector<int> costs;
  const std::vector<uint64_t> items = folded_schedule(cache->geom, planned, span, &costs);
  long long work = 0;
  for (int cost : costs) work += cost;
  std::vector<int4> parts;
  int tokens = 1;
  // (the decode kernel counts its tiles, of at least 128 keys, in 32 bits)
  const bool in_line = prefill_is_short(costs, cache->num_sms) && c.form == AOH_PAGES_BF16;
  if (parts_of(cache, seqs, planned, items.size(), work, in_line, &parts, &tokens) &&
      (int64_t)parts.size() * c.n_kv_heads * ((holds + 127) / 128) <= INT32_MAX) {
    PagedPartsArgs p;
    p.pages = cache->pages;
    p.states = cache->d_states;
    p.counters = cache->d_counters;
    p.pool = cache->pool;
    p.geom = cache->geom;
    p.q = q;
    p.q_stride = q_stride;
    p.out = out;
    p.lens = lens;
    p.table = table;
    p.table_stride = table_stride;
    p.n_seqs = (int)parts.size();
    p.max_len = 1;
    for (const int4& b : planned) p.max_len = std::max(p.max_len, b.w);
    p.err = cache->d_err;
    p.scale_log2 = (float)(1.4426950408889634 / sqrt((double)c.d_head));
    p.tokens = tokens;
    p.rcp = 65536 / cache->geom.G + 1;
    cudaError_t e = cudaSuccess;
    p.seqs.table = nullptr;
    if (parts.size() <= (size_t)PackedSeqs::kMost) {
      std::copy(parts.begin(), parts.end(), p.seqs.by_value);
    } else {
      p.seqs.table = cache->d_seqs;
      e = launch_packed_seqs(cache->d_seqs, parts, s);
    }
    if (e == cudaSuccess) e = launch_paged_parts(p, cache->num_sms, s);
    return e == cudaSuccess ? AOH_OK : cuda_fail(e, "paged attention launch");
  }

  PagedAttendArgs a;
  memset(&a, 0, sizeof(a));
  a.geom = cache->geom;
  a.out = out;
  a.q = q;
  a.q_stride = q_stride;
  a.err = cache->d_err;
  a.scale_log2 = (float)(1.4426950408889634 / sqrt((double)c.d_head));
  a.span = span;
  a.rcp = 65536 / a.geom.G + 1;
  a.pages = cache->pages;
  a.pool = cache->pool;
  a.lens = lens;
  a.table = table;
  a.table_stride = table_stride;
  a.holds = (int)holds;
  if (!make_rows_map(&a.tq, q, 1, n_q, c.n_q_heads, c.d_head, q_stride, a.span, a.geom.G))
    return fail(AOH_ERR_CUDA, "cuTensorMapEncodeTiled failed for q");
  bool lone = true;
  int lone_items = 0;
  for (const int4& b : planned) {
    lone = lone && b.y <= a.span;
    if ((b.y - 1) % (2 * a.span) < a.span) lone_items += c.n_kv_heads;
  }
  const int n_with = (int)seqs.size();
  double end = 0;
  int split = folded_split(costs, lone, decode_tc_max_clusters, cache->num_sms, &end);
  int slots = 0;
  const std::vector<uint64_t> joined = joined_plan(items, costs, lone_items, cache->num_sms, end, &a.most_parts, &slots);
  void* states = nullptr;
  if (!joined.empty()) {
    const size_t bytes = (size_t)slots * a.most_parts * 256 * (c.d_head * 4 + 8);
    states = expand_memory(cache->device, bytes + slots * sizeof(int), s);
    if (states) {
      a.states = static_cast<float4*>(states);
      a.arrived = reinterpret_cast<int*>(static_cast<uint8_t*>(states) + bytes);
      const cudaError_t e = cudaMemsetAsync(a.arrived, 0, slots * sizeof(int), s);
      if (e != cudaSuccess) {
        expand_free(states, s);
        return cuda_fail(e, "cudaMemsetAsync");
      }
      split = 1;
    }
  }
  const std::vector<uint64_t>& entries = states ? joined : items;
  const bool is_short = split == 1 && !states && prefill_is_short(costs, cache->num_sms);
  void* written = nullptr;
  if (expand_plan(cache, planned, work, &seqs))
    written = expand_memory(cache->device, (size_t)seqs[n_with].w * 2 * c.n_kv_heads * 128 * c.d_head * 2, s);
  cudaError_t e = cudaSuccess;
  if (seqs.size() <= (size_t)PackedSeqs::kMost) {
    std::copy(seqs.begin(), seqs.end(), a.seqs.by_value);
  } else {
    a.seqs.table = cache->d_seqs;
    e = launch_packed_seqs(cache->d_seqs, seqs, s);
  }
  bool covered = false;  // whether all sequences fit there, whatever their lengths
  if (written) {
    PagedAttendArgs w = a;
    w.written = 1;
    w.table = nullptr;
    w.pool.data = written;
    w.pool.powers = nullptr;
    w.pool.n_pages = seqs[n_with].w;
    w.pool.ps = 128;
    w.pool.lg_ps = 7;
    w.pool.form = AOH_PAGES_BF16;
    PagedExpandArgs x;
    memset(&x, 0, sizeof(x));
    x.from = cache->pool;
    x.to = w.pool;
    x.geom = cache->geom;
    x.seqs = a.seqs;
    x.n_seqs = n_with;
    x.lens = lens;
    x.table = table;
    x.table_stride = table_stride;
    x.holds = a.holds;
    x.err = cache->d_err;
    covered = true;
    for (int i = 0; i < n_with; ++i) covered = covered && (seqs[i + 1].w - seqs[i].w) * 128ll >= holds;
    if (e == cudaSuccess && !make_pages_map(&w.pages, w.pool)) e = cudaErrorInvalidValue;
    if (e == cudaSuccess) e = launch_paged_expand(x, s);
    if (e == cudaSuccess) e = launch_paged_attend(w, entries, split, is_short, cache->num_sms, s);
    a.written = 1;
  }
  if (e == cudaSuccess && !covered) e = launch_paged_attend(a, entries, split, is_short, cache->num_sms, s);
  for (void* p : {written, states})
    if (p) {
      const cudaError_t f = expand_free(p, s);
      if (e == cudaSuccess) e = f;
    }
  return e == cudaSuccess ? AOH_OK : cuda_fail(e, "paged attention launch");
} catch (const std::exception& x) {
  return fail(AOH_ERR_CUDA, "paged attention: %s", x.what());
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
  if (cache->meta) cudaFree(cache->meta);  // (waits for the handle's calls)
  expand_memories(cache->device, -1);
  delete cache;
}

}  // extern "C"
