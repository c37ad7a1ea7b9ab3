// Host side of the operators over several sequences (include/aio.h): argument
// checks and launches, and the page tables.
#include <math.h>
#include <string.h>

#include <algorithm>
#include <functional>
#include <new>
#include <utility>
#include <vector>

#include "aio_internal.h"
#include "paged.h"

namespace {

bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
bool good(const void* p, uintptr_t to) { return p && aligned(p, to); }
int done(hipError_t e) { return e == hipSuccess ? AIO_OK : aio_hip_fail(e); }

bool page_size_ok(int32_t n) { return n >= kMinPage && n <= kMaxPage && (n & (n - 1)) == 0; }

int check_table(const aio_seqs& s) {
  if (s.n_seqs == 0) return AIO_OK;
  if (!good(s.lens_dev, 4) || !good(s.table_dev, 4) || !aligned(s.cu_q_dev, 4)) return AIO_EINVAL;
  if (s.table_stride < 1) return AIO_EINVAL;
  return AIO_OK;
}

KeysArgs paged_keys(const aio_paged_kv& kv, const aio_seqs& s) {
  KeysArgs k{};
  k.k = (const uint16_t*)kv.k_dev;
  k.v = (const uint16_t*)kv.v_dev;
  k.stride = kv.page_stride;
  k.head_stride = kv.head_stride;
  k.limit = kv.n_pages;
  while ((1 << k.shift) < kv.page_size) ++k.shift;
  k.Hkv = kv.n_kv_heads;
  k.table = s.table_dev;
  k.tstride = s.table_stride;
  k.lens = s.lens_dev;
  return k;
}

// What both attentions check of the rows, and their launch.
int attention(const KeysArgs& keys, int Hkv, int hd, const aio_seqs& s, const aio_attn& a,
              void* ws, size_t ws_bytes, void* stream) {
  AttnPlan p;
  const int rc = aio_attn_plan(s, a.n_heads, Hkv, hd, a.dtype, &p);
  if (rc) return rc;
  if (a.dtype != AIO_F32 && a.dtype != AIO_BF16) return AIO_EINVAL;
  const int64_t unit = a.dtype == AIO_F32 ? 4 : 8;  // elements in 16 bytes
  if (a.q_stride < 0 || a.q_stride % unit || a.out_stride < 0 || a.out_stride % unit)
    return AIO_EINVAL;
  // (times log2 e: an infinite factor would make every score of 0 a NaN)
  const float scale_log2 = (float)(1.4426950408889634 * (double)a.scale);
  if (!(a.scale > 0.f) || !isfinite(scale_log2)) return AIO_EINVAL;
  if (s.n_rows > 1 && a.out_stride < (int64_t)a.n_heads * hd) return AIO_EINVAL;  // (rows overlap)
  if (s.n_rows == 0 || s.n_seqs == 0) return AIO_OK;
  if (!good(a.q_dev, 16) || !good(a.out_dev, 16) || !aligned(a.lse_dev, 4)) return AIO_EINVAL;
  if (p.ws && (!good(ws, 16) || ws_bytes < p.ws)) return AIO_EINVAL;
  AttnArgs t{};
  t.kv = keys;
  t.cu_q = s.cu_q_dev;
  t.n_seqs = s.n_seqs;
  t.n_rows = s.n_rows;
  t.max_len = s.max_len;
  t.H = a.n_heads;
  t.G = a.n_heads / Hkv;
  const unsigned groups = (unsigned)p.groups;
  t.by_g = make_udiv((unsigned)t.G, (unsigned)std::min<int64_t>((int64_t)s.n_rows * t.G, 0x7fffffff));
  t.by_hkv = make_udiv((unsigned)Hkv, groups);
  t.by_s = make_udiv(p.rows ? (unsigned)(p.tiles * Hkv) : (unsigned)p.splits, groups);
  t.q = a.q_dev;
  t.out = a.out_dev;
  t.lse = a.lse_dev;
  t.ldq = a.q_stride;
  t.ldo = a.out_stride;
  t.scale_log2 = scale_log2;
  t.S = p.splits;
  t.chunk = p.chunk;
  if (p.ws) {
    t.part_o = (float*)ws;
    t.part_ml = t.part_o + (size_t)p.splits * s.n_rows * t.H * hd;
  }
  return done(aio_launch_attention(t, p, hd, a.dtype, (hipStream_t)stream));
}

}  // namespace

int aio_check_paged(const aio_paged_kv& kv) {
  if (!good(kv.k_dev, 16) || !good(kv.v_dev, 16)) return AIO_EINVAL;
  if (kv.n_pages < 1 || kv.n_kv_heads < 1 || kv.page_stride < 0 || kv.page_stride % 8 ||
      kv.head_stride < 0 || kv.head_stride % 8)
    return AIO_EINVAL;
  if (!page_size_ok(kv.page_size) || (kv.head_dim != 64 && kv.head_dim != 128))
    return AIO_EUNSUPPORTED;
  return AIO_OK;
}

bool aio_grid_overlaps(int64_t n1, int64_t s1, int64_t n2, int64_t s2, int64_t size) {
  typedef __int128 wide;  // (strides are any 63-bit numbers)
  if ((n1 > 1 && s1 < size) || (n2 > 1 && s2 < size)) return true;
  if (n1 == 1 || n2 == 1) return false;
  // one dimension within a step of the other
  if ((wide)(n1 - 1) * s1 + size <= s2 || (wide)(n2 - 1) * s2 + size <= s1) return false;
  if (n1 > n2) {
    std::swap(n1, n2);
    std::swap(s1, s2);
  }
  // i steps of one against the nearest two counts j of the other
  for (int64_t i = 1; i < n1; ++i) {
    const wide at = (wide)i * s1;
    if (at - (wide)(n2 - 1) * s2 >= size) return false;
    const wide j = at / s2;
    if ((j < n2 && at - j * s2 < size) || (j + 1 < n2 && (j + 1) * s2 - at < size)) return true;
  }
  return false;
}

bool aio_pages_overlap(const aio_paged_kv& kv) {
  return aio_grid_overlaps(kv.n_pages, kv.page_stride, kv.n_kv_heads, kv.head_stride,
                           (int64_t)kv.page_size * kv.head_dim);
}

bool aio_pool_overlaps(const aio_paged_kv& kv, int64_t layer_stride, int32_t n_layers) {
  const int64_t one = (int64_t)kv.page_size * kv.head_dim;
  const intptr_t k = (intptr_t)kv.k_dev, v = (intptr_t)kv.v_dev;
  const int64_t apart = (int64_t)(k < v ? v - k : k - v) / 2;  // K and V: a dimension of two
  const struct {
    int64_t n, stride;
  } dim[] = {{n_layers, layer_stride}, {2, apart}, {kv.n_pages, kv.page_stride},
             {kv.n_kv_heads, kv.head_stride}};
  for (int a = 0; a < 4; ++a)
    for (int b = a + 1; b < 4; ++b)
      if (aio_grid_overlaps(dim[a].n, dim[a].stride, dim[b].n, dim[b].stride, one)) return true;
  return false;
}

// ------------------------------------------------------------- page tables

struct PageSeq {
  bool open = false;
  int32_t len = 0;
  std::vector<int32_t> pages;
};

struct aio_pages {
  int32_t page_size, max_seqs;
  std::vector<int32_t> held;  // sequences that hold each page
  std::vector<int32_t> spare; // free pages, a heap whose top is the lowest
  std::vector<PageSeq> seqs;  // up to max_seqs, grown as they are opened

  PageSeq* at(int32_t s) {
    return s >= 0 && (size_t)s < seqs.size() && seqs[(size_t)s].open ? &seqs[(size_t)s] : nullptr;
  }
  const PageSeq* at(int32_t s) const { return const_cast<aio_pages*>(this)->at(s); }
  int32_t take() {
    std::pop_heap(spare.begin(), spare.end(), std::greater<int32_t>());
    const int32_t p = spare.back();
    spare.pop_back();
    held[(size_t)p] = 1;
    return p;
  }
  // (spare has room for every page: this does not allocate)
  void drop(int32_t p) {
    if (--held[(size_t)p] > 0) return;
    spare.push_back(p);
    std::push_heap(spare.begin(), spare.end(), std::greater<int32_t>());
  }
  void trim(PageSeq& s, size_t keep) {
    while (s.pages.size() > keep) {
      drop(s.pages.back());
      s.pages.pop_back();
    }
  }
  // The lowest closed place, or -1 where all are open.
  int32_t place() {
    for (size_t i = 0; i < seqs.size(); ++i)
      if (!seqs[i].open) return (int32_t)i;
    if ((int64_t)seqs.size() >= max_seqs) return -1;
    seqs.emplace_back();
    return (int32_t)seqs.size() - 1;
  }
};

namespace {
// Host memory can run out; no exception crosses the interface.
template <class F>
int guarded(F f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return AIO_ENOMEM;
  } catch (...) {
    return AIO_EINVAL;
  }
}
}  // namespace

extern "C" {

size_t aio_attn_workspace_bytes(const aio_seqs* s, int32_t n_heads, int32_t n_kv_heads,
                                int32_t head_dim) {
  if (!s) return 0;
  AttnPlan p;  // (fp32 takes no more)
  return aio_attn_plan(*s, n_heads, n_kv_heads, head_dim, AIO_BF16, &p) == AIO_OK ? p.ws : 0;
}

int aio_paged_attention(const aio_paged_kv* kv, const aio_seqs* s, const aio_attn* a,
                        void* ws_dev, size_t ws_bytes, void* hip_stream) {
  if (!kv || !s || !a) return AIO_EINVAL;
  if (s->cu_k_dev) return AIO_EINVAL;
  int rc = aio_check_paged(*kv);
  if (rc == AIO_OK) rc = check_table(*s);
  if (rc) return rc;
  return attention(paged_keys(*kv, *s), kv->n_kv_heads, kv->head_dim, *s, *a, ws_dev, ws_bytes,
                   hip_stream);
}

int aio_packed_attention(const aio_packed_kv* kv, const aio_seqs* s, const aio_attn* a,
                         void* ws_dev, size_t ws_bytes, void* hip_stream) {
  if (!kv || !s || !a) return AIO_EINVAL;
  if (kv->n_rows < 0) return AIO_ERANGE;
  if (kv->n_kv_heads < 1 || kv->row_stride < 0 || kv->row_stride % 8 || kv->head_stride < 0 ||
      kv->head_stride % 8)
    return AIO_EINVAL;
  if (!aligned(kv->k_dev, 16) || !aligned(kv->v_dev, 16) ||
      (kv->n_rows > 0 && (!kv->k_dev || !kv->v_dev)))
    return AIO_EINVAL;
  if (!good(s->cu_q_dev, 4) || !good(s->cu_k_dev, 4)) return AIO_EINVAL;
  KeysArgs k{};
  k.k = (const uint16_t*)kv->k_dev;
  k.v = (const uint16_t*)kv->v_dev;
  k.stride = kv->row_stride;
  k.head_stride = kv->head_stride;
  k.limit = kv->n_rows;
  k.Hkv = kv->n_kv_heads;
  k.cu_k = s->cu_k_dev;
  return attention(k, kv->n_kv_heads, kv->head_dim, *s, *a, ws_dev, ws_bytes, hip_stream);
}

int aio_page_append(const aio_paged_kv* kv, const aio_seqs* s, const void* k_rows_dev,
                    const void* v_rows_dev, int32_t dtype, int64_t row_stride,
                    int64_t head_stride, void* hip_stream) {
  if (!kv || !s) return AIO_EINVAL;
  int rc = aio_check_paged(*kv);
  if (rc == AIO_OK) rc = check_table(*s);
  if (rc) return rc;
  if (s->n_seqs < 0 || s->n_rows < 0 || s->max_len < 0) return AIO_ERANGE;
  if (!s->cu_q_dev && s->n_rows != s->n_seqs) return AIO_ERANGE;
  if (s->n_rows > kMostGroups) return AIO_ERANGE;
  if (aio_pages_overlap(*kv)) return AIO_EINVAL;
  if (dtype != AIO_F32 && dtype != AIO_BF16) return AIO_EINVAL;
  const int64_t unit = dtype == AIO_F32 ? 4 : 8;
  if (row_stride < 0 || row_stride % unit || head_stride < 0 || head_stride % unit)
    return AIO_EINVAL;
  if (s->n_rows == 0 || s->n_seqs == 0) return AIO_OK;
  if (!good(k_rows_dev, 16) || !good(v_rows_dev, 16)) return AIO_EINVAL;
  // (the same rows to one place for K and V are written twice, but alike)
  if ((kv->k_dev != kv->v_dev || k_rows_dev != v_rows_dev) && aio_pool_overlaps(*kv, 0, 1))
    return AIO_EINVAL;
  AppendArgs t{};
  t.kv = paged_keys(*kv, *s);
  t.k = (uint16_t*)kv->k_dev;
  t.v = (uint16_t*)kv->v_dev;
  t.cu_q = s->cu_q_dev;
  t.n_seqs = s->n_seqs;
  t.n_rows = s->n_rows;
  t.max_len = s->max_len;
  t.hd = kv->head_dim;
  t.k_rows = k_rows_dev;
  t.v_rows = v_rows_dev;
  t.row_stride = row_stride;
  t.head_stride = head_stride;
  return done(aio_launch_append(t, dtype, (hipStream_t)hip_stream));
}

int aio_page_copy(void* pool_dev, int32_t n_planes, int64_t plane_bytes, int32_t n_pages,
                  int64_t page_stride_bytes, int64_t page_bytes, const int32_t* src,
                  const int32_t* dst, int32_t n, void* hip_stream) {
  if (n < 0 || n > kMostSteps || n_planes < 1 || n_planes > kMostSteps || n_pages < 1)
    return AIO_ERANGE;
  if (plane_bytes < 0 || page_bytes < 0 || page_stride_bytes < page_bytes || plane_bytes % 16 ||
      page_bytes % 16 || page_stride_bytes % 16)
    return AIO_EINVAL;
  if (n == 0) return AIO_OK;
  if (!good(pool_dev, 16) || !src || !dst) return AIO_EINVAL;
  if (page_bytes > ((int64_t)1 << 37)) return AIO_ERANGE;  // (below kMostGroups chunks of 16 KB)
  if (aio_grid_overlaps(n_planes, plane_bytes, n_pages, page_stride_bytes, page_bytes))
    return AIO_EINVAL;
  for (int32_t i = 0; i < n; ++i)
    if (src[i] < 0 || src[i] >= n_pages || dst[i] < 0 || dst[i] >= n_pages) return AIO_ERANGE;
  const int rc = guarded([&] {
    std::vector<uint8_t> used((size_t)n_pages, 0);  // 1: a source, 2: a destination
    for (int32_t i = 0; i < n; ++i) used[(size_t)src[i]] = 1;
    for (int32_t i = 0; i < n; ++i) {
      if (used[(size_t)dst[i]]) return (int)AIO_EINVAL;
      used[(size_t)dst[i]] = 2;
    }
    return (int)AIO_OK;
  });
  if (rc || page_bytes == 0) return rc;
  CopyArgs t{};
  t.pool = (char*)pool_dev;
  t.plane = plane_bytes;
  t.stride = page_stride_bytes;
  t.bytes = page_bytes;
  for (int32_t i = 0; i < n; i += kCopyPairs) {
    t.n = std::min(n - i, kCopyPairs);
    for (int32_t j = 0; j < t.n; ++j) {
      t.pair[j][0] = src[i + j];
      t.pair[j][1] = dst[i + j];
    }
    const hipError_t e = aio_launch_copy(t, n_planes, (hipStream_t)hip_stream);
    if (e != hipSuccess) return aio_hip_fail(e);
  }
  return AIO_OK;
}

size_t aio_logprobs_workspace_bytes(int32_t rows, int32_t n, int32_t top) {
  if (rows < 1 || rows > kMostSteps || n < 1 || n > (1 << 30) || top < 0 || top > AIO_MAX_TOP)
    return 0;
  return aio_logprob_plan(rows, n, top).ws;
}

int aio_logprobs(const void* logits_dev, int32_t dtype, int32_t rows, int32_t n, int64_t stride,
                 const int32_t* targets_dev, int32_t top, float* logprob_dev, float* entropy_dev,
                 int32_t* top_ids_dev, float* top_logprobs_dev, void* ws_dev, size_t ws_bytes,
                 void* hip_stream) {
  if (rows < 0 || rows > kMostSteps || n < 1 || n > (1 << 30) || stride < n || top < 0 ||
      top > std::min(n, (int32_t)AIO_MAX_TOP))
    return AIO_ERANGE;
  if (dtype != AIO_F32 && dtype != AIO_BF16) return AIO_EINVAL;
  if (rows == 0) return AIO_OK;
  if (!good(logits_dev, dtype == AIO_F32 ? 4 : 2)) return AIO_EINVAL;
  if (!targets_dev != !logprob_dev || !aligned(targets_dev, 4) || !aligned(logprob_dev, 4) ||
      !aligned(entropy_dev, 4))
    return AIO_EINVAL;
  if (top > 0 && (!good(top_ids_dev, 4) || !good(top_logprobs_dev, 4))) return AIO_EINVAL;
  const LogprobPlan p = aio_logprob_plan(rows, n, top);
  if (p.ws && (!good(ws_dev, 16) || ws_bytes < p.ws)) return AIO_EINVAL;
  LogprobArgs t{};
  t.x = logits_dev;
  t.rows = rows;
  t.n = n;
  t.top = top;
  t.stride = stride;
  t.target = targets_dev;
  t.logprob = logprob_dev;
  t.entropy = entropy_dev;
  t.ids = top_ids_dev;
  t.top_lp = top_logprobs_dev;
  t.slices = p.slices;
  t.per = p.per;
  if (p.ws) {
    t.part = (double*)ws_dev;
    t.part_top = (uint64_t*)(t.part + (size_t)std::min(rows, 65535) * p.slices * 3);
  }
  return done(aio_launch_logprobs(t, dtype, (hipStream_t)hip_stream));
}

// ------------------------------------------------------------- page tables

int aio_pages_create(int32_t n_pages, int32_t page_size, int32_t max_seqs, aio_pages** out) {
  if (!out) return AIO_EINVAL;
  *out = nullptr;
  if (n_pages < 1 || n_pages > (1 << 30) || max_seqs < 1 || max_seqs > (1 << 30) ||
      !page_size_ok(page_size))
    return AIO_ERANGE;
  return guarded([&] {
    aio_pages* p = new aio_pages;
    try {
      p->page_size = page_size;
      p->max_seqs = max_seqs;
      p->held.assign((size_t)n_pages, 0);
      p->spare.resize((size_t)n_pages);
      for (int32_t i = 0; i < n_pages; ++i) p->spare[(size_t)i] = i;  // (ascending: a heap)
    } catch (...) {
      delete p;
      throw;
    }
    *out = p;
    return (int)AIO_OK;
  });
}

void aio_pages_destroy(aio_pages* p) { delete p; }

int aio_pages_open(aio_pages* p, int32_t* seq) {
  if (!p || !seq) return AIO_EINVAL;
  return guarded([&] {
    const int32_t i = p->place();
    if (i < 0) return (int)AIO_ENOMEM;
    p->seqs[(size_t)i].open = true;
    *seq = i;
    return (int)AIO_OK;
  });
}

int aio_pages_close(aio_pages* p, int32_t seq) {
  if (!p) return AIO_EINVAL;
  PageSeq* s = p->at(seq);
  if (!s) return AIO_ERANGE;
  p->trim(*s, 0);
  *s = PageSeq{};
  return AIO_OK;
}

int aio_pages_fork(aio_pages* p, int32_t seq, int32_t* child) {
  if (!p || !child) return AIO_EINVAL;
  if (!p->at(seq)) return AIO_ERANGE;
  return guarded([&] {
    const int32_t i = p->place();  // (may move the sequences)
    if (i < 0) return (int)AIO_ENOMEM;
    const PageSeq& s = p->seqs[(size_t)seq];
    PageSeq& c = p->seqs[(size_t)i];
    c.pages = s.pages;
    c.len = s.len;
    c.open = true;
    for (const int32_t g : c.pages) ++p->held[(size_t)g];
    *child = i;
    return (int)AIO_OK;
  });
}

int aio_pages_extend(aio_pages* p, int32_t seq, int32_t n, int32_t* src, int32_t* dst,
                     int32_t* n_copies) {
  if (!p || !src || !dst || !n_copies) return AIO_EINVAL;
  PageSeq* s = p->at(seq);
  if (!s || n < 0 || (int64_t)s->len + n > (1 << 30)) return AIO_ERANGE;
  *n_copies = 0;
  if (n == 0) return AIO_OK;
  return guarded([&] {
    const size_t have = s->pages.size();
    const size_t want = (size_t)((s->len + n + p->page_size - 1) / p->page_size);
    // the page that the next position falls into, if others hold it too
    const bool copy = s->len % p->page_size && p->held[(size_t)s->pages.back()] > 1;
    if (want - have + (copy ? 1 : 0) > p->spare.size()) return (int)AIO_ENOMEM;
    s->pages.reserve(want);
    if (copy) {
      *src = s->pages.back();
      *dst = p->take();
      --p->held[(size_t)*src];
      s->pages.back() = *dst;
      *n_copies = 1;
    }
    while (s->pages.size() < want) s->pages.push_back(p->take());
    s->len += n;
    return (int)AIO_OK;
  });
}

int aio_pages_truncate(aio_pages* p, int32_t seq, int32_t len) {
  if (!p) return AIO_EINVAL;
  PageSeq* s = p->at(seq);
  if (!s || len < 0 || len > s->len) return AIO_ERANGE;
  p->trim(*s, (size_t)((len + p->page_size - 1) / p->page_size));
  s->len = len;
  return AIO_OK;
}

int aio_pages_compact(aio_pages* p, int32_t* src, int32_t* dst, int32_t room, int32_t* n) {
  if (!p || !src || !dst || !n) return AIO_EINVAL;
  return guarded([&] {
    const size_t all = p->held.size(), used = all - p->spare.size();
    // pages behind the first `used` go to the free ones among those
    int32_t moves = 0;
    for (size_t i = used; i < all; ++i) moves += p->held[i] > 0;
    *n = moves;
    if (moves > room) return (int)AIO_ERANGE;
    std::vector<int32_t> to(all - used, -1);
    size_t hole = 0;
    int32_t k = 0;
    for (size_t i = used; i < all; ++i) {
      if (p->held[i] == 0) continue;
      while (p->held[hole] > 0) ++hole;
      src[k] = (int32_t)i;
      dst[k++] = to[i - used] = (int32_t)hole;
      p->held[hole] = p->held[i];
      p->held[i] = 0;
    }
    for (PageSeq& s : p->seqs)
      for (int32_t& g : s.pages)
        if ((size_t)g >= used) g = to[(size_t)g - used];
    for (size_t i = used; i < all; ++i) p->spare[i - used] = (int32_t)i;  // (ascending: a heap)
    return (int)AIO_OK;
  });
}

int aio_pages_row(const aio_pages* p, int32_t seq, int32_t* row, int32_t width, int32_t* len) {
  if (!p || !len) return AIO_EINVAL;
  const PageSeq* s = p->at(seq);
  if (!s) return AIO_ERANGE;
  if (row) {
    if (width < 0 || s->pages.size() > (size_t)width) return AIO_ERANGE;
    std::copy(s->pages.begin(), s->pages.end(), row);
    std::fill(row + s->pages.size(), row + width, -1);
  }
  *len = s->len;
  return AIO_OK;
}

int aio_pages_free(const aio_pages* p) { return p ? (int)p->spare.size() : AIO_EINVAL; }

}  // extern "C"
