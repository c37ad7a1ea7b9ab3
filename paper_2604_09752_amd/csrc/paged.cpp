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

KeysArgs paged_keys(const aio_q8_kv& kv, const aio_seqs& s) {
  const aio_paged_kv as = {kv.k_dev,   kv.v_dev,     kv.page_stride, kv.head_stride,
                           kv.n_pages, kv.page_size, kv.n_kv_heads,  kv.head_dim};
  return paged_keys(as, s);
}

int check_q8(const aio_q8_kv& kv) {
  if (!good(kv.k_dev, 16) || !good(kv.v_dev, 16) || !good(kv.k_exp_dev, 8) ||
      !good(kv.v_exp_dev, 8))
    return AIO_EINVAL;
  if (kv.n_pages < 1 || kv.n_kv_heads < 1 || kv.page_stride < 0 || kv.page_stride % 16 ||
      kv.head_stride < 0 || kv.head_stride % 16 || kv.exp_page_stride < 0 ||
      kv.exp_page_stride % 8 || kv.exp_head_stride < 0 || kv.exp_head_stride % 8)
    return AIO_EINVAL;
  if (!page_size_ok(kv.page_size) || (kv.head_dim != 64 && kv.head_dim != 128))
    return AIO_EUNSUPPORTED;
  return AIO_OK;
}

typedef __int128 wide;  // (addresses and strides are any 64-bit numbers)
wide floor_div(wide a, wide b) { return a / b - (a % b < 0); }  // b > 0

// Blocks of `size` bytes in a grid of pages and heads.
struct Blocks {
  const void* at;
  int64_t page, head, size;
};

// Rows of n blocks, of na and nb bytes, sa and sb apart, the second row d behind the first: whether a
// block of one and one of the other share a byte.
bool lines_overlap(wide d, int64_t n, int64_t sa, wide na, int64_t sb, wide nb) {
  if (d >= (n - 1) * (wide)sa + na || -d >= (n - 1) * (wide)sb + nb) return false;
  if (n == 1) return true;
  if (sa == sb) {
    if (sa == 0) return true;  // (d lies between -nb and na)
    // the first of the differences d + t s, |t| < n, above -nb
    const wide t = std::max<wide>(floor_div(-nb - d, sa) + 1, -(n - 1));
    return t < n && d + t * sa < na;
  }
  for (int64_t i = 0; i < n; ++i) {
    const wide at = d - i * (wide)sa;  // from block i of the first row
    const wide j = sb ? std::max<wide>(floor_div(-nb - at, sb) + 1, 0) : 0;
    if (j < n && at + j * sb < na && at + j * sb > -nb) return true;
  }
  return false;
}

// Whether a block of one grid and one of the other share a byte.
bool grids_overlap(const Blocks& a, const Blocks& b, int64_t pages, int64_t heads) {
  const wide d = (wide)(uintptr_t)b.at - (wide)(uintptr_t)a.at;
  // all heads of a page, all pages of a head, as one block each: what pools look like
  const wide a_heads = (heads - 1) * (wide)a.head + a.size, b_heads = (heads - 1) * (wide)b.head + b.size;
  if (a.page == b.page && !lines_overlap(d, pages, a.page, a_heads, b.page, b_heads)) return false;
  const wide a_pages = (pages - 1) * (wide)a.page + a.size, b_pages = (pages - 1) * (wide)b.page + b.size;
  if (!lines_overlap(d, heads, a.head, a_pages, b.head, b_pages)) return false;
  if (pages == 1) return true;  // (one block each indeed)
  auto at = [&](wide from) { return lines_overlap(from, pages, a.page, a.size, b.page, b.size); };
  if (a.head == b.head) {
    for (int64_t h = 1 - heads; h < heads; ++h)
      if (at(d + h * (wide)a.head)) return true;
    return false;
  }
  for (int64_t i = 0; i < heads; ++i) {
    // the heads of b that begin before the last page of a's head i ends, from the first that
    // ends behind its start
    const wide from = d - i * (wide)a.head;
    wide j = b.head ? std::max<wide>(floor_div(-b_pages - from, b.head) + 1, 0) : 0;
    for (; j < heads && from + j * b.head < a_pages; ++j)
      if (at(from + j * b.head)) return true;
  }
  return false;
}

// Codes, bytes, K or V that would take each other's place.
bool q8_overlaps(const aio_q8_kv& kv) {
  const int64_t codes = (int64_t)kv.page_size * kv.head_dim, exps = kv.page_size;
  if (aio_grid_overlaps(kv.n_pages, kv.page_stride, kv.n_kv_heads, kv.head_stride, codes) ||
      aio_grid_overlaps(kv.n_pages, kv.exp_page_stride, kv.n_kv_heads, kv.exp_head_stride, exps))
    return true;
  const Blocks all[] = {{kv.k_dev, kv.page_stride, kv.head_stride, codes},
                        {kv.v_dev, kv.page_stride, kv.head_stride, codes},
                        {kv.k_exp_dev, kv.exp_page_stride, kv.exp_head_stride, exps},
                        {kv.v_exp_dev, kv.exp_page_stride, kv.exp_head_stride, exps}};
  for (int i = 0; i < 4; ++i)
    for (int j = i + 1; j < 4; ++j)
      if (grids_overlap(all[i], all[j], kv.n_pages, kv.n_kv_heads)) return true;
  return false;
}

ExpArgs q8_exps(const aio_q8_kv& kv) {
  return {(const uint8_t*)kv.k_exp_dev, (const uint8_t*)kv.v_exp_dev, kv.exp_page_stride,
          kv.exp_head_stride};
}

// What both appends check of their sequences and rows: AIO_OK, kNothing where there are no
// rows, or an error.
constexpr int kNothing = 1;
int check_append(const aio_seqs& s, const void* k_rows, const void* v_rows, int32_t dtype,
                 int64_t row_stride, int64_t head_stride) {
  if (s.n_seqs < 0 || s.n_rows < 0 || s.max_len < 0) return AIO_ERANGE;
  if (!s.cu_q_dev && s.n_rows != s.n_seqs) return AIO_ERANGE;
  if (s.n_rows > kMostGroups) return AIO_ERANGE;
  if (dtype != AIO_F32 && dtype != AIO_BF16) return AIO_EINVAL;
  const int64_t unit = dtype == AIO_F32 ? 4 : 8;
  if (row_stride < 0 || row_stride % unit || head_stride < 0 || head_stride % unit)
    return AIO_EINVAL;
  if (s.n_rows == 0 || s.n_seqs == 0) return kNothing;
  return good(k_rows, 16) && good(v_rows, 16) ? AIO_OK : AIO_EINVAL;
}

template <class KV>
void set_append(AppendArgs& t, const KV& kv, const aio_seqs& s, const void* k_rows,
                const void* v_rows, int64_t row_stride, int64_t head_stride) {
  t.kv = paged_keys(kv, s);
  t.k = (uint16_t*)kv.k_dev;
  t.v = (uint16_t*)kv.v_dev;
  t.cu_q = s.cu_q_dev;
  t.n_seqs = s.n_seqs;
  t.n_rows = s.n_rows;
  t.max_len = s.max_len;
  t.hd = kv.head_dim;
  t.k_rows = k_rows;
  t.v_rows = v_rows;
  t.row_stride = row_stride;
  t.head_stride = head_stride;
}

// What all attentions check of the rows, and their launch: over 8-bit keys with exps, with
// groups that share keys with groups.
int attention(const KeysArgs& keys, const ExpArgs* exps, int Hkv, int hd, const aio_seqs& s,
              const aio_prefixes* groups_of, const aio_attn& a, void* ws, size_t ws_bytes,
              void* stream) {
  AttnPlan p;
  PrefixArgs px{};
  const int key_bytes = exps ? 1 : 2;
  const int rc = groups_of ? aio_groups_plan(s, *groups_of, a.n_heads, Hkv, hd, a.dtype, &p, &px,
                                             key_bytes)
                           : aio_attn_plan(s, a.n_heads, Hkv, hd, a.dtype, &p, key_bytes);
  if (rc) return rc;
  if (groups_of && groups_of->n_groups > 0 &&
      (!good(groups_of->cu_seqs_dev, 4) || !good(groups_of->prefix_lens_dev, 4)))
    return AIO_EINVAL;
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
  AttnMoreArgs t{};
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
  const int own = px.S ? px.own : p.splits;  // splits of a sequence's own keys
  t.by_s = make_udiv(p.rows ? (unsigned)(p.tiles * Hkv) : (unsigned)own, groups);
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
  if (exps) t.exp = *exps;
  if (px.S) {
    t.px = px;
    t.px.cu_seqs = groups_of->cu_seqs_dev;
    t.px.lens = groups_of->prefix_lens_dev;
  }
  const auto launch = px.S ? (exps ? aio_launch_attention8_groups : aio_launch_attention_groups)
                           : aio_launch_attention8;
  return done(px.S || exps ? launch(t, p, hd, a.dtype, (hipStream_t)stream)
                           : aio_launch_attention(t, p, hd, a.dtype, (hipStream_t)stream));
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

bool aio_rows_overlap(const void* a, int64_t sa, int64_t wa, const void* b, int64_t sb, int64_t wb,
                      int64_t n) {
  const wide x = (uintptr_t)a, y = (uintptr_t)b;
  if (x + (wide)(n - 1) * sa + wa <= y || y + (wide)(n - 1) * sb + wb <= x) return false;
  if (sa != sb || n == 1 || sa == 0) return true;
  // rows of one stride: the one's place within the other's
  const wide d = x < y ? (y - x) % sa : (sa - (x - y) % sa) % sa;
  return d < wa || d + wb > sa;
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

int aio_rows_overlap_test(int64_t a, int64_t sa, int64_t wa, int64_t b, int64_t sb, int64_t wb,
                          int64_t n) {
  return aio_rows_overlap((const void*)a, sa, wa, (const void*)b, sb, wb, n);
}

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
  return attention(paged_keys(*kv, *s), nullptr, kv->n_kv_heads, kv->head_dim, *s, nullptr, *a,
                   ws_dev, ws_bytes, hip_stream);
}

int aio_q8_attention(const aio_q8_kv* kv, const aio_seqs* s, const aio_attn* a, void* ws_dev,
                     size_t ws_bytes, void* hip_stream) {
  if (!kv || !s || !a) return AIO_EINVAL;
  if (s->cu_k_dev) return AIO_EINVAL;
  int rc = check_q8(*kv);
  if (rc == AIO_OK) rc = check_table(*s);
  if (rc) return rc;
  const ExpArgs e = q8_exps(*kv);
  return attention(paged_keys(*kv, *s), &e, kv->n_kv_heads, kv->head_dim, *s, nullptr, *a, ws_dev,
                   ws_bytes, hip_stream);
}

size_t aio_q8_workspace_bytes(const aio_seqs* s, int32_t n_heads, int32_t n_kv_heads,
                              int32_t head_dim) {
  if (!s) return 0;
  size_t most = 0;
  for (const int dtype : {AIO_F32, AIO_BF16}) {
    AttnPlan p;
    if (aio_attn_plan(*s, n_heads, n_kv_heads, head_dim, dtype, &p, 1) == AIO_OK)
      most = std::max(most, p.ws);
  }
  return most;
}

size_t aio_prefix_workspace_bytes(const aio_seqs* s, const aio_prefixes* x, int32_t n_heads,
                                  int32_t n_kv_heads, int32_t head_dim) {
  if (!s || !x) return 0;
  size_t most = 0;
  for (const int dtype : {AIO_F32, AIO_BF16})
    for (const int key_bytes : {1, 2}) {
      AttnPlan p;
      PrefixArgs px;
      if (aio_groups_plan(*s, *x, n_heads, n_kv_heads, head_dim, dtype, &p, &px, key_bytes) ==
          AIO_OK)
        most = std::max(most, p.ws);
    }
  return most;
}

int aio_prefix_attention(const aio_paged_kv* kv, const aio_seqs* s, const aio_prefixes* x,
                         const aio_attn* a, void* ws_dev, size_t ws_bytes, void* hip_stream) {
  if (!kv || !s || !x || !a) return AIO_EINVAL;
  if (s->cu_k_dev) return AIO_EINVAL;
  int rc = aio_check_paged(*kv);
  if (rc == AIO_OK) rc = check_table(*s);
  if (rc) return rc;
  return attention(paged_keys(*kv, *s), nullptr, kv->n_kv_heads, kv->head_dim, *s, x, *a, ws_dev,
                   ws_bytes, hip_stream);
}

int aio_q8_prefix_attention(const aio_q8_kv* kv, const aio_seqs* s, const aio_prefixes* x,
                            const aio_attn* a, void* ws_dev, size_t ws_bytes, void* hip_stream) {
  if (!kv || !s || !x || !a) return AIO_EINVAL;
  if (s->cu_k_dev) return AIO_EINVAL;
  int rc = check_q8(*kv);
  if (rc == AIO_OK) rc = check_table(*s);
  if (rc) return rc;
  const ExpArgs e = q8_exps(*kv);
  return attention(paged_keys(*kv, *s), &e, kv->n_kv_heads, kv->head_dim, *s, x, *a, ws_dev,
                   ws_bytes, hip_stream);
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
  return attention(k, nullptr, kv->n_kv_heads, kv->head_dim, *s, nullptr, *a, ws_dev, ws_bytes,
                   hip_stream);
}

int aio_page_append(const aio_paged_kv* kv, const aio_seqs* s, const void* k_rows_dev,
                    const void* v_rows_dev, int32_t dtype, int64_t row_stride,
                    int64_t head_stride, void* hip_stream) {
  if (!kv || !s) return AIO_EINVAL;
  int rc = aio_check_paged(*kv);
  if (rc == AIO_OK) rc = check_table(*s);
  if (rc) return rc;
  rc = check_append(*s, k_rows_dev, v_rows_dev, dtype, row_stride, head_stride);
  if (rc < 0) return rc;
  if (aio_pages_overlap(*kv)) return AIO_EINVAL;
  if (rc == kNothing) return AIO_OK;
  // (the same rows to one place for K and V are written twice, but alike)
  if ((kv->k_dev != kv->v_dev || k_rows_dev != v_rows_dev) && aio_pool_overlaps(*kv, 0, 1))
    return AIO_EINVAL;
  AppendArgs t{};
  set_append(t, *kv, *s, k_rows_dev, v_rows_dev, row_stride, head_stride);
  return done(aio_launch_append(t, dtype, (hipStream_t)hip_stream));
}

int aio_q8_append(const aio_q8_kv* kv, const aio_seqs* s, const void* k_rows_dev,
                  const void* v_rows_dev, int32_t dtype, int64_t row_stride,
                  int64_t head_stride, void* hip_stream) {
  if (!kv || !s) return AIO_EINVAL;
  int rc = check_q8(*kv);
  if (rc == AIO_OK) rc = check_table(*s);
  if (rc) return rc;
  rc = check_append(*s, k_rows_dev, v_rows_dev, dtype, row_stride, head_stride);
  if (rc < 0) return rc;
  if (q8_overlaps(*kv)) return AIO_EINVAL;
  if (rc == kNothing) return AIO_OK;
  Append8Args t{};
  set_append(t, *kv, *s, k_rows_dev, v_rows_dev, row_stride, head_stride);
  t.k_exp = (uint8_t*)kv->k_exp_dev;
  t.v_exp = (uint8_t*)kv->v_exp_dev;
  t.exp_stride = kv->exp_page_stride;
  t.exp_head_stride = kv->exp_head_stride;
  return done(aio_launch_append8(t, dtype, (hipStream_t)hip_stream));
}

int aio_qk_norm_rope(const aio_qk_rows* r, const int32_t* positions_dev,
                     const void* q_weight_dev, const void* k_weight_dev, float eps, float base,
                     void* hip_stream) {
  if (!r) return AIO_EINVAL;
  if (r->n_rows < 0 || r->n_rows > kMostGroups || r->n_heads < 1 || r->n_heads > (1 << 16) ||
      r->n_kv_heads < 1 || r->n_kv_heads > (1 << 16))
    return AIO_ERANGE;
  if (r->head_dim != 64 && r->head_dim != 128) return AIO_EUNSUPPORTED;
  if (r->dtype != AIO_F32 && r->dtype != AIO_BF16) return AIO_EINVAL;
  if (!(eps > 0.f) || !isfinite(eps) || !(base > 1.f) || !isfinite(base)) return AIO_EINVAL;
  const int64_t size = r->dtype == AIO_F32 ? 4 : 2;
  const int64_t strides[4] = {r->q_stride, r->k_stride, r->q_out_stride, r->k_out_stride};
  for (const int64_t n : strides)
    if (n < 0 || n > ((int64_t)1 << 56) || n * size % 16) return AIO_EINVAL;
  const int64_t q_width = r->n_heads * r->head_dim * size, k_width = r->n_kv_heads * r->head_dim * size;
  const struct Rows {
    const void* p;
    int64_t stride, width;  // bytes
  } rows[4] = {{r->q_dev, strides[0] * size, q_width},
               {r->k_dev, strides[1] * size, k_width},
               {r->q_out_dev, strides[2] * size, q_width},
               {r->k_out_dev, strides[3] * size, k_width}};
  for (int i = 2; i < 4; ++i)
    if (r->n_rows > 1 && rows[i].stride < rows[i].width) return AIO_EINVAL;
  if (r->n_rows == 0) return AIO_OK;
  for (const Rows& x : rows)
    if (!good(x.p, 16)) return AIO_EINVAL;
  if (!good(positions_dev, 4) || !aligned(q_weight_dev, 16) || !aligned(k_weight_dev, 16))
    return AIO_EINVAL;
  // every output against the other and against what is read, but for its own place
  for (int o = 2; o < 4; ++o)
    for (int i = 0; i < 4; ++i) {
      if (i == o || (i == o - 2 && rows[i].p == rows[o].p &&
                     (r->n_rows == 1 || rows[i].stride == rows[o].stride)))
        continue;
      if (aio_rows_overlap(rows[o].p, rows[o].stride, rows[o].width, rows[i].p, rows[i].stride,
                           rows[i].width, r->n_rows))
        return AIO_EINVAL;
    }
  QkArgs t{};
  for (int i = 0; i < 2; ++i) {
    t.in[i] = rows[i].p;
    t.out[i] = (void*)rows[2 + i].p;
    t.ldi[i] = strides[i];
    t.ldo[i] = strides[2 + i];
  }
  t.w[0] = (const uint16_t*)q_weight_dev;
  t.w[1] = (const uint16_t*)k_weight_dev;
  t.n_rows = r->n_rows;
  t.H = r->n_heads;
  t.Hkv = r->n_kv_heads;
  t.pos = positions_dev;
  t.eps = eps;
  const double pi = 3.14159265358979323846;
  for (int i = 0; i < r->head_dim / 2; ++i)
    t.turns[i] = pow((double)base, -2.0 * i / r->head_dim) / (2 * pi);
  return done(aio_launch_qk(t, r->head_dim, r->dtype, (hipStream_t)hip_stream));
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
