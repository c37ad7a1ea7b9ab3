// Attention over bf16 keys, in pages or packed (attn_kernels.h has the kernels), and how an
// attention is split.
#include "attn_kernels.h"

// Workgroups up to which the keys are split.
constexpr int64_t kStepGroups = 4 * kCUs, kRowsGroups = 2 * kCUs;
// Columns of a group, on average, from which one token each takes k_attn_wide (behind 8192 keys, 8 kv
// heads, bf16: 32 columns 27.7 us as steps, 28.1 so; 48: 30.1, 27.5; 128: 38.3, 32.5; over 8-bit
// keys 26.4 and 26.1 at 48; four groups of 32: 41.5, 50.4).  fp32 rows take three products and one wave
// per SIMD, and stay steps.
constexpr int64_t kWideGroup = 48;


int aio_attn_plan(const aio_seqs& s, int H, int Hkv, int hd, int dtype, AttnPlan* p,
                  int key_bytes) {
  *p = AttnPlan{};
  if (s.n_seqs < 0 || s.n_rows < 0 || s.max_len < 0 || s.max_len > (1 << 30)) return AIO_ERANGE;
  if (Hkv < 1 || H < 1 || H % Hkv) return AIO_EINVAL;
  if (H / Hkv > kMaxGroup || (hd != 64 && hd != 128)) return AIO_EUNSUPPORTED;
  p->rows = s.cu_q_dev || s.cu_k_dev;
  if (!p->rows && s.n_rows != s.n_seqs) return AIO_ERANGE;
  const int64_t G = H / Hkv;
  const bool fp32 = dtype == AIO_F32;
  p->splits = 1;
  if (!p->rows) {
    // Splits of at least 128 keys (a block of 32 per wave), up to the workgroups that the
    // GPU holds at once, or twice as many for many sequences, whose lengths differ.  Up to 7
    // sequences the smaller limit never lost (7 of 37 to 4096 keys, 8 kv heads: 23.6
    // against 28.7 us; 2 of 32768, 32 kv heads: 169 against 173).  Beyond, it depends on how
    // evenly the smaller one fills the CUs and how far the lengths lie apart, which
    // the host does not know: 8 of 37 to 4096 keys 25.0 with the smaller one, 30.0 with the larger;
    // 16: 38.5, 48.5; 24: 55.1, 50.6; 14 of 1000 to 20000: 124, 109; 24: 232, 192; 24 of 30000 to
    // 32768: 493, 511; 10 of 8192, 32 kv heads: 234, 217.  None up to 512 keys: a launch that joins
    // them costs more than four blocks per wave.
    const int64_t units = std::max<int64_t>(1, ((int64_t)s.max_len + 127) / 128);
    const int64_t base = std::max<int64_t>(1, (int64_t)s.n_seqs * Hkv);
    const int64_t most = s.n_seqs < 8 ? kStepGroups / 2 : kStepGroups;
    const int64_t want = s.max_len <= 512 ? 1 : std::max<int64_t>(1, std::min(units, most / base));
    p->chunk = (int)((units + want - 1) / want * 128);
    p->splits = (int)std::max<int64_t>(1, ((int64_t)s.max_len + p->chunk - 1) / p->chunk);
    p->groups = (int64_t)s.n_seqs * Hkv * p->splits;
  } else {
    // Tiles of 256 rows stage each key for twice the rows; where that leaves less than
    // four rounds of workgroups, 128 balance better (one prompt of 8192 rows, 32 heads: 594
    // against 564 us; eight of up to 2048, 8 kv heads: 136 against 143)
    p->waves = fp32 || (int64_t)s.n_rows * G / 256 * Hkv < 4 * kCUs ? 4 : 8;
    // 8-bit keys become bf16 once per workgroup: 256 rows as soon as sequences fill half of them
    // (six of 600 rows behind 2000 keys, 16 heads on 8: 123 us in tiles of 128, 95 of 256; six of 64 rows
    // 50 and 46; one of 64 rows 28 and 32).
    if (key_bytes == 1 && !fp32 && (int64_t)s.n_rows * G >= 128 * (int64_t)s.n_seqs &&
        (int64_t)s.n_rows * G * Hkv >= 4096)
      p->waves = 8;
    // (full tiles, and a last one of each sequence that has rows)
    const int64_t full = (int64_t)s.n_rows * G / (32 * p->waves);
    p->tiles = full + std::min(s.n_seqs, s.n_rows);
    const int64_t base = std::max<int64_t>(1, (full + s.n_seqs) * Hkv);
    // Few tiles: their keys are split until the workgroups that a CU holds are there (one
    // with fp32 queries, two with bf16), down to one key tile each (5 rows behind 3000 keys,
    // at most 256 keys per split: 25 us, 64: 17)
    const int64_t units = std::max<int64_t>(1, ((int64_t)s.max_len + kKeys - 1) / kKeys);
    p->splits = (int)std::max<int64_t>(1, std::min(units, kRowsGroups / (fp32 ? 2 : 1) / base));
    p->groups = p->tiles * Hkv * p->splits;
  }
  if (p->groups > (p->waves == 8 ? kMostGroups512 : kMostGroups) ||
      (int64_t)s.n_rows * H > 0x7fffffff)
    return AIO_ERANGE;
  if (p->rows && (int64_t)s.n_rows * G > 0x7fffffff - 256) return AIO_ERANGE;
  // Keys of a large batch pass the caches by: those of the next layer come before they are
  // read again (217 MB of at most 403: 59.3 against 55.6 us, 1.07 GB: 188 against 172).  A
  // small one's may stay in the 256 MB in front of memory.  (Below 2^24 sequences x heads
  // are left here, so the product stays in 64 bits.)
  p->stream = !p->rows && (int64_t)s.n_seqs * s.max_len * Hkv * hd * 2 * key_bytes > (int64_t)64 << 20;
  if (p->splits > 1) p->ws = (size_t)p->splits * s.n_rows * H * (hd + 2) * 4;
  return AIO_OK;
}

int aio_groups_plan(const aio_seqs& s, const aio_prefixes& x, int H, int Hkv, int hd, int dtype,
                    AttnPlan* p, PrefixArgs* px, int key_bytes) {
  *px = PrefixArgs{};
  if (x.n_groups < 0 || x.n_groups > (1 << 30) || x.max_prefix < 0) return AIO_ERANGE;
  const int rc = aio_attn_plan(s, H, Hkv, hd, dtype, p, key_bytes);
  const int most_shared = std::min(x.max_prefix, s.max_len);
  if (rc || x.n_groups == 0 || most_shared < kSharedUnit || s.n_rows == 0 || s.n_seqs == 0) return rc;
  const int64_t G = H / Hkv;
  px->n = x.n_groups;
  px->max = most_shared;
  // A place for every full tile of the groups' rows, and one more for each group with rows.
  p->wide = !p->rows && dtype == AIO_BF16 && (int64_t)s.n_rows * G >= kWideGroup * (int64_t)x.n_groups;
  const int64_t width = p->rows ? 32 * p->waves : p->wide ? 32 * kWaves : kMaxGroup;
  const int64_t tiles = (int64_t)s.n_rows * G / width + std::min(x.n_groups, s.n_rows);
  auto splits = [](int64_t most, int64_t base, int64_t units) {
    return (int)std::max<int64_t>(1, std::min(units, most / std::max<int64_t>(1, base)));
  };
  const int64_t most_rows = dtype == AIO_F32 ? kRowsGroups / 2 : kRowsGroups;
  const int64_t units = ((int64_t)s.max_len + kKeys - 1) / kKeys;
  const int64_t shared_units = (most_shared + kKeys - 1) / kKeys;
  const int64_t own = p->rows ? p->tiles : s.n_seqs;
  // (128 keys each of what the longest may have beyond the longest prefix, where both are given
  // closely; four at least, for sequences that share less.  Splits without keys are not free: about
  // 220 workgroups start in a microsecond)
  const int64_t own_units = std::max<int64_t>(
      std::min<int64_t>(4, (units + 1) / 2), ((int64_t)s.max_len - most_shared) / 128 + 1);
  if (p->rows) {
    // One round of workgroups, the own keys' among them; a sequence's own keys are split from
    // kOwnPer key tiles on.
    px->own = splits(most_rows / 2, own * Hkv, (units + kOwnPer - 1) / kOwnPer);
    px->S = splits(most_rows - std::min(most_rows / 2, own * Hkv), tiles * Hkv, shared_units);
  } else if (p->wide) {
    // (a shared workgroup per CU at least, own ones beside it: 48 rows of 32 heads on 8 behind 8192
    // keys take 38.7 us with 12 splits, 35.7 with 16, 46 with 32)
    px->own = splits(kRowsGroups, own * Hkv, own_units);
    px->S = splits(std::max<int64_t>(kCUs, kRowsGroups - own * Hkv), tiles * Hkv, shared_units);
  } else {
    px->S = splits(kStepGroups, tiles * Hkv, (shared_units + 1) / 2);
    px->own = splits(kStepGroups, own * Hkv, own_units);
  }
  const int64_t shared = tiles * Hkv * px->S;
  p->groups = shared + own * Hkv * px->own;
  if (p->groups > (p->waves == 8 ? kMostGroups512 : kMostGroups)) return AIO_ERANGE;
  px->groups = (int)shared;
  px->by_s = make_udiv((unsigned)(tiles * Hkv), (unsigned)p->groups);
  p->splits = px->S + px->own;
  p->stream = false;
  p->ws = (size_t)p->splits * s.n_rows * H * (hd + 2) * 4;
  return AIO_OK;
}

int aio_attention_plan(const aio_seqs* s, int H, int Hkv, int hd, int dtype, int32_t* out) {
  if (!s || !out) return AIO_EINVAL;
  AttnPlan p;
  const int rc = aio_attn_plan(*s, H, Hkv, hd, dtype, &p);
  if (rc) return rc;
  out[0] = p.waves;
  out[1] = p.splits;
  out[2] = p.stream;
  return AIO_OK;
}

int aio_groups_attention_plan(const aio_seqs* s, const aio_prefixes* x, int H, int Hkv, int hd,
                              int dtype, int key_bytes, int32_t* out) {
  if (!s || !x || !out) return AIO_EINVAL;
  AttnPlan p;
  PrefixArgs px;
  const int rc = aio_groups_plan(*s, *x, H, Hkv, hd, dtype, &p, &px, key_bytes);
  if (rc) return rc;
  out[0] = p.waves;
  out[1] = p.wide;
  out[2] = px.S;
  out[3] = px.S ? px.own : p.splits;
  out[4] = px.groups;
  return AIO_OK;
}

size_t aio_attn_workspace_bound(int H, int Hkv, int hd) {
  // step: splits n Hkv <= kStepGroups, so splits n H <= kStepGroups G; rows: splits tiles
  // Hkv <= kRowsGroups and n_rows G <= 256 tiles, so splits n_rows H <= 256 kRowsGroups
  const size_t rh = std::max<size_t>((size_t)kStepGroups * (H / Hkv), (size_t)kRowsGroups * 256);
  return rh * (hd + 2) * 4;
}

hipError_t aio_launch_attention(const AttnArgs& a, const AttnPlan& p, int hd, int dtype,
                                hipStream_t stream) {
  return launch_any<false, false>(a, p, hd, dtype, stream);
}
