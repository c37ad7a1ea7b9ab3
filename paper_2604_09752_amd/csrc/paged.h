// What the kernels over several sequences share: how a sequence's rows and
// keys are found, and how an attention is split.
#pragma once

#include <stddef.h>

#include "aio.h"
#include "lanes.h"

// Page sizes: powers of two from 8, so that the 8 keys of an aligned group lie
// in one page, to 256.
constexpr int kMinPage = 8, kMaxPage = 256;

// Most query heads per kv head: the columns of a 16-wide matrix instruction.
constexpr int kMaxGroup = 16;

// CUs that the splits are made for: those of the one GPU this is written for.
// (Sizes of workspaces are asked for without a device.)
constexpr int kCUs = 256;
// A grid's axis holds fewer than 2^32 threads: workgroups of 256 or 512 of them.
constexpr int64_t kMostGroups = 0xffffffffll / 256, kMostGroups512 = 0xffffffffll / 512;
// Counts that go out in several launches, each of at most 65535: up to here 32 bits hold the
// step past the last.
constexpr int32_t kMostSteps = 0x7fff0000;

// AIO_OK, or what the entry points return for this pool.
int aio_check_paged(const aio_paged_kv& kv);
// Blocks of `size` in a grid of n1 x n2, s1 and s2 apart (none negative): whether two of them
// share an element.
bool aio_grid_overlaps(int64_t n1, int64_t s1, int64_t n2, int64_t s2, int64_t size);
// Two lists of n rows, of wa and wb bytes: whether any rows share a byte (also true where ranges
// of different strides mingle).
bool aio_rows_overlap(const void* a, int64_t sa, int64_t wa, const void* b, int64_t sb, int64_t wb,
                      int64_t n);
// The same for the tests (not part of the ABI; pure host), by addresses.
extern "C" int aio_rows_overlap_test(int64_t a, int64_t sa, int64_t wa, int64_t b, int64_t sb,
                                     int64_t wb, int64_t n);
// Pages or heads that would take each other's rows, or K those of V, in n_layers layers
// (one: layer_stride 0): not to be written.
bool aio_pages_overlap(const aio_paged_kv& kv);
bool aio_pool_overlaps(const aio_paged_kv& kv, int64_t layer_stride, int32_t n_layers);

// A pure host description of one attention's launch.
struct AttnPlan {
  bool rows;       // several rows per sequence (k_attn_rows), else one (k_attn_step)
  int splits;      // workgroups over the keys
  int waves;       // of a workgroup (k_attn_rows)
  bool stream;     // keys pass the caches by (k_attn_step)
  int chunk;       // keys per split (k_attn_step); 0: the splits share a tile's key blocks
  int64_t tiles;   // row tiles of all sequences, at most (k_attn_rows)
  int64_t groups;  // workgroups
  size_t ws;       // bytes of partial results
  bool wide;       // one token each in groups of many columns (k_attn_wide)
};
// AIO_OK, or the error that the entry points return for these sizes.
// (key_bytes: of an element of the keys)
int aio_attn_plan(const aio_seqs& s, int H, int Hkv, int hd, int dtype, AttnPlan* p,
                  int key_bytes = 2);
// The same with groups (PrefixArgs's sizes); without any that can share, as without groups
// (px->S: 0).
struct PrefixArgs;
int aio_groups_plan(const aio_seqs& s, const aio_prefixes& x, int H, int Hkv, int hd, int dtype,
                    AttnPlan* p, PrefixArgs* px, int key_bytes = 2);
// What an attention takes, for the tests (not part of the ABI; pure host): out[3] = waves of
// a workgroup of prompt rows (0: one new token per sequence), splits of the keys, and
// whether the keys pass the caches by.
extern "C" int aio_attention_plan(const aio_seqs* s, int H, int Hkv, int hd, int dtype,
                                  int32_t* out);
// The same with groups (over 8-bit keys: key_bytes 1): out[5] = waves of a workgroup of prompt
// rows (0: one new token per sequence), whether shared keys are taken as those, splits of the
// shared and of the own keys (0, 1: nothing is shared), workgroups of the shared part.
extern "C" int aio_groups_attention_plan(const aio_seqs* s, const aio_prefixes* x, int H, int Hkv,
                                         int hd, int dtype, int key_bytes, int32_t* out);
// No attention of these heads takes more workspace, whatever its sequences.
size_t aio_attn_workspace_bound(int H, int Hkv, int hd);

// Where an attention's keys lie: pages, or (table null) packed rows.
struct KeysArgs {
  const uint16_t* k;    // (8-bit pages: their codes)
  const uint16_t* v;
  int64_t stride;       // elements between pages, packed: between rows
  int64_t head_stride;
  int limit;            // pages, packed: rows
  int shift;            // log2 of the page size
  int Hkv;
  const int32_t* table;
  int tstride;
  const int32_t* lens;  // pages
  const int32_t* cu_k;  // packed
};

struct AttnArgs {
  KeysArgs kv;
  const int32_t* cu_q;  // null: row i of sequence i
  int n_seqs, n_rows, max_len;
  int H, G;
  UDiv by_g, by_hkv, by_s;
  const void* q;
  void* out;
  float* lse;
  int64_t ldq, ldo;
  float scale_log2;  // scores in units of log2
  int S, chunk;
  float* part_o;     // [S][n_rows][H][hd]
  float* part_ml;    // [S][n_rows][H][2]: maximum (log2 units), sum
};

// The bytes of 8-bit rows.
struct ExpArgs {
  const uint8_t* k;
  const uint8_t* v;
  int64_t stride, head_stride;
};

// Groups of sequences that share their first keys (the shared part's workgroups come first).
struct PrefixArgs {
  const int32_t* cu_seqs;  // [n + 1]
  const int32_t* lens;     // [n]
  int n, max;
  int S, own;              // splits of a group's shared keys and of a sequence's own
  int groups;              // workgroups of the shared part
  UDiv by_s;               // ... of one split of it
};

// What 8-bit keys and groups take besides.
struct AttnMoreArgs : AttnArgs {
  ExpArgs exp;
  PrefixArgs px;  // S = px.S + px.own
};

// Over bf16 keys; over 8-bit ones; the same with groups of shared keys.
hipError_t aio_launch_attention(const AttnArgs& a, const AttnPlan& p, int hd, int dtype,
                                hipStream_t stream);
hipError_t aio_launch_attention8(const AttnMoreArgs& a, const AttnPlan& p, int hd, int dtype,
                                 hipStream_t stream);
hipError_t aio_launch_attention_groups(const AttnMoreArgs& a, const AttnPlan& p, int hd, int dtype,
                                       hipStream_t stream);
hipError_t aio_launch_attention8_groups(const AttnMoreArgs& a, const AttnPlan& p, int hd, int dtype,
                                        hipStream_t stream);

struct AppendArgs {
  KeysArgs kv;          // pages
  uint16_t* k;          // (8-bit pages: their codes)
  uint16_t* v;
  const int32_t* cu_q;
  int n_seqs, n_rows, max_len, hd;
  const void* k_rows;
  const void* v_rows;
  int64_t row_stride, head_stride;
};
hipError_t aio_launch_append(const AppendArgs& a, int dtype, hipStream_t stream);
struct Append8Args : AppendArgs {
  uint8_t* k_exp;
  uint8_t* v_exp;
  int64_t exp_stride, exp_head_stride;
};
hipError_t aio_launch_append8(const Append8Args& a, int dtype, hipStream_t stream);

struct QkArgs {
  const void* in[2];     // queries, keys
  void* out[2];
  int64_t ldi[2], ldo[2];
  const uint16_t* w[2];  // null: 1
  int n_rows, H, Hkv;
  const int32_t* pos;
  float eps;
  double turns[64];      // of pair i per position: base^(-2i / hd) / 2 pi
};
hipError_t aio_launch_qk(const QkArgs& a, int hd, int dtype, hipStream_t stream);

// One launch's copies travel in the kernel's arguments (4 KB at most): no
// memory that has to outlive the call, or to be kept apart per stream.
constexpr int kCopyPairs = 448;
struct CopyArgs {
  char* pool;
  int64_t plane, stride;
  int64_t bytes;
  int n;
  int32_t pair[kCopyPairs][2];
};
hipError_t aio_launch_copy(const CopyArgs& a, int planes, hipStream_t stream);

struct LogprobPlan {
  int slices;  // workgroups per row
  int per;     // values per slice
  size_t ws;
};
LogprobPlan aio_logprob_plan(int rows, int n, int top);
struct LogprobArgs {
  const void* x;
  int rows, n, top;
  int64_t stride;
  const int32_t* target;
  float* logprob;
  float* entropy;
  int32_t* ids;
  float* top_lp;
  int slices, per;
  double* part;          // [rows][slices][3]: maximum, sum, weighted sum
  uint64_t* part_top;    // [rows][slices][top]
};
hipError_t aio_launch_logprobs(const LogprobArgs& a, int dtype, hipStream_t stream);

#ifdef __HIPCC__
// Keys of sequence i in pages, within what the caller promised and the table
// has room for (device values are not trusted).
AIO_DEV int paged_len(const KeysArgs& kv, int i, int max_len) {
  const int64_t room = (int64_t)kv.tstride << kv.shift;
  const int m = (int)min((int64_t)max_len, room);
  return max(0, min(kv.lens[i], m));
}

// First row and number of rows of sequence i.
AIO_DEV void seq_rows(const int32_t* cu_q, int n_rows, int i, int& first, int& count) {
  if (!cu_q) {
    first = i;
    count = 1;
    return;
  }
  first = min(max(cu_q[i], 0), n_rows);
  // (both ends bounded before they are subtracted: what lies there may be any number)
  count = max(min(max(cu_q[i + 1], 0), n_rows) - first, 0);
}
#endif
