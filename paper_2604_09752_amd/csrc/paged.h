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
};
// AIO_OK, or the error that the entry points return for these sizes.
int aio_attn_plan(const aio_seqs& s, int H, int Hkv, int hd, int dtype, AttnPlan* p);
// What an attention takes, for the tests (not part of the ABI; pure host): out[3] = waves of
// a workgroup of prompt rows (0: one new token per sequence), splits of the keys, and
// whether the keys pass the caches by.
extern "C" int aio_attention_plan(const aio_seqs* s, int H, int Hkv, int hd, int dtype,
                                  int32_t* out);
// No attention of these heads takes more workspace, whatever its sequences.
size_t aio_attn_workspace_bound(int H, int Hkv, int hd);

// Where an attention's keys lie: pages, or (table null) packed rows.
struct KeysArgs {
  const uint16_t* k;
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

hipError_t aio_launch_attention(const AttnArgs& a, const AttnPlan& p, int hd, int dtype,
                                hipStream_t stream);

struct AppendArgs {
  KeysArgs kv;          // pages
  uint16_t* k;
  uint16_t* v;
  const int32_t* cu_q;
  int n_seqs, n_rows, max_len, hd;
  const void* k_rows;
  const void* v_rows;
  int64_t row_stride, head_stride;
};
hipError_t aio_launch_append(const AppendArgs& a, int dtype, hipStream_t stream);

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
