// Attention over the keys of several sequences, in pages or packed: one new
// token per sequence (k_attn_step) and the rows of prompts (k_attn_rows).
//
// For a row with scores s_j = scale q.k_j over its visible keys j, with the
// running maximum m and sum l over the key blocks seen so far:
//   m' = max(m, max_j s_j),  p_j = e^(s_j - m'),  c = e^(m - m'),
//   l' = c l + sum_j p_j,    o' = c o + sum_j p_j v_j,    out = o / l.
// Two such states join by the same rule, so the keys can be split over waves
// and workgroups (k_attn_join).
//
// Both products run on MFMA with the keys (the value tile, transposed) as the
// A operand: S^T = K Q^T, O^T += V^T P^T.  A column is a query, so a lane's
// scores all belong to one query and the weights stay in registers: the k
// slots of the second product are taken in the order in which the scores of the
// first lie in a lane, and the value rows are read through transposing LDS
// reads in that order.  fp32 queries and their softmax weights are split into
// three bf16 terms each (truncation, exact), accumulated into one tile.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "paged.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWaves = 4;
constexpr int kBlock = kWaves * AIO_WAVE;

AIO_DEV bf16x8 as_bf16x8(u32x4 u) { return __builtin_bit_cast(bf16x8, u); }

AIO_DEV f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
AIO_DEV f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Eight fp32 values as NT bf16 operands: one, rounded to nearest even, or
// three that add up to the value exactly.
template <int NT>
AIO_DEV void terms(const float (&x)[8], bf16x8 (&t)[NT]) {
  if constexpr (NT == 1) {
#pragma unroll
    for (int j = 0; j < 8; ++j) t[0][j] = (__bf16)x[j];
  } else {
    uint32_t w[3][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      w[0][j] = __float_as_uint(x[j]);
      const float r1 = x[j] - __uint_as_float(w[0][j] & 0xffff0000u);
      w[1][j] = __float_as_uint(r1);
      w[2][j] = __float_as_uint(r1 - __uint_as_float(w[1][j] & 0xffff0000u));
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      u32x4 u;
#pragma unroll
      for (int j = 0; j < 4; ++j) u[j] = w[k][2 * j] >> 16 | (w[k][2 * j + 1] & 0xffff0000u);
      t[k] = as_bf16x8(u);
    }
  }
}

// Eight elements of a query row.
template <int NT>
AIO_DEV void load_query(const AttnArgs& a, int row, int head, int hd, int d0, bool live,
                        bf16x8 (&t)[NT]) {
  const int64_t at = (int64_t)row * a.ldq + (int64_t)head * hd + d0;
  if constexpr (NT == 1) {
    u32x4 u = {0, 0, 0, 0};
    if (live) u = *(const u32x4*)((const uint16_t*)a.q + at);
    t[0] = as_bf16x8(u);
  } else {
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (live) {
      const float4 u = *(const float4*)((const float*)a.q + at);
      const float4 v = *(const float4*)((const float*)a.q + at + 4);
      x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
      x[4] = v.x; x[5] = v.y; x[6] = v.z; x[7] = v.w;
    }
    terms<3>(x, t);
  }
}

AIO_DEV void store_out(const AttnArgs& a, bool f32, int64_t at, float v) {
  if (f32) ((float*)a.out)[at] = v;
  else ((uint16_t*)a.out)[at] = f32_to_bf16(v);
}

constexpr float kLn2 = 0.69314718055994530942f;

// A long sum in two floats: hi becomes the rounded hi + lo, lo what that is off by (exactly
// where hi is the larger, to 2^-24 of lo else), from which the next additions go on.  In one
// float, weights that are all alike (repeated keys) round the same way each time: 32768
// keys of one score, added one by one, left a row's sum 1.8e-4 off, 131072 9e-4.  With
// the sum carried after every block only the additions within a block round, 16 units of
// 2^-24 at most for 32 of them.
template <class T>
AIO_DEV void carry(T& hi, T& lo) {
  const T s = hi + lo;
  lo -= s - hi;
  hi = s;
}

// Output tiles of fp32 queries are carried alike, after this many blocks of 32 keys in
// k_attn_step and of 64 in k_attn_rows: 96 and 384 matrix instructions on one sum in
// between.  Equal values under 131072 equal keys: 1e-3 off in one sum of the prompt rows,
// 4e-6 carried every 32 blocks, 2e-6 every 16; 8192 rows of 32 heads take 1406, 1432 and
// 1457 us.  (bf16 outputs round to 2^-9, which no such chain comes near.)
constexpr int kStepCarry = 32, kRowsCarry = 32;

// ------------------------------------------------ one new token per sequence

// Workgroup (sequence, kv head, split): the G query heads of the kv head are
// columns of one 16-wide tile; each wave takes every fourth block of 32 keys of
// the split, and the waves' states join in LDS.  What bounds it is the reading of
// the keys and values; few requests split them until there are 4 workgroups per CU.
// Two requests of 32768 keys, 32 heads of 128, fp32: 169 us with the join, 6.3 TB/s;
// 24 of 37 to 4096 keys on 8 kv heads, bf16: 51 us; one of 129 keys: 7.4.
template <int HD>
struct StepLds {
  // bytes of a key and a value row: the 16 and the 8 rows that one access takes lie in
  // distinct banks
  static constexpr int KROW = HD * 2 + 16, VROW = HD * 2 + 32;
  static constexpr int TBYTES = 32 * VROW;  // a wave's tile: the keys, then the values
  static constexpr int OROW = HD + 4;             // floats of an output row
  static constexpr int OBYTES = kWaves * kMaxGroup * OROW * 4;
  static constexpr int TILES = kWaves * TBYTES > OBYTES ? kWaves * TBYTES : OBYTES;
  // the upper parts of a wave's output tile, and the maxima that they refer to
  static constexpr int HBYTES = HD * 16 * 4 + AIO_WAVE * 4;
  static constexpr int BYTES(int NT) { return TILES + (NT == 3 ? kWaves * HBYTES : 0); }
};

template <int HD, int NT, bool STREAM>
__global__ __launch_bounds__(kBlock, NT == 1 ? 3 : HD == 64 ? 4 : 2) void k_attn_step(AttnArgs a) {
  using L = StepLds<HD>;
  extern __shared__ __align__(16) char smem[];
  __shared__ float wm[kWaves][kMaxGroup], wl[kWaves][kMaxGroup];
  constexpr int NC = HD / 32;              // k chunks of a score product
  constexpr int TPR = HD / 8;              // lanes of a row
  constexpr int RPL = AIO_WAVE / TPR;      // rows per load: 4 or 8, all in one page
  constexpr int NV = 32 / RPL;             // loads of a tile
  constexpr int ND = HD / 16;              // output tiles
  const int tid = threadIdx.x, lane = tid & (AIO_WAVE - 1);
  const int wid = __builtin_amdgcn_readfirstlane(tid / AIO_WAVE);
  const int col = lane & 15, grp = lane >> 4;
  const int b = blockIdx.x, sh = udiv(b, a.by_s), split = b - sh * a.S;
  const int seq = udiv(sh, a.by_hkv), kvh = sh - seq * a.kv.Hkv;
  const int len = paged_len(a.kv, seq, a.max_len);
  const int c0 = split * a.chunk, c1 = min(len, c0 + a.chunk);
  const int h0 = kvh * a.G;
  if (split > 0 && c0 >= len) {  // a split without keys
    if (tid < a.G) a.part_ml[(((int64_t)split * a.n_rows + seq) * a.H + h0 + tid) * 2] = -INFINITY;
    return;
  }
  bf16x8 q[NC][NT];
#pragma unroll
  for (int c = 0; c < NC; ++c)
    load_query<NT>(a, seq, h0 + col, HD, c * 32 + 8 * grp, col < a.G, q[c]);

  const int32_t* table = a.kv.table + (int64_t)seq * a.kv.tstride;
  const int nt = (c1 - c0 + 31) / 32, pm = (1 << a.kv.shift) - 1;
  const uint16_t* kb = a.kv.k + kvh * a.kv.head_stride;
  const uint16_t* vb = a.kv.v + kvh * a.kv.head_stride;
  // Lane l holds the page of key l mod 32 of a block (-1: not visible).
  auto load_page = [&](int t) {
    const int key = c0 + t * 32 + (lane & 31);
    int p = -1;
    if (key < c1) p = table[key >> a.kv.shift];
    return (unsigned)p < (unsigned)a.kv.limit ? p : -1;
  };
  // Rows as they lie in memory, 4 or 8 per load (in the operand's order, a load of the keys
  // would take half a 128-byte line of 16 rows); the 8 keys of an aligned group share
  // a page, so pages are wave uniform.  Keys that are not visible read page 0.
  const int lr = lane / TPR, ld = lane % TPR * 8;
  u32x4 kr[NV], vr[NV];
  auto load_block = [&](u32x4 (&r)[NV], const uint16_t* from, int t, int page) {
    const int j0 = c0 + t * 32;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t at = max(__builtin_amdgcn_readlane(page, i * RPL), 0) * a.kv.stride +
                         ((j0 + i * RPL) & pm) * HD;
      const u32x4* p = (const u32x4*)(from + at + (uint32_t)(lr * HD + ld));
      r[i] = STREAM ? __builtin_nontemporal_load(p) : *p;
    }
  };
  f32x4 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f, lh = 0.f;
  // The upper parts of o wait in LDS (in registers, 20 of them spill), with the maximum of
  // then.
  f32x4* park = (f32x4*)(smem + L::TILES + wid * L::HBYTES) + lane;
  float* park_m = (float*)(smem + L::TILES + wid * L::HBYTES + HD * 16 * 4) + lane;
  auto parked_scale = [&] {
    const float mh = *park_m;
    return mh == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mh - m) * a.scale_log2);
  };
  char* tile = smem + wid * L::TBYTES;
  const char* ktr = tile + col * L::KROW + 16 * grp;
  const char* vtr = tile + (4 * grp + col / 4) * L::VROW + (col & 3) * 8;

  int page = load_page(wid), next = load_page(wid + kWaves);
  if (wid < nt) {
    load_block(kr, kb, wid, page);
    load_block(vr, vb, wid, page);
  }
  for (int t = wid; t < nt;) {
    const int te = NT == 3 ? min(nt, t + kStepCarry * kWaves) : nt;
    for (; t < te; t += kWaves) {
      const uint32_t vis = (uint32_t)__ballot(page >= 0);  // bit j: key j of the block
      // the wave's next block (its last one is read again: no branch)
      const bool more = t + kWaves < nt;
      const int tn = more ? t + kWaves : t, pn = more ? next : page;
#pragma unroll
      for (int i = 0; i < NV; ++i) *(u32x4*)(tile + (i * RPL + lr) * L::KROW + ld * 2) = kr[i];
      load_block(kr, kb, tn, pn);
      wave_lds_sync();  // the keys are in LDS
      float p[8];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const bf16x8 ak = as_bf16x8(*(const u32x4*)(ktr + kt * 16 * L::KROW + c * 64));
#pragma unroll
          for (int n = 0; n < NT; ++n) s = mfma16(ak, q[c][n], s);
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) p[4 * kt + v] = s[v];
      }
      wave_lds_sync();  // ... and read: the values take their place
      // (those that may not be seen are zero: 0 x NaN is not)
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        u32x4 w = vr[i];
        if (vis != 0xffffffffu && !(vis >> (i * RPL + lr) & 1)) w = u32x4{0, 0, 0, 0};
        *(u32x4*)(tile + (i * RPL + lr) * L::VROW + ld * 2) = w;
      }
      load_block(vr, vb, tn, pn);
      page = next;
      next = load_page(t + 2 * kWaves);
      if (vis != 0xffffffffu) {
#pragma unroll
        for (int v = 0; v < 8; ++v)
          if (!(vis >> (v / 4 * 16 + 4 * grp + v % 4) & 1)) p[v] = -INFINITY;
      }
      float mx = p[0];
#pragma unroll
      for (int v = 1; v < 8; ++v) mx = fmaxf(mx, p[v]);
      float other = mx;
      swap32(mx, other);
      mx = fmaxf(mx, other);
      other = mx;
      swap16(mx, other);
      mx = fmaxf(mx, other);
      const float mnew = fmaxf(m, mx);
      const float mref = mnew == -INFINITY ? 0.f : mnew * a.scale_log2;
      if (__any(mnew > m)) {
        const float c = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m * a.scale_log2 - mref);
        l *= c;
        lh *= c;
#pragma unroll
        for (int d = 0; d < ND; ++d) o[d] *= c;
      }
      m = mnew;
#pragma unroll
      for (int v = 0; v < 8; ++v) {
        p[v] = __builtin_amdgcn_exp2f(fmaf(p[v], a.scale_log2, -mref));
        l += p[v];
      }
      carry(lh, l);
      bf16x8 pt[NT];
      terms<NT>(p, pt);
      wave_lds_sync();  // the values are in LDS
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        const uint2 v0 = lds_read_tr16(vtr + d * 32);
        const uint2 v1 = lds_read_tr16(vtr + 16 * L::VROW + d * 32);
        const bf16x8 av = as_bf16x8(u32x4{v0.x, v0.y, v1.x, v1.y});
#pragma unroll
        for (int n = 0; n < NT; ++n) o[d] = mfma16(av, pt[n], o[d]);
      }
      wave_lds_sync();  // every read of the tile is done before the next writes
    }
    if (NT == 3 && t < nt) {
      const bool first = t == wid + kStepCarry * kWaves;
      const float c = first ? 0.f : parked_scale();
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        f32x4 h = {0.f, 0.f, 0.f, 0.f};
        if (!first) h = park[d * AIO_WAVE] * c;
        carry(h, o[d]);
        park[d * AIO_WAVE] = h;
      }
      *park_m = m;
    }
  }
  if (NT == 3 && wid + kStepCarry * kWaves < nt) {
    const float c = parked_scale();
#pragma unroll
    for (int d = 0; d < ND; ++d) o[d] += park[d * AIO_WAVE] * c;
  }
  l += lh;
  l += __shfl_xor(l, 16, AIO_WAVE);
  l += __shfl_xor(l, 32, AIO_WAVE);
  if (l != l) m = l;  // (the maximum passes over a NaN, the states' join must not)

  // join the waves
  __syncthreads();
  float* om = (float*)smem;  // [wave][column][OROW]
  if (col < a.G) {
#pragma unroll
    for (int d = 0; d < ND; ++d)
      *(f32x4*)(om + (wid * kMaxGroup + col) * L::OROW + d * 16 + 4 * grp) = o[d];
    if (grp == 0) {
      wm[wid][col] = m * a.scale_log2;
      wl[wid][col] = l;
    }
  }
  __syncthreads();
  for (int e = tid; e < a.G * HD; e += kBlock) {
    const int g = e / HD, d = e % HD;
    float M = wm[0][g];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, wm[w][g]);
    float ls = 0.f, os = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float x = wm[w][g];
      const float c = x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x - M);
      ls += c * wl[w][g];
      os += c * om[(w * kMaxGroup + g) * L::OROW + d];
    }
    const int64_t rh = (int64_t)seq * a.H + h0 + g;
    if (a.S == 1) {
      const bool none = ls == 0.f;  // no visible key
      store_out(a, NT == 3, (int64_t)seq * a.ldo + (int64_t)(h0 + g) * HD + d, none ? 0.f : os / ls);
      if (d == 0 && a.lse) a.lse[rh] = none ? -INFINITY : M * kLn2 + logf(ls);
    } else {
      const int64_t at = (int64_t)split * a.n_rows * a.H + rh;
      a.part_o[at * HD + d] = os;
      if (d == 0) {
        a.part_ml[at * 2] = ls != ls ? ls : M;
        a.part_ml[at * 2 + 1] = ls;
      }
    }
  }
}

// ------------------------------------------------------- the rows of prompts

// A sequence's rows and the G heads of a kv head form one list of q G packed
// rows (row-major: packed row r G + g is row r of head h0 + g), cut into tiles of
// 32 W; workgroup (tile, kv head, split) of W waves.  Each wave owns 32 packed rows (the
// columns of 32-wide tiles) and all of them share the key and value tiles in LDS, kKeys keys
// at a time, the next ones in flight in registers.  What bounds it is the matrix units
// at the clock that the card's power leaves them (about 2.0 GHz, 49 % busy; LDS takes
// the second place): 8192 rows of 32 heads of 128, bf16: 559 us, 984 TFLOP/s, where a
// plain matrix product reaches 1177.
constexpr int kKeys = 64;

// Two buffers of a key and of a value tile: while one is multiplied, the next is
// written.  The row pitches put the rows that one LDS access takes (16 of the keys,
// 4 of the values) into distinct banks.
template <int HD>
struct RowsLds {
  static constexpr int KROW = HD * 2 + 16, VROW = HD * 2 + 64;  // bytes
  static constexpr int KBYTES = kKeys * KROW, VBYTES = kKeys * VROW;
  static constexpr int TILES = 2 * (KBYTES + VBYTES);
  // the upper parts of a wave's output tile, and the references that they have
  static constexpr int HBYTES = HD * 32 * 4 + AIO_WAVE * 4;
  static constexpr int BYTES(int NT, int W) { return TILES + (NT == 3 ? W * HBYTES : 0); }
};

// First key of sequence i, how many of its keys are there, and how many it has by the
// caller's word (its rows are the last of those).
template <bool PAGED>
AIO_DEV void seq_keys(const AttnArgs& a, int i, int& key0, int& len, int& full) {
  if constexpr (PAGED) {
    key0 = 0;
    len = paged_len(a.kv, i, a.max_len);
    full = min(max(a.kv.lens[i], 0), 1 << 30);
  } else {
    key0 = min(max(a.kv.cu_k[i], 0), a.kv.limit);
    full = min(max(min(max(a.kv.cu_k[i + 1], 0), a.kv.limit) - key0, 0), 1 << 30);
    len = min(full, a.max_len);
  }
}

// Workgroups start in index order, and a causal tile's work grows with its last
// position: the longest first.  Tile `t` of the launch in that order, for 2 to 64
// sequences: a tile's level is its number in the sequence plus the rows in tiles
// that the sequence has had before; the tiles of the highest level come first (eight
// packed prompts of 540 to 2048 rows, sequence after sequence: 139 us, so 120).  With
// more sequences they come one after the other, each from its end: sequence i's from
// place first(i) G / ROWS + min(i, first(i)) on, which leaves room for its last, partly filled
// tile, takes none for sequences without rows, and is searched for 64 places at a time.
// seq and tile receive its place; false where there is none.
template <int ROWS, bool PAGED>
AIO_DEV bool find_tile(const AttnArgs& a, int t, int& seq, int& tile) {
  const int lane = threadIdx.x & (AIO_WAVE - 1);
  auto tiles_of = [&](int rows) { return (int)(((int64_t)rows * a.G + ROWS - 1) / ROWS); };
  if (a.n_seqs == 1 || a.n_seqs > AIO_WAVE) {
    auto place = [&](int i) {
      const int first = min(max(a.cu_q[i], 0), a.n_rows);
      return (int)((int64_t)first * a.G / ROWS) + min(i, first);
    };
    int lo = 0, hi = a.n_seqs;  // the last sequence whose place is at most t is in [lo, hi)
    while (hi - lo > 1) {
      const int step = (hi - lo + AIO_WAVE - 1) / AIO_WAVE;
      const int64_t p = lo + (int64_t)lane * step;
      const int c = __popcll(__ballot(p < hi && place((int)min(p, (int64_t)hi - 1)) <= t));
      if (c == 0) return false;
      lo += (c - 1) * step;
      hi = min(hi, lo + step);
    }
    int first, count;
    seq_rows(a.cu_q, a.n_rows, lo, first, count);
    const int at = t - place(lo), n = tiles_of(count);
    if (at < 0 || at >= n) return false;
    seq = lo;
    tile = n - 1 - at;
    return true;
  }
  int n = 0, first, count = 0, key0, len = 0, full;
  if (lane < a.n_seqs) {
    seq_rows(a.cu_q, a.n_rows, lane, first, count);
    n = tiles_of(count);
  }
  if (n > 0) seq_keys<PAGED>(a, lane, key0, len, full);
  const int64_t before = (int64_t)max(len - count, 0) * a.G / ROWS;
  const int lo = (int)min(before, (int64_t)1 << 22), hi = lo + n;
  // tiles of at least level v (below 2^24 of them: exact)
  auto from = [&](int v) {
    return (int)__builtin_amdgcn_readfirstlane((int)wave_sum((float)max(hi - max(v, lo), 0)));
  };
  if (from(0) <= t) return false;
  int at = 0, past = (int)wave_max((float)(n > 0 ? hi : 0));  // from(at) > t >= from(past)
  past = __builtin_amdgcn_readfirstlane(past);
  while (past - at > 1) {
    const int mid = (at + past) / 2;
    if (from(mid) > t) at = mid;
    else past = mid;
  }
  const int r = t - from(at + 1);  // the r-th of the sequences with a tile of this level
  const uint64_t has = __ballot(lo <= at && at < hi);
  const int before_me = __popcll(has & ((1ull << lane) - 1));
  const uint64_t me = __ballot((has >> lane & 1) && before_me == r);
  if (!me) return false;  // (boundaries that overlap)
  seq = __ffsll((unsigned long long)me) - 1;
  tile = at - __builtin_amdgcn_readlane(lo, seq);
  return true;
}

AIO_DEV bool not_finite(u32x4 w) {  // of eight bf16
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    bad |= (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
  return bad;
}

// A row's weights refer to a maximum that is raised only when it would be passed by
// 2^kSlack: weights then reach 2^kSlack instead of 1, which costs no precision (they
// are floating point), and the outputs are rarely rescaled (in the first few dozen
// blocks nearly every block raises the maximum of one of a wave's 32 rows).
constexpr float kSlack = 8.f;

// Products by which LDS reads run ahead of their use.
constexpr int kAhead = 4;

template <int HD, int NT, bool PAGED, int W>
__global__ __launch_bounds__(W * AIO_WAVE, NT == 1 ? 2 : 1) void k_attn_rows(AttnArgs a) {
  using L = RowsLds<HD>;
  constexpr int kThreads = W * AIO_WAVE, kRows = W * 32;
  extern __shared__ __align__(16) char smem[];
  __shared__ uint8_t seen[kKeys];
  constexpr int NC = HD / 16;                      // k chunks of a score product
  constexpr int NHB = HD / 32;                     // output tiles
  constexpr int TPR = HD / 8;                      // threads of a row
  constexpr int RPP = kThreads / TPR;                // rows per pass
  constexpr int RPW = AIO_WAVE / TPR;              // ... of a wave: 4 or 8, all in one page
  constexpr int NP = kKeys / RPP;                  // passes of a tile
  const int tid = threadIdx.x, lane = tid & (AIO_WAVE - 1);
  const int wid = __builtin_amdgcn_readfirstlane(tid / AIO_WAVE);
  const int rl = lane & 31, kh = lane >> 5;
  const int split = udiv(blockIdx.x, a.by_s);  // by_s: workgroups per split
  const int lin = blockIdx.x - split * a.by_s.d;
  const int tg = udiv(lin, a.by_hkv), kvh = lin - tg * a.kv.Hkv;
  int seq, tile;
  if (!find_tile<kRows, PAGED>(a, tg, seq, tile)) return;
  int first, count, key0, len, full;
  seq_rows(a.cu_q, a.n_rows, seq, first, count);
  seq_keys<PAGED>(a, seq, key0, len, full);
  const int packed = count * a.G, p0 = tile * kRows;
  const int h0 = kvh * a.G;
  // this lane's query
  const int pr = p0 + wid * 32 + rl;
  const bool live = pr < packed;
  const int row = udiv(min(pr, packed - 1), a.by_g), g = min(pr, packed - 1) - row * a.G;
  auto sees = [&](int r) { return min(full - count + r, len - 1); };  // row r's last key
  const int lim = sees(row);
  // the last key that any row of the wave, of the workgroup sees, and the last
  // that all rows of the workgroup see
  const int wave_lim = sees(udiv(min(p0 + wid * 32 + 31, packed - 1), a.by_g));
  const int wg_lim = sees(udiv(min(p0 + kRows, packed) - 1, a.by_g));
  const int all_lim = sees(udiv(p0, a.by_g));
  const int nkt = wg_lim < 0 ? 0 : wg_lim / kKeys + 1;
  // this split's key tiles
  const int each = nkt / a.S, rest = nkt - each * a.S;
  const int t0 = split * each + min(split, rest), t1 = t0 + each + (split < rest ? 1 : 0);

  bf16x8 q[NC][NT];
#pragma unroll
  for (int c = 0; c < NC; ++c)
    load_query<NT>(a, first + row, h0 + g, HD, c * 16 + 8 * kh, live, q[c]);

  // staging: pass p of this wave is rows p RPP + wid RPW .. + RPW - 1, of a lane 16
  // bytes of one
  const int wr = wid * RPW, lr = lane / TPR, sd = lane % TPR * 8;
  const uint16_t* kb = a.kv.k + kvh * a.kv.head_stride;
  const uint16_t* vb = a.kv.v + kvh * a.kv.head_stride;
  const int64_t lane_at = PAGED ? lr * HD + sd : lr * a.kv.stride + sd;
  const int32_t* table = PAGED ? a.kv.table + (int64_t)seq * a.kv.tstride : nullptr;
  const int pmask = (1 << a.kv.shift) - 1;

  // Plain tiles t0 .. tp - 1: every row sees every key of them.  (One hole among them sends them
  // all through the loop below: 2048 rows of the 1B behind 1637 keys, bf16, 90 us without a hole,
  // 263 with one.)
  int tp = min(t1, max(t0, all_lim < 0 ? 0 : (all_lim + 1) / kKeys));
  if constexpr (PAGED) {
    // (not with holes among them)
    if (tp > t0) {
      bool hole = false;
      const int e1 = (tp * kKeys - 1) >> a.kv.shift;
      for (int e = (t0 * kKeys >> a.kv.shift) + tid; e <= e1; e += kThreads)
        hole |= (unsigned)table[e] >= (unsigned)a.kv.limit;
      if (__syncthreads_or(hole)) tp = t0;
    }
  }

  f32x16 o[NHB];
#pragma unroll
  for (int hb = 0; hb < NHB; ++hb)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[hb][i] = 0.f;
  float m = -INFINITY, l = 0.f, lh = 0.f;  // m: reference of the weights, in log2 units
  // The upper parts of o wait in LDS, with the reference of then.
  f32x4* park = (f32x4*)(smem + L::TILES + wid * L::HBYTES) + lane;
  float* park_m = (float*)(smem + L::TILES + wid * L::HBYTES + HD * 32 * 4) + lane;
  bool parked = false;
  auto parked_scale = [&] {
    const float mh = *park_m;
    return mh == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mh - m);
  };
  // (after every kRowsCarry of the tiles)
  auto carry_out = [&](int tiles) {
    if (NT != 3 || tiles % kRowsCarry) return;
    const float c = parked ? parked_scale() : 0.f;
#pragma unroll
    for (int i = 0; i < 4 * NHB; ++i) {
      f32x4 h = {0.f, 0.f, 0.f, 0.f}, low;
      if (parked) h = park[i * AIO_WAVE] * c;
#pragma unroll
      for (int e = 0; e < 4; ++e) low[e] = o[i / 4][4 * (i % 4) + e];
      carry(h, low);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i / 4][4 * (i % 4) + e] = low[e];
      park[i * AIO_WAVE] = h;
      __builtin_amdgcn_sched_barrier(0);  // (few at a time: registers)
    }
    *park_m = m;
    parked = true;
  };
  const int st_at = (wr + lr) * L::KROW + sd * 2, sv_at = (wr + lr) * L::VROW + sd * 2;
  const int k_at = rl * L::KROW + 16 * kh;
  const int v_at = (4 * kh + (lane & 15) / 4) * L::VROW +
                   ((lane >> 4 & 1) * 16 + (lane & 3) * 4) * 2;
  auto key_frag = [&](int buf, int i) {  // i: chunk of 16 dims, block of 32 keys
    return as_bf16x8(*(const u32x4*)(smem + buf * L::KBYTES + k_at + i % 2 * 32 * L::KROW +
                                     i / 2 * 32));
  };
  auto value_frag = [&](int buf, int i) {  // i: chunk of 16 keys, tile of 32 dims
    const char* v = smem + 2 * L::KBYTES + buf * L::VBYTES + v_at + i / NHB * 16 * L::VROW +
                    i % NHB * 64;
    const uint2 v0 = lds_read_tr16(v), v1 = lds_read_tr16(v + 8 * L::VROW);
    return as_bf16x8(u32x4{v0.x, v0.y, v1.x, v1.y});
  };
  // The reference of a tile whose largest score in this lane is mx.
  auto refer = [&](float mx) {
    float other = mx;
    swap32(mx, other);
    mx = fmaxf(mx, other) * a.scale_log2;
    const bool raise = mx > m + kSlack;  // (the first visible key: above -inf)
    if (__any(raise)) {
      const float mnew = raise ? mx : m;
      // (o holds nothing but what is not finite before the first visible key)
      const float c = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mnew);
      m = mnew;
      l *= c;
      lh *= c;
#pragma unroll
      for (int hb = 0; hb < NHB; ++hb)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[hb][i] *= c;
    }
    return m == -INFINITY ? 0.f : m;
  };

  if (tp > t0) {
    // Tile t into registers: no branches, tiles past the last read it again.  Its pages
    // (one of each pass's rows) are looked up well before.
    struct PageIds {
      int id[NP];
    };
    auto pages_of = [&](int t) {
      PageIds pg{};
      if constexpr (PAGED) {
#pragma unroll
        for (int p = 0; p < NP; ++p)
          pg.id[p] = table[(min(t, tp - 1) * kKeys + p * RPP + wr) >> a.kv.shift];
      }
      return pg;
    };
    auto load_tile = [&](u32x4 (&r)[NP], const uint16_t* from, int t, const PageIds& pg) {
      const int key = min(t, tp - 1) * kKeys + wr;
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        if constexpr (PAGED) {
          const int64_t at = pg.id[p] * a.kv.stride + (int64_t)((key + p * RPP) & pmask) * HD;
          r[p] = *(const u32x4*)(from + at + (uint32_t)lane_at);
        } else {
          r[p] = *(const u32x4*)(from + (int64_t)(key0 + key + p * RPP) * a.kv.stride + lane_at);
        }
      }
    };
    auto store_keys = [&](const u32x4 (&r)[NP], int buf) {
#pragma unroll
      for (int p = 0; p < NP; ++p)
        *(u32x4*)(smem + buf * L::KBYTES + st_at + p * RPP * L::KROW) = r[p];
    };
    auto store_values = [&](const u32x4 (&r)[NP], int buf) {
#pragma unroll
      for (int p = 0; p < NP; ++p)
        *(u32x4*)(smem + 2 * L::KBYTES + buf * L::VBYTES + sv_at + p * RPP * L::VROW) = r[p];
    };
    u32x4 kr[NP], vr[NP];
    PageIds pg2 = pages_of(t0 + 2), pg3 = pages_of(t0 + 3), pg4 = pages_of(t0 + 4);
    float mx;
    // One tile: its softmax while the next tile's scores (sn) are multiplied, then
    // its values while the next tile's maximum is taken.  Score v of block b is key 32 b +
    // 8 (v / 4) + 4 kh + v mod 4 of the tile.
    auto step = [&](int t, auto buf_c, f32x16 (&s)[2], f32x16 (&sn)[2]) {
      constexpr int buf = decltype(buf_c)::value;
      // K of t + 1 and V of t are in their buffers; every wave is done with K of t and
      // V of t - 1, whose buffers take K of t + 2 and V of t + 1
      __syncthreads();
      store_keys(kr, buf);
      store_values(vr, buf ^ 1);
      const float mref = refer(mx);
      // Matrix instructions with a few vector instructions behind each: those then
      // cost next to nothing (8 of these MFMAs with 16 exponentials among them
      // take as long as without, with 48 multiply-adds 14 % longer; one kind after the
      // other, two waves per SIMD hide about half).
      bf16x8 pt[4][NT];
      bf16x8 ak[kAhead + 1];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) ak[i] = key_frag(buf ^ 1, i);
#pragma unroll
      for (int i = 0; i < 2 * NC; ++i) {
        if (i + kAhead < 2 * NC)
          ak[(i + kAhead) % (kAhead + 1)] = key_frag(buf ^ 1, i + kAhead);
        if (i < 2) {
#pragma unroll
          for (int e = 0; e < 16; ++e) sn[i][e] = 0.f;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) sn[i % 2] = mfma32(ak[i % (kAhead + 1)], q[i / 2][n], sn[i % 2]);
        constexpr int E = 16 / NC;  // scores of this step
#pragma unroll
        for (int e = i * E; e < (i + 1) * E; ++e) {
          const float x = __builtin_amdgcn_exp2f(fmaf(s[e / 16][e % 16], a.scale_log2, -mref));
          s[e / 16][e % 16] = x;
          l += x;
        }
        if ((i + 1) * E % 8 == 0) {
          const int c = ((i + 1) * E - 1) / 8;
          float p[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) p[e] = s[c / 2][8 * (c & 1) + e];
          terms<NT>(p, pt[c]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      load_tile(kr, kb, t + 3, pg3);
      load_tile(vr, vb, t + 2, pg2);
      pg2 = pg3;
      pg3 = pg4;
      pg4 = pages_of(t + 5);
      bf16x8 av[kAhead + 1];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) av[i] = value_frag(buf, i);
      mx = sn[0][0];
#pragma unroll
      for (int i = 0; i < 4 * NHB; ++i) {
        if (i + kAhead < 4 * NHB)
          av[(i + kAhead) % (kAhead + 1)] = value_frag(buf, i + kAhead);
#pragma unroll
        for (int n = 0; n < NT; ++n) o[i % NHB] = mfma32(av[i % (kAhead + 1)], pt[i / NHB][n], o[i % NHB]);
        constexpr int E = 32 / (4 * NHB);  // scores of the next tile to take the maximum of
#pragma unroll
        for (int e = i * E; e < (i + 1) * E; ++e) mx = fmaxf(mx, sn[e / 16][e % 16]);
        __builtin_amdgcn_sched_barrier(0);
      }
      carry(lh, l);
    };
    // (buffers by t - t0's parity: K of t0 in 0, of t0 + 1 in 1, V of t0 in 0)
    f32x16 sa[2], sb[2];
    {
      const PageIds pg0 = pages_of(t0), pg1 = pages_of(t0 + 1);
      load_tile(kr, kb, t0, pg0);
      load_tile(vr, vb, t0, pg0);
      store_keys(kr, 0);
      store_values(vr, 0);
      load_tile(kr, kb, t0 + 1, pg1);
      store_keys(kr, 1);
      load_tile(kr, kb, t0 + 2, pg2);
      load_tile(vr, vb, t0 + 1, pg1);
    }
    __syncthreads();
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sa[b][i] = 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const bf16x8 ak = key_frag(0, 2 * c + b);
#pragma unroll
        for (int n = 0; n < NT; ++n) sa[b] = mfma32(ak, q[c][n], sa[b]);
      }
    }
    mx = sa[0][0];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int v = 0; v < 16; ++v) mx = fmaxf(mx, sa[b][v]);
    int t = t0;
    for (; t + 1 < tp; t += 2) {
      step(t, std::integral_constant<int, 0>{}, sa, sb);
      step(t + 1, std::integral_constant<int, 1>{}, sb, sa);
      carry_out(t + 2 - t0);
    }
    if (t < tp) step(t, std::integral_constant<int, 0>{}, sa, sb);
  }

  // The other tiles, one after the other: at the causal edge or the keys' end, or with
  // holes.
  for (int t = tp; t < t1; ++t) {
    const int j0 = t * kKeys;
    u32x4 kr[NP], vr[NP];
    uint32_t ok = 0;  // bit p: the row of pass p is there
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int key = j0 + p * RPP + wr;
      bool there = key + lr < len;
      int64_t at = (int64_t)(key0 + key) * a.kv.stride;
      if constexpr (PAGED) {
        const int page = key < len ? table[key >> a.kv.shift] : -1;
        there &= (unsigned)page < (unsigned)a.kv.limit;
        at = page * a.kv.stride + (int64_t)(key & pmask) * HD;
      }
      kr[p] = vr[p] = u32x4{0, 0, 0, 0};
      if (there) {
        kr[p] = *(const u32x4*)(kb + at + lane_at);
        vr[p] = *(const u32x4*)(vb + at + lane_at);
        ok |= 1u << p;
      }
    }
    __syncthreads();  // every wave is done with the tile before
    bool odd = false;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      *(u32x4*)(smem + st_at + p * RPP * L::KROW) = kr[p];
      *(u32x4*)(smem + 2 * L::KBYTES + sv_at + p * RPP * L::VROW) = vr[p];
      if (sd == 0) seen[p * RPP + wr + lr] = ok >> p & 1;
      odd |= not_finite(vr[p]);
    }
    if (__syncthreads_or(odd)) {
      // Values that are not finite must not meet a weight of 0 in a product: they go
      // straight to the rows that see them, and out of the tile.
      char* v = smem + 2 * L::KBYTES;
#pragma unroll 1
      for (int kk = 0; kk < kKeys; ++kk) {
        if (j0 + kk > lim || !seen[kk]) continue;
#pragma unroll
        for (int hb = 0; hb < NHB; ++hb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int d = hb * 32 + 8 * (i / 4) + 4 * kh + i % 4;
            const uint16_t x = *(const uint16_t*)(v + kk * L::VROW + d * 2);
            if ((x & 0x7f80u) == 0x7f80u) o[hb][i] += bf16_to_f32(x);
          }
      }
      __syncthreads();
      for (int e = tid; e < kKeys * HD; e += kThreads) {
        uint16_t* x = (uint16_t*)(v + e / HD * L::VROW) + e % HD;
        if ((*x & 0x7f80u) == 0x7f80u) *x = 0;
      }
      __syncthreads();
    }
    if (j0 > wave_lim) continue;
    f32x16 s[2];
    float mx = -INFINITY;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const bf16x8 ak = key_frag(0, 2 * c + b);
#pragma unroll
        for (int n = 0; n < NT; ++n) s[b] = mfma32(ak, q[c][n], s[b]);
      }
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int kk = 32 * b + 8 * (v / 4) + 4 * kh + v % 4;
        if (j0 + kk > lim || !seen[kk]) s[b][v] = -INFINITY;
        mx = fmaxf(mx, s[b][v]);
      }
    }
    const float mref = refer(mx);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(fmaf(s[c / 2][8 * (c & 1) + e], a.scale_log2, -mref));
        l += p[e];
      }
      bf16x8 pt[NT];
      terms<NT>(p, pt);
#pragma unroll
      for (int hb = 0; hb < NHB; ++hb) {
        const bf16x8 av = value_frag(0, c * NHB + hb);
#pragma unroll
        for (int n = 0; n < NT; ++n) o[hb] = mfma32(av, pt[n], o[hb]);
      }
    }
    carry(lh, l);
    carry_out(t + 1 - t0);
  }
  if (!live) return;
  if (NT == 3 && parked) {
    const float c = parked_scale();
#pragma unroll
    for (int i = 0; i < 4 * NHB; ++i) {
      const f32x4 h = park[i * AIO_WAVE] * c;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i / 4][4 * (i % 4) + e] += h[e];
    }
  }
  l += lh;
  l += __shfl_xor(l, 32, AIO_WAVE);
  if (l != l) m = l;  // (the maximum passes over a NaN, the states' join must not)
  const int64_t rh = (int64_t)(first + row) * a.H + h0 + g;
  if (a.S > 1) {
    const int64_t at = (int64_t)split * a.n_rows * a.H + rh;
    if (kh == 0) {
      a.part_ml[at * 2] = m;
      a.part_ml[at * 2 + 1] = l;
    }
    if (m == -INFINITY) return;
#pragma unroll
    for (int hb = 0; hb < NHB; ++hb)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(f32x4*)(a.part_o + at * HD + hb * 32 + 8 * i + 4 * kh) =
            f32x4{o[hb][4 * i], o[hb][4 * i + 1], o[hb][4 * i + 2], o[hb][4 * i + 3]};
    return;
  }
  const bool none = l == 0.f;  // no visible key
  const float inv = none ? 0.f : 1.f / l;
  if (kh == 0 && a.lse) a.lse[rh] = none ? -INFINITY : m * kLn2 + logf(l);
  const int64_t to = (int64_t)(first + row) * a.ldo + (int64_t)(h0 + g) * HD + 4 * kh;
#pragma unroll
  for (int hb = 0; hb < NHB; ++hb)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 v = {o[hb][4 * i] * inv, o[hb][4 * i + 1] * inv, o[hb][4 * i + 2] * inv,
                       o[hb][4 * i + 3] * inv};
      const int64_t at = to + hb * 32 + 8 * i;
      if constexpr (NT == 3) {
        *(f32x4*)((float*)a.out + at) = v;
      } else {
        const uint2 w = {f32_to_bf16(v[0]) | (uint32_t)f32_to_bf16(v[1]) << 16,
                         f32_to_bf16(v[2]) | (uint32_t)f32_to_bf16(v[3]) << 16};
        *(uint2*)((uint16_t*)a.out + at) = w;
      }
    }
}

// Joins the splits of a row and head: one wave each.  4 to 5 us behind its attention
// (launch and two dependent reads), whatever the sizes here.
template <int HD, bool F32>
__global__ __launch_bounds__(kBlock) void k_attn_join(AttnArgs a) {
  const int lane = threadIdx.x & (AIO_WAVE - 1);
  const int64_t rh = (int64_t)blockIdx.x * kWaves + threadIdx.x / AIO_WAVE;
  const int64_t all = (int64_t)a.n_rows * a.H;
  if (rh >= all) return;
  const int row = (int)(rh / a.H), head = (int)(rh - (int64_t)row * a.H);
  // rows of no sequence are left alone
  if (a.cu_q && (row < a.cu_q[0] || row >= a.cu_q[a.n_seqs])) return;
  float M = -INFINITY;
  for (int s = lane; s < a.S; s += AIO_WAVE) M = fmaxf(M, a.part_ml[(s * all + rh) * 2]);
  M = wave_max(M);
  constexpr int PER = HD / AIO_WAVE;
  float os[PER] = {}, oh[PER] = {}, ls = 0.f;
  // a split's weight in its lane, then the splits with keys (the others' values were
  // not written), their loads independent of one another
  for (int s0 = 0; s0 < a.S; s0 += AIO_WAVE) {
    float c = 0.f;
    bool keys = false;
    if (s0 + lane < a.S) {
      const float* ml = a.part_ml + ((s0 + lane) * all + rh) * 2;
      const float x = ml[0];
      keys = x != -INFINITY;
      if (keys) {
        c = __builtin_amdgcn_exp2f(x - M);
        ls += c * ml[1];
      }
    }
    // (those whose weight underflows among them: 0 x inf shows that they saw an infinity)
    const uint64_t some = __ballot(keys);
    if (!some) continue;
    const int n = min(a.S - s0, AIO_WAVE), valid = __ffsll((unsigned long long)some) - 1;
    constexpr int B = 8;
    for (int s1 = 0; s1 < n; s1 += B) {
      float v[B][PER];
#pragma unroll
      for (int b = 0; b < B; ++b) {
        const int s = s1 + b < n && some >> (s1 + b) & 1 ? s1 + b : valid;
        const float* o = a.part_o + ((s0 + s) * all + rh) * HD + lane;
#pragma unroll
        for (int i = 0; i < PER; ++i) v[b][i] = o[i * AIO_WAVE];
      }
#pragma unroll
      for (int b = 0; b < B; ++b) {
        if (s1 + b >= n || !(some >> (s1 + b) & 1)) continue;
        const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(c), s1 + b));
#pragma unroll
        for (int i = 0; i < PER; ++i) os[i] += w * v[b][i];
      }
#pragma unroll
      for (int i = 0; i < PER; ++i) carry(oh[i], os[i]);
    }
  }
  ls = wave_sum(ls);
  const bool none = ls == 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i)
    store_out(a, F32, (int64_t)row * a.ldo + (int64_t)head * HD + i * AIO_WAVE + lane,
              none ? 0.f : (oh[i] + os[i]) / ls);
  if (lane == 0 && a.lse) a.lse[rh] = none ? -INFINITY : M * kLn2 + logf(ls);
}

template <int HD, int NT, bool PAGED, int W>
hipError_t launch_rows_w(const AttnArgs& a, const AttnPlan& p, hipStream_t stream) {
  constexpr int lds = RowsLds<HD>::BYTES(NT, W);
  const auto fn = k_attn_rows<HD, NT, PAGED, W>;
  const hipError_t e =
      hipFuncSetAttribute((const void*)fn, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(fn, dim3((unsigned)p.groups), dim3(W * AIO_WAVE), lds, stream, a);
  return hipGetLastError();
}

template <int HD, int NT, bool PAGED>
hipError_t launch_rows(const AttnArgs& a, const AttnPlan& p, hipStream_t stream) {
  if constexpr (NT == 1) {
    if (p.waves == 8) return launch_rows_w<HD, NT, PAGED, 8>(a, p, stream);
  }
  return launch_rows_w<HD, NT, PAGED, 4>(a, p, stream);
}

template <int HD, int NT>
hipError_t launch(const AttnArgs& a, const AttnPlan& p, hipStream_t stream) {
  hipError_t e;
  if (!p.rows) {
    constexpr int lds = StepLds<HD>::BYTES(NT);
    const auto fn = p.stream ? k_attn_step<HD, NT, true> : k_attn_step<HD, NT, false>;
    e = hipFuncSetAttribute((const void*)fn, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(fn, dim3((unsigned)p.groups), dim3(kBlock), lds, stream, a);
    e = hipGetLastError();
  } else {
    e = a.kv.table ? launch_rows<HD, NT, true>(a, p, stream) : launch_rows<HD, NT, false>(a, p, stream);
  }
  if (e != hipSuccess || a.S == 1) return e;
  const int64_t rh = (int64_t)a.n_rows * a.H;
  hipLaunchKernelGGL((k_attn_join<HD, NT == 3>), dim3((unsigned)((rh + kWaves - 1) / kWaves)),
                     dim3(kBlock), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

// Workgroups up to which the keys are split.
constexpr int64_t kStepGroups = 4 * kCUs, kRowsGroups = 2 * kCUs;

int aio_attn_plan(const aio_seqs& s, int H, int Hkv, int hd, int dtype, AttnPlan* p) {
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
  p->stream = !p->rows && (int64_t)s.n_seqs * s.max_len * Hkv * hd * 4 > (int64_t)64 << 20;
  if (p->splits > 1) p->ws = (size_t)p->splits * s.n_rows * H * (hd + 2) * 4;
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

size_t aio_attn_workspace_bound(int H, int Hkv, int hd) {
  // step: splits n Hkv <= kStepGroups, so splits n H <= kStepGroups G; rows: splits tiles
  // Hkv <= kRowsGroups and n_rows G <= 256 tiles, so splits n_rows H <= 256 kRowsGroups
  const size_t rh = std::max<size_t>((size_t)kStepGroups * (H / Hkv), (size_t)kRowsGroups * 256);
  return rh * (hd + 2) * 4;
}

hipError_t aio_launch_attention(const AttnArgs& a, const AttnPlan& p, int hd, int dtype,
                                hipStream_t stream) {
  if (hd == 128)
    return dtype == AIO_F32 ? launch<128, 3>(a, p, stream) : launch<128, 1>(a, p, stream);
  return dtype == AIO_F32 ? launch<64, 3>(a, p, stream) : launch<64, 1>(a, p, stream);
}
