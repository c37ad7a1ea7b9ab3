// Log probabilities, entropy and top alternatives of logit rows.
//
// With m = max x, z = sum e^(x - m), w = sum e^(x - m) (x - m):
//   log sum e^x = m + log z,  entropy = log z - w / z.
// One pass over the row; a new maximum m' rescales z and w of the values seen:
//   z' = c z,  w' = c (w + z (m - m')),  c = e^(m - m').
// z and w are 64-bit sums of 32-bit terms: a confident row has z = 1 + 1e-6,
// whose logarithm is what is asked for.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "paged.h"

namespace {

constexpr int kBlock = 256;
constexpr int kPer = 32;                  // values per thread and chunk
constexpr int kPerFew = 8;                // ... where a slice is short
constexpr int kMaxSlices = 64;
// A chunk's candidates: the values from the top-th largest of the threads'
// maxima on.  Only the `top` threads of the largest maxima hold any, at most
// kPer each; the best `top` of the chunks before join them.
constexpr int kCand = AIO_MAX_TOP * kPer + AIO_MAX_TOP;

// A value and its index as one number: larger value first, then the lower
// index; NaN above everything, -0 equal to +0.  0 is no value.
AIO_DEV uint64_t order_key(float v, int i) {
  uint32_t u = __float_as_uint(v + 0.f);
  u = (u & 0x80000000u) ? ~u : u | 0x80000000u;
  if (v != v) u = 0xffffffffu;
  return (uint64_t)u << 32 | (uint32_t)~i;
}
AIO_DEV int key_index(uint64_t k) { return (int)~(uint32_t)k; }
AIO_DEV float key_value(uint64_t k) {
  const uint32_t u = (uint32_t)(k >> 32);
  if (u == 0xffffffffu) return __uint_as_float(0x7fc00000u);
  return __uint_as_float((u & 0x80000000u) ? u & 0x7fffffffu : ~u);
}

constexpr float kLog2e = 1.44269504088896340736f;

struct Stats {
  float m;
  double z, w;
};

// e^(a - b), 1 for equal ones (infinities among them)
AIO_DEV double exp_diff(float a, float b) {
  return a == b ? 1.0 : (double)expf(a - b);
}

AIO_DEV Stats join(const Stats& a, const Stats& b) {
  const float m = fmaxf(a.m, b.m);
  if (m == -INFINITY) return Stats{m, a.z + b.z, a.w + b.w};
  const double ca = exp_diff(a.m, m), cb = exp_diff(b.m, m);
  // (an empty side: c = 0 and z = 0, but its difference is infinite)
  const double da = a.m == -INFINITY ? 0.0 : (double)a.m - m;
  const double db = b.m == -INFINITY ? 0.0 : (double)b.m - m;
  return Stats{m, ca * a.z + cb * b.z, ca * (a.w + a.z * da) + cb * (b.w + b.z * db)};
}

AIO_DEV Stats wave_join(Stats s) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    Stats o;
    o.m = __shfl_xor(s.m, off, AIO_WAVE);
    o.z = __shfl_xor(s.z, off, AIO_WAVE);
    o.w = __shfl_xor(s.w, off, AIO_WAVE);
    s = join(s, o);
  }
  return s;
}

// The `top` largest of n candidates in descending order into best[0 .. top):
// a candidate's place is the number of larger ones.
AIO_DEV void rank_candidates(const uint64_t* cand, int n, int top, uint64_t* best) {
  for (int i = threadIdx.x; i < n; i += kBlock) {
    const uint64_t k = cand[i];
    int r = 0, j = 0;
    for (; j + 8 <= n; j += 8) {  // (reads in flight together)
#pragma unroll
      for (int u = 0; u < 8; ++u) r += cand[j + u] > k;
    }
    for (; j < n; ++j) r += cand[j] > k;
    if (r < top) best[r] = k;
  }
}

AIO_DEV float load1(const float* x, int64_t i) { return x[i]; }
AIO_DEV float load1(const uint16_t* x, int64_t i) { return bf16_to_f32(x[i]); }

template <class T>
AIO_DEV void finish_row(const LogprobArgs& a, int row, const Stats& s, const uint64_t* best) {
  // a row with nothing above -inf has no distribution, nor one with +inf
  const double nan = (double)__uint_as_float(0x7fc00000u);
  const bool none = s.m == -INFINITY || s.m == INFINITY;
  const double logz = none ? nan : log(s.z);
  if (threadIdx.x == 0 && a.entropy) a.entropy[row] = (float)(logz - s.w / s.z);
  if (threadIdx.x == 0 && a.logprob) {
    const int t = a.target[row];
    a.logprob[row] = (unsigned)t < (unsigned)a.n
                         ? (float)((double)load1((const T*)a.x + row * a.stride, t) - s.m - logz)
                         : (float)nan;
  }
  if ((int)threadIdx.x < a.top) {
    const uint64_t k = best[threadIdx.x];
    a.ids[(int64_t)row * a.top + threadIdx.x] = key_index(k);
    a.top_lp[(int64_t)row * a.top + threadIdx.x] = (float)((double)key_value(k) - s.m - logz);
  }
}

// kPer values per thread from c0 on, in groups of 16 bytes where rows allow
// it, and their indices; behind `hi`, -inf.
template <class T, int PER, bool VEC>
struct Chunk {
  static constexpr int V = VEC ? 16 / (int)sizeof(T) : 1;  // values per load
  static constexpr int N = kBlock * PER;
  float v[PER];
  AIO_DEV static int index(int c0, int i) {
    return c0 + (i / V * kBlock + (int)threadIdx.x) * V + i % V;
  }
  AIO_DEV void load(const T* x, int c0, int hi) {
    if (VEC && c0 + N <= hi) {
#pragma unroll
      for (int i = 0; i < PER; i += V) {
        // (long stretches per workgroup come in numbers: they pass the caches by)
        const u32x4* at = (const u32x4*)(x + index(c0, i));
        const u32x4 w = PER == kPer ? __builtin_nontemporal_load(at) : *at;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
          for (int j = 0; j < V; ++j) v[i + j] = __uint_as_float(w[j]);
        } else {
#pragma unroll
          for (int j = 0; j < V; ++j) v[i + j] = j & 1 ? bf16_hi(w[j / 2]) : bf16_lo(w[j / 2]);
        }
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = index(c0, i);
      v[i] = e < hi ? load1(x, e) : -INFINITY;
    }
  }
};

// Workgroup (slice, row): the slice's statistics and its best candidates; with
// one slice per row, the row's results.
//
// A chunk's candidates are the values from a cut on: for the first chunk the
// `top`-th largest of the maxima of the 64 groups of four threads, later the
// smallest of the best so far (its equals come later and lose).  That leaves
// about as many as are asked for.  Where it does not (equal values, rising ones, NaN),
// the chunk's cut is made exactly: the top-th largest (value, index) among the
// threads' own, which lets at most PER top through.
//
// 2048 rows of 32000 fp32 logits, top 8: 61 us, 4.3 TB/s (a large copy runs at 5.2, and
// without alternatives the same rows take 52).  What bounds it: about 13 vector
// instructions per value, and the barriers of the first chunk's cut, which the other
// workgroups of a CU hide as far as registers allow (64 of them: the exact cut reads
// its values again; kept in registers, 128 and 78 us).  One row of 32000, top 5: 16
// workgroups, 6.9 us and 4.5 for the join, launches and dependent steps.  Rows that do not
// start at 16 bytes are read element by element, with 36 bytes of scratch per lane:
// 2048 of 50257, top 8, 94 us in fp32 (the bytes take 80) and 219 in bf16 (40).
template <class T, int PER, bool VEC>
__global__ __launch_bounds__(kBlock, 4) void k_logprobs(LogprobArgs a) {
  using C = Chunk<T, PER, VEC>;
  __shared__ uint64_t cand[kCand];
  __shared__ uint64_t maxima[kBlock];
  __shared__ uint64_t best[AIO_MAX_TOP];
  __shared__ uint32_t group_max[2][kBlock / 4];
  __shared__ uint64_t cut_s;
  __shared__ int n_cand;
  __shared__ Stats ws[kBlock / AIO_WAVE];
  const int tid = threadIdx.x, lane = tid & (AIO_WAVE - 1);
  const int row = blockIdx.y, slice = blockIdx.x;
  const T* x = (const T*)a.x + row * a.stride;
  const int lo = slice * a.per, hi = min(a.n, lo + a.per);
  Stats st{-INFINITY, 0.0, 0.0};
  if (tid < AIO_MAX_TOP) best[tid] = 0;
  if (tid == 0) n_cand = 0;
  int parity = 0;
  for (int c0 = lo; c0 < hi; c0 += C::N, parity ^= 1) {
    C c;
    c.load(x, c0, hi);
    float m = c.v[0];
#pragma unroll
    for (int i = 1; i < PER; ++i) m = fmaxf(m, c.v[i]);
    Stats s{m, 0.0, 0.0};
    if (m != -INFINITY) {
      // z in 64 bits, so that a 1 does not swallow the rest (w's terms are 0 there);
      // e^-150 is 0: the clamp only keeps 0 x -inf out of w
      float w = 0.f;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const float d = c.v[i] - m;
        const float e = __builtin_amdgcn_exp2f(d * kLog2e);
        s.z += (double)e;
        w = fmaf(e, fmaxf(d, -150.f), w);
      }
      s.w = (double)w;
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (c.v[i] != c.v[i]) s.z = (double)c.v[i];
    }
    const bool nan = s.z != s.z;  // (or +inf - inf: its keys are sorted exactly as well)
    st = join(st, s);
    if (a.top == 0) continue;
    // the largest of the thread as a sortable number, 0 for none
    const uint32_t mine = nan ? 0xffffffffu
                              : (C::index(c0, 0) < hi ? (uint32_t)(order_key(m, 0) >> 32) : 0u);
    uint32_t g = max(mine, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)mine, 0xB1, 0xF, 0xF, false));
    g = max(g, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)g, 0x4E, 0xF, 0xF, false));
    if ((tid & 3) == 0) group_max[parity][tid / 4] = g;
    __syncthreads();  // (also: the chunk before is ranked, n_cand is 0)
    g = group_max[parity][lane];
    uint32_t cut;
    const uint64_t kth = best[a.top - 1];
    if (kth) {
      cut = (uint32_t)(kth >> 32);
      if (cut != 0xffffffffu) ++cut;
      if (!__any(g >= cut)) continue;
    } else {
      // (the last 6 bits give way to the group's number, so that no two are equal)
      const uint32_t mark = (g & ~63u) | lane;
      int r = 0;
#pragma unroll 8
      for (int j = 0; j < kBlock / 4; ++j)
        r += ((group_max[parity][j] & ~63u) | (uint32_t)j) > mark;
      const uint64_t at = __ballot(r == a.top - 1);
      cut = __builtin_amdgcn_readlane(g, __ffsll((unsigned long long)at) - 1) & ~63u;
      if (cut == 0) cut = 1;
    }
    bool exact = __any(g == 0xffffffffu);
    if (!exact) {
      if (mine >= cut) {
        // (a cut below every number lets all through)
        const float cut_v = key_value((uint64_t)cut << 32);
        const bool all = cut < 0x00800000u;
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if ((c.v[i] >= cut_v || all) && C::index(c0, i) < hi) {
            const int to = atomicAdd(&n_cand, 1);
            if (to < kCand - AIO_MAX_TOP) cand[to] = order_key(c.v[i], C::index(c0, i));
          }
      }
      __syncthreads();
      exact = n_cand > kCand - AIO_MAX_TOP;
    }
    if (exact) {
      // (rare: the values are read again, so that their registers are free by now)
      uint64_t mk = 0;
#pragma unroll 1
      for (int i = 0; i < PER; ++i) {
        const int e = C::index(c0, i);
        if (e < hi) mk = max(mk, order_key(load1(x, e), e));
      }
      __syncthreads();  // every thread has read n_cand
      maxima[tid] = mk;
      if (tid == 0) {
        cut_s = 1;
        n_cand = 0;
      }
      __syncthreads();
      int r = 0;
#pragma unroll 4
      for (int j = 0; j < kBlock; ++j) r += maxima[j] > mk;
      if (mk && r == a.top - 1) cut_s = mk;
      __syncthreads();
      const uint64_t from = max(cut_s, kth);
#pragma unroll 1
      for (int i = 0; i < PER; ++i) {
        const int e = C::index(c0, i);
        const uint64_t k = e < hi ? order_key(load1(x, e), e) : 0;
        if (k >= from) cand[atomicAdd(&n_cand, 1)] = k;
      }
      __syncthreads();
    }
    // the best so far join them
    const int n = n_cand;
    const uint64_t old = tid < a.top ? best[tid] : 0;
    const int have = __popcll(__ballot(old != 0));  // (a prefix; wave 0 holds them all)
    if (old) cand[n + tid] = old;
    if (tid == 0) maxima[0] = have;
    __syncthreads();
    rank_candidates(cand, n + (int)maxima[0], a.top, best);
    if (tid == 0) n_cand = 0;
  }
  st = wave_join(st);
  if (lane == 0) ws[tid / AIO_WAVE] = st;
  __syncthreads();
  st = ws[0];
#pragma unroll
  for (int w = 1; w < kBlock / AIO_WAVE; ++w) st = join(st, ws[w]);
  if (a.slices == 1) {
    finish_row<T>(a, row, st, best);
    return;
  }
  const int64_t at = (int64_t)row * a.slices + slice;
  if (tid == 0) {
    a.part[at * 3] = st.m;
    a.part[at * 3 + 1] = st.z;
    a.part[at * 3 + 2] = st.w;
  }
  if (tid < a.top) a.part_top[at * a.top + tid] = best[tid];
}

// One workgroup per row: joins its slices (at most 64), each with its candidates in
// descending order.  With d = ceil(top / slices) and k = ceil(top / d) slices whose d-th
// candidates are the largest, d k >= top candidates lie at or above the k-th of those:
// only what is not below it is ranked, about `top` of them in place of slices top (one row
// of 32000, top 20: 12.5 us in both launches, 19.8 with all ranked; 131072, top 8: 12 and 25).
template <class T>
__global__ __launch_bounds__(kBlock) void k_logprobs_join(LogprobArgs a) {
  __shared__ uint64_t cand[kMaxSlices * AIO_MAX_TOP];
  __shared__ uint64_t best[AIO_MAX_TOP];
  __shared__ uint64_t heads[kMaxSlices];
  __shared__ int n_cand;
  const int tid = threadIdx.x, lane = tid & (AIO_WAVE - 1), row = blockIdx.x;
  const int64_t at = (int64_t)row * a.slices;
  Stats st{-INFINITY, 0.0, 0.0};
  if (lane < a.slices) {
    const double* p = a.part + (at + lane) * 3;
    st = Stats{(float)p[0], p[1], p[2]};
  }
  if (a.top) {
    const int d = (a.top + a.slices - 1) / a.slices, k = (a.top + d - 1) / d;
    const uint64_t head = lane < a.slices ? a.part_top[(at + lane) * a.top + d - 1] : 0;
    if (tid < a.slices) heads[tid] = head;
    if (tid == 0) n_cand = 0;
    __syncthreads();
    int r = 0;
    for (int j = 0; j < a.slices; ++j) r += heads[j] > head;
    // (a slice with fewer than d values has a 0 there; if it is the k-th, nothing is cut)
    const uint64_t is = __ballot(head != 0 && r == k - 1);
    const uint64_t cut = is ? heads[__ffsll((unsigned long long)is) - 1] : 1;
    for (int i = tid; i < a.slices * a.top; i += kBlock) {
      const uint64_t c = a.part_top[at * a.top + i];
      if (c >= cut) cand[atomicAdd(&n_cand, 1)] = c;
    }
    __syncthreads();
    rank_candidates(cand, n_cand, a.top, best);
  }
  st = wave_join(st);
  __syncthreads();
  finish_row<T>(a, row, st, best);
}

template <class T, int PER, bool VEC>
void launch_slices(const LogprobArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL((k_logprobs<T, PER, VEC>), dim3(a.slices, a.rows), dim3(kBlock), 0, stream, a);
}

template <class T>
void launch(const LogprobArgs& a, hipStream_t stream) {
  for (int r0 = 0; r0 < a.rows; r0 += 65535) {  // (grid.y holds 65535)
    LogprobArgs b = a;
    b.rows = std::min(a.rows - r0, 65535);
    b.x = (const T*)a.x + r0 * a.stride;
    if (a.target) b.target = a.target + r0;
    if (a.logprob) b.logprob = a.logprob + r0;
    if (a.entropy) b.entropy = a.entropy + r0;
    if (a.top) {
      b.ids = a.ids + (int64_t)r0 * a.top;
      b.top_lp = a.top_lp + (int64_t)r0 * a.top;
    }
    const bool vec = ((uintptr_t)b.x | (uintptr_t)(b.stride * sizeof(T))) % 16 == 0;
    // (256 rows of 131072, two slices each: 46 us with 32 values per thread, 69 with 8; one row
    // of 32000, 16 slices of 2048: 10.9 with 8, a quarter of the threads would work with 32)
    if (a.slices > 1 && a.per < kBlock * kPer)
      vec ? launch_slices<T, kPerFew, true>(b, stream) : launch_slices<T, kPerFew, false>(b, stream);
    else
      vec ? launch_slices<T, kPer, true>(b, stream) : launch_slices<T, kPer, false>(b, stream);
    if (a.slices > 1)
      hipLaunchKernelGGL(k_logprobs_join<T>, dim3(b.rows), dim3(kBlock), 0, stream, b);
  }
}

}  // namespace

LogprobPlan aio_logprob_plan(int rows, int n, int top) {
  LogprobPlan p{1, std::max(n, 1), 0};
  // few rows: a row goes to several workgroups, each at least one chunk
  constexpr int chunk = kBlock * kPerFew;
  const int chunks = (n + chunk - 1) / chunk;
  const int want = std::min({chunks, 2 * kCUs / std::max(rows, 1), kMaxSlices});
  if (want > 1) {
    p.per = (chunks + want - 1) / want * chunk;
    p.slices = (n + p.per - 1) / p.per;
  }
  if (p.slices > 1) p.ws = (size_t)std::min(rows, 65535) * p.slices * (24 + 8 * (size_t)top);
  return p;
}

hipError_t aio_launch_logprobs(const LogprobArgs& a, int dtype, hipStream_t stream) {
  if (dtype == AIO_F32) launch<float>(a, stream);
  else launch<uint16_t>(a, stream);
  return hipGetLastError();
}
