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
constexpr int kChunk = kBlock * kPer;
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
    int r = 0;
    for (int j = 0; j < n; ++j) r += cand[j] > k;
    if (r < top) best[r] = k;
  }
}

AIO_DEV void write_stats(const LogprobArgs& a, int row, const Stats& s, double& logz) {
  // a row with nothing above -inf has no distribution
  logz = s.m == -INFINITY ? (double)__uint_as_float(0x7fc00000u) : log(s.z);
  if (threadIdx.x == 0 && a.entropy) a.entropy[row] = (float)(logz - s.w / s.z);
}

AIO_DEV float load1(const float* x, int64_t i) { return x[i]; }
AIO_DEV float load1(const uint16_t* x, int64_t i) { return bf16_to_f32(x[i]); }

template <class T>
AIO_DEV void finish_row(const LogprobArgs& a, int row, const Stats& s, const uint64_t* best) {
  double logz;
  write_stats(a, row, s, logz);
  if (threadIdx.x == 0 && a.logprob) {
    const int t = a.target[row];
    float lp = __uint_as_float(0x7fc00000u);
    if ((unsigned)t < (unsigned)a.n)
      lp = (float)((double)load1((const T*)a.x + row * a.stride, t) - s.m - logz);
    a.logprob[row] = lp;
  }
  if ((int)threadIdx.x < a.top) {
    const uint64_t k = best[threadIdx.x];
    a.ids[(int64_t)row * a.top + threadIdx.x] = key_index(k);
    a.top_lp[(int64_t)row * a.top + threadIdx.x] = (float)((double)key_value(k) - s.m - logz);
  }
}

// Workgroup (slice, row): the slice's statistics and its best candidates; with
// one slice per row, the row's results.
template <class T>
__global__ __launch_bounds__(kBlock) void k_logprobs(LogprobArgs a) {
  __shared__ uint64_t cand[kCand];
  __shared__ uint64_t maxima[kBlock];
  __shared__ uint64_t best[AIO_MAX_TOP];
  __shared__ uint64_t cut;
  __shared__ int n_cand;
  __shared__ Stats ws[kBlock / AIO_WAVE];
  const int tid = threadIdx.x, row = blockIdx.y, slice = blockIdx.x;
  const T* x = (const T*)a.x + row * a.stride;
  const int lo = slice * a.per, hi = min(a.n, lo + a.per);
  Stats st{-INFINITY, 0.0, 0.0};
  if (tid < AIO_MAX_TOP) best[tid] = 0;
  for (int c0 = lo; c0 < hi; c0 += kChunk) {
    float v[kPer];
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = c0 + i * kBlock + tid;
      v[i] = e < hi ? load1(x, e) : -INFINITY;
      m = fmaxf(m, v[i]);
    }
    Stats s{m, 0.0, 0.0};
    bool nan = false;
#pragma unroll
    for (int i = 0; i < kPer; ++i) nan |= v[i] != v[i];
    if (m != -INFINITY || nan) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const float d = v[i] - m;
        const float e = expf(d);
        s.z += (double)e;
        s.w += v[i] == -INFINITY ? 0.0 : (double)e * (double)d;
      }
    }
    st = join(st, s);
    if (a.top > 0) {
      uint64_t mk = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int e = c0 + i * kBlock + tid;
        if (e < hi) mk = max(mk, order_key(v[i], e));
      }
      __syncthreads();  // the chunk before is ranked
      maxima[tid] = mk;
      if (tid == 0) {
        cut = 0;
        n_cand = 0;
      }
      __syncthreads();
      int r = 0;
      for (int j = 0; j < kBlock; ++j) r += maxima[j] > mk;
      if (mk && r == a.top - 1) cut = mk;
      __syncthreads();
      // (fewer than `top` threads with values: cut is 0, and all values are candidates)
      const uint64_t from = max(cut, best[a.top - 1]);
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int e = c0 + i * kBlock + tid;
        if (e < hi) {
          const uint64_t k = order_key(v[i], e);
          if (k >= from) cand[atomicAdd(&n_cand, 1)] = k;
        }
      }
      if (tid < a.top && best[tid]) cand[atomicAdd(&n_cand, 1)] = best[tid];
      __syncthreads();
      rank_candidates(cand, n_cand, a.top, best);
    }
  }
  st = wave_join(st);
  if ((tid & (AIO_WAVE - 1)) == 0) ws[tid / AIO_WAVE] = st;
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

// One workgroup per row: joins its slices.
template <class T>
__global__ __launch_bounds__(kBlock) void k_logprobs_join(LogprobArgs a) {
  __shared__ uint64_t cand[kCand];
  __shared__ uint64_t best[AIO_MAX_TOP];
  const int tid = threadIdx.x, row = blockIdx.x;
  const int64_t at = (int64_t)row * a.slices;
  Stats st{-INFINITY, 0.0, 0.0};
  for (int s = 0; s < a.slices; ++s) {
    const double* p = a.part + (at + s) * 3;
    st = join(st, Stats{(float)p[0], p[1], p[2]});
  }
  const int n = a.slices * a.top;
  for (int i = tid; i < n; i += kBlock) cand[i] = a.part_top[at * a.top + i];
  __syncthreads();
  rank_candidates(cand, n, a.top, best);
  __syncthreads();
  finish_row<T>(a, row, st, best);
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
    hipLaunchKernelGGL(k_logprobs<T>, dim3(a.slices, b.rows), dim3(kBlock), 0, stream, b);
    if (a.slices > 1)
      hipLaunchKernelGGL(k_logprobs_join<T>, dim3(b.rows), dim3(kBlock), 0, stream, b);
  }
}

}  // namespace

LogprobPlan aio_logprob_plan(int rows, int n, int top) {
  LogprobPlan p{1, std::max(n, 1), 0};
  const int chunks = (n + kChunk - 1) / kChunk;
  // few rows: a row goes to several workgroups, each at least one chunk
  const int want = std::max(1, std::min({chunks, kCUs / std::max(rows, 1), 32}));
  if (want > 1) {
    const int each = (chunks + want - 1) / want;
    p.per = each * kChunk;
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
