// Rows into the pages of a cache, and copies of pages.  Both only move bytes:
// what bounds them is HBM, or for a few rows the launch.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "paged.h"

namespace {

constexpr int kBlock = 256;

// One workgroup per new row: 8 elements (16 bytes of cache) per thread, K and
// V (2224 rows of the 7B's 32 heads, fp32: 24 us, 4.5 TB/s; 16 rows of the 1B: 3.5,
// the launch and two dependent reads).  The row's sequence is the number of sequences that end at or before it,
// counted 64 at a time by ballot.
template <bool F32>
__global__ __launch_bounds__(kBlock) void k_page_append(AppendArgs a) {
  const int r = blockIdx.x, lane = threadIdx.x & (AIO_WAVE - 1);
  int seq = r, first = r, count = 1;
  if (a.cu_q) {
    seq = 0;
    for (int base = 0; base < a.n_seqs; base += AIO_WAVE) {
      const int i = base + lane;
      const bool before = i < a.n_seqs && a.cu_q[i + 1] <= r;
      const int c = __popcll(__ballot(before));
      seq += c;
      if (c < AIO_WAVE) break;
    }
    if (seq >= a.n_seqs) return;  // behind the last sequence
    seq_rows(a.cu_q, a.n_rows, seq, first, count);
    if (r < first || r >= first + count) return;
  }
  // the length as given: a row past what the table or max_len has room for
  // has no slot, and must not fall on another row's
  const int64_t pos = (int64_t)a.kv.lens[seq] - count + (r - first);
  if (pos < 0 || pos >= a.max_len) return;
  const int64_t idx = pos >> a.kv.shift;
  if (idx >= a.kv.tstride) return;
  const int page = a.kv.table[(int64_t)seq * a.kv.tstride + idx];
  if ((unsigned)page >= (unsigned)a.kv.limit) return;
  const int slot = (int)(pos & ((1 << a.kv.shift) - 1));
  const int per = a.hd / 8, vecs = a.kv.Hkv * per;
  const int64_t to = page * a.kv.stride + (int64_t)slot * a.hd;
  for (int e = threadIdx.x; e < vecs; e += kBlock) {
    const int h = e >> (hd_shift(a.hd) - 3), d0 = (e & (per - 1)) * 8;
    const int64_t src = r * a.row_stride + h * a.head_stride + d0;
    const int64_t dst = to + h * a.kv.head_stride + d0;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const void* rows = w ? a.v_rows : a.k_rows;
      uint16_t* out = (w ? a.v : a.k) + dst;
      u32x4 o;
      if constexpr (F32) {
        const float* f = (const float*)rows + src;
        const float4 x = *(const float4*)f, y = *(const float4*)(f + 4);
        o.x = f32_to_bf16(x.x) | (uint32_t)f32_to_bf16(x.y) << 16;
        o.y = f32_to_bf16(x.z) | (uint32_t)f32_to_bf16(x.w) << 16;
        o.z = f32_to_bf16(y.x) | (uint32_t)f32_to_bf16(y.y) << 16;
        o.w = f32_to_bf16(y.z) | (uint32_t)f32_to_bf16(y.w) << 16;
      } else {
        o = *(const u32x4*)((const uint16_t*)rows + src);
      }
      *(u32x4*)out = o;
    }
  }
}

// Workgroup (chunk, copy, plane): 16 KB of one page of one plane, past the caches.
// 200 pages of the 1B (629 MB read and written): 112 us, 5.6 TB/s, where a large copy
// runs at 5.2 (through the caches 124 us).
constexpr int kCopyUnroll = 4;
constexpr int kCopyChunk = kBlock * 16 * kCopyUnroll;

__global__ __launch_bounds__(kBlock) void k_page_copy(CopyArgs a) {
  const int64_t at = (int64_t)blockIdx.x * kCopyChunk + threadIdx.x * 16;
  char* plane = a.pool + (int64_t)blockIdx.z * a.plane;
  const char* src = plane + a.pair[blockIdx.y][0] * a.stride + at;
  char* dst = plane + a.pair[blockIdx.y][1] * a.stride + at;
  u32x4 v[kCopyUnroll];
#pragma unroll
  for (int i = 0; i < kCopyUnroll; ++i)
    if (at + i * kBlock * 16 < a.bytes) v[i] = __builtin_nontemporal_load((const u32x4*)(src + i * kBlock * 16));
#pragma unroll
  for (int i = 0; i < kCopyUnroll; ++i)
    if (at + i * kBlock * 16 < a.bytes) __builtin_nontemporal_store(v[i], (u32x4*)(dst + i * kBlock * 16));
}

}  // namespace

hipError_t aio_launch_append(const AppendArgs& a, int dtype, hipStream_t stream) {
  if (dtype == AIO_F32)
    hipLaunchKernelGGL(k_page_append<true>, dim3(a.n_rows), dim3(kBlock), 0, stream, a);
  else
    hipLaunchKernelGGL(k_page_append<false>, dim3(a.n_rows), dim3(kBlock), 0, stream, a);
  return hipGetLastError();
}

hipError_t aio_launch_copy(const CopyArgs& a, int planes, hipStream_t stream) {
  const int64_t chunks = (a.bytes + kCopyChunk - 1) / kCopyChunk;
  // (grid.z holds 65535)
  for (int p0 = 0; p0 < planes; p0 += 65535) {
    CopyArgs b = a;
    b.pool += (int64_t)p0 * a.plane;
    hipLaunchKernelGGL(k_page_copy, dim3((unsigned)chunks, a.n, std::min(planes - p0, 65535)),
                       dim3(kBlock), 0, stream, b);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
