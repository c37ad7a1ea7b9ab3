// Rows into the pages of a cache, and copies of pages.  Both only move bytes:
// what bounds them is HBM, or for a few rows the launch.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "paged.h"

namespace {

constexpr int kBlock = 256;

// Page and slot of new row r; false where it has none.  The row's sequence is the number of
// sequences that end at or before it, counted 64 at a time by ballot.
AIO_DEV bool row_place(const AppendArgs& a, int r, int& page, int& slot) {
  const int lane = threadIdx.x & (AIO_WAVE - 1);
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
    if (seq >= a.n_seqs) return false;  // behind the last sequence
    seq_rows(a.cu_q, a.n_rows, seq, first, count);
    if (r < first || r >= first + count) return false;
  }
  // the length as given: a row past what the table or max_len has room for
  // has no slot, and must not fall on another row's
  const int64_t pos = (int64_t)a.kv.lens[seq] - count + (r - first);
  if (pos < 0 || pos >= a.max_len) return false;
  const int64_t idx = pos >> a.kv.shift;
  if (idx >= a.kv.tstride) return false;
  page = a.kv.table[(int64_t)seq * a.kv.tstride + idx];
  if ((unsigned)page >= (unsigned)a.kv.limit) return false;
  slot = (int)(pos & ((1 << a.kv.shift) - 1));
  return true;
}

// One workgroup per new row: 8 elements (16 bytes of cache) per thread, K and
// V (2224 rows of the 7B's 32 heads, fp32: 24 us, 4.5 TB/s; 16 rows of the 1B: 3.5,
// the launch and two dependent reads).
template <bool F32>
__global__ __launch_bounds__(kBlock) void k_page_append(AppendArgs a) {
  const int r = blockIdx.x;
  int page, slot;
  if (!row_place(a, r, page, slot)) return;
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

// The same into 8-bit pages: a head's row is hd / 8 lanes, which find its largest magnitude
// (as an integer: NaN above infinity) and with it the least exponent e for which no code passes
// 127.  With A = (1 + f) 2^E that is E - 6, and one more where A / 2^(E - 6) = 64 (1 + f) rounds to
// 128, that is f >= 127/128 (the tie 127.5 goes to the even 128): a carry of f + 1/128 into
// the exponent.  What bounds it is HBM (1705 rows of the 7B's 32 heads, fp32: 13.2 us, 5.3 TB/s), or
// for a few rows the launch and two dependent reads (16 rows of the 1B: 4.1 us).
template <int HD, bool F32>
__global__ __launch_bounds__(kBlock) void k_q8_append(Append8Args a) {
  const int r = blockIdx.x;
  int page, slot;
  if (!row_place(a, r, page, slot)) return;
  constexpr int PER = HD / 8;
  for (int e = threadIdx.x; e < a.kv.Hkv * PER; e += kBlock) {
    const int h = e / PER, d0 = e % PER * 8;
    const int64_t src = r * a.row_stride + h * a.head_stride + d0;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const void* rows = w ? a.v_rows : a.k_rows;
      float x[8];
      if constexpr (F32) {
        const float4 u = *(const float4*)((const float*)rows + src);
        const float4 v = *(const float4*)((const float*)rows + src + 4);
        x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
        x[4] = v.x; x[5] = v.y; x[6] = v.z; x[7] = v.w;
      } else {
        const u32x4 u = *(const u32x4*)((const uint16_t*)rows + src);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[2 * i] = bf16_lo(u[i]);
          x[2 * i + 1] = bf16_hi(u[i]);
        }
      }
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
      top = max(top, dpp_bits<0xB1>(top));
      top = max(top, dpp_bits<0x4E>(top));
      top = max(top, dpp_bits<0x141>(top));
      if (PER == 16) top = max(top, dpp_bits<0x140>(top));
      const bool finite = top < 0x7f800000u;
      // biased by 127, as the byte
      const int b = min(max((int)((top + 0x10000u) >> 23) - 6, 8), 248);
      const float by = __uint_as_float((uint32_t)(254 - b) << 23);  // 2^(127 - b)
      uint32_t c[2] = {0, 0};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int v = (int)__builtin_rintf(x[i] * by);
        c[i / 4] |= (uint32_t)(min(max(v, -127), 127) & 0xff) << (i % 4 * 8);
      }
      uint8_t* out = (uint8_t*)(w ? a.v : a.k) + page * a.kv.stride + h * a.kv.head_stride +
                     (int64_t)slot * HD + d0;
      *(uint2*)out = finite ? make_uint2(c[0], c[1]) : make_uint2(0, 0);
      if (d0 == 0)
        (w ? a.v_exp : a.k_exp)[page * a.exp_stride + h * a.exp_head_stride + slot] =
            (uint8_t)(finite ? b : 255);
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

hipError_t aio_launch_append8(const Append8Args& a, int dtype, hipStream_t stream) {
  const auto fn = a.hd == 128 ? (dtype == AIO_F32 ? k_q8_append<128, true> : k_q8_append<128, false>)
                              : (dtype == AIO_F32 ? k_q8_append<64, true> : k_q8_append<64, false>);
  hipLaunchKernelGGL(fn, dim3(a.n_rows), dim3(kBlock), 0, stream, a);
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
