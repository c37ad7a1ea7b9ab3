// Query and key rows before they are used: the norm of each head and the rotation by
// position in one pass.  Every element is read and written once; what bounds it is HBM (4096 rows
// of 40 heads of 128, bf16: 18.4 us, 4.6 TB/s, where a large copy runs at 5.2), or for a few
// rows the launch (8 rows of 24 heads: 3.8 us).
#include <hip/hip_runtime.h>

#include "paged.h"

namespace {

constexpr int kBlock = 256;

// Cosine and sine of `turns` full turns.  The turn is taken apart in 64 bits, so that positions
// of any size keep their angle: |r| is at most an eighth of a turn, where a float is off by at
// most 2^-28 of a turn.
AIO_DEV float2 cos_sin(double turns) {
  turns -= rint(turns);
  const double q = rint(4.0 * turns);
  float s, c;
  sincospif((float)(2.0 * (turns - 0.25 * q)), &s, &c);
  const int n = (int)q & 3;
  const float a = n & 1 ? s : c, b = n & 1 ? c : s;
  return make_float2(n == 1 || n == 2 ? -a : a, n >= 2 ? -b : b);
}

// Eight elements.
template <bool F32>
AIO_DEV void load8(const void* p, int64_t at, float (&x)[8]) {
  if constexpr (F32) {
    const float4 u = *(const float4*)((const float*)p + at);
    const float4 v = *(const float4*)((const float*)p + at + 4);
    x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
    x[4] = v.x; x[5] = v.y; x[6] = v.z; x[7] = v.w;
  } else {
    const u32x4 u = *(const u32x4*)((const uint16_t*)p + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = bf16_lo(u[i]);
      x[2 * i + 1] = bf16_hi(u[i]);
    }
  }
}
template <bool F32>
AIO_DEV void store8(void* p, int64_t at, const float (&x)[8]) {
  if constexpr (F32) {
    *(float4*)((float*)p + at) = make_float4(x[0], x[1], x[2], x[3]);
    *(float4*)((float*)p + at + 4) = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    u32x4 u;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      u[i] = f32_to_bf16(x[2 * i]) | (uint32_t)f32_to_bf16(x[2 * i + 1]) << 16;
    *(u32x4*)((uint16_t*)p + at) = u;
  }
}

// Sum over the lanes of a head: 4 or 8.
template <int LANES>
AIO_DEV float head_sum(float v) {
  v += dpp_mov<0xB1>(v);
  v += dpp_mov<0x4E>(v);
  if (LANES == 8) v += dpp_mov<0x141>(v);
  return v;
}

// One workgroup per row.  A lane holds 8 elements of a head's lower half and the 8 that they are
// rotated with.
template <int HD, bool F32>
__global__ __launch_bounds__(kBlock) void k_qk_norm_rope(QkArgs a) {
  constexpr int HALF = HD / 2, LANES = HALF / 8;
  __shared__ __align__(16) float2 turn[HALF];
  const int row = blockIdx.x, tid = threadIdx.x;
  if (tid < HALF) turn[tid] = cos_sin((double)a.pos[row] * a.turns[tid]);
  __syncthreads();
  for (int e = tid; e < (a.H + a.Hkv) * LANES; e += kBlock) {
    const int head = e / LANES, d0 = e % LANES * 8;
    const int w = head < a.H ? 0 : 1, h = head - (w ? a.H : 0);
    float x[8], y[8];
    const int64_t in = row * a.ldi[w] + h * HD + d0;
    load8<F32>(a.in[w], in, x);
    load8<F32>(a.in[w], in + HALF, y);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += x[i] * x[i] + y[i] * y[i];
    sum = head_sum<LANES>(sum);
    const float mean = sum * (1.f / HD) + a.eps;
    float inv = rsqrtf(mean);
    if (!(mean >= 0x1p-90f && mean < INFINITY)) {
      // the squares, eps or their sum past the largest float, or next to the smallest, where floats
      // have few bits: of elements 2^-70 or 2^60 times as large, and eps by the square of that
      const float by = mean < 0x1p-90f ? 0x1p60f : 0x1p-70f;
      sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] *= by;
        y[i] *= by;
        sum += x[i] * x[i] + y[i] * y[i];
      }
      inv = rsqrtf(head_sum<LANES>(sum) * (1.f / HD) + a.eps * by * by);
    }
    float wx[8], wy[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) wx[i] = wy[i] = 1.f;
    if (a.w[w]) {
      load8<false>(a.w[w], d0, wx);
      load8<false>(a.w[w], d0 + HALF, wy);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 t = turn[d0 + i];
      const float p = x[i] * inv * wx[i], q = y[i] * inv * wy[i];
      x[i] = p * t.x - q * t.y;
      y[i] = q * t.x + p * t.y;
    }
    const int64_t out = row * a.ldo[w] + h * HD + d0;
    store8<F32>(a.out[w], out, x);
    store8<F32>(a.out[w], out + HALF, y);
  }
}

}  // namespace

hipError_t aio_launch_qk(const QkArgs& a, int hd, int dtype, hipStream_t stream) {
  const auto fn = hd == 128 ? (dtype == AIO_F32 ? k_qk_norm_rope<128, true> : k_qk_norm_rope<128, false>)
                            : (dtype == AIO_F32 ? k_qk_norm_rope<64, true> : k_qk_norm_rope<64, false>);
  hipLaunchKernelGGL(fn, dim3(a.n_rows), dim3(kBlock), 0, stream, a);
  return hipGetLastError();
}
