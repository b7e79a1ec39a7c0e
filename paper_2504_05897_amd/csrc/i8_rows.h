// Quantisation of rows to 8-bit integers on the device (HMOE_BF16_I8): what the quantising launches and the decode kernel,
// which quantises a few rows itself, share.
#pragma once

#include "common.h"

namespace hmoe {

// 8 consecutive values of a row as fp32
__device__ __forceinline__ void load_8(const bf16_t* p, float (&v)[8]) {
  const u32x4 u = *(const u32x4*)p;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(u[i] << 16);
    v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load_8(const float* p, float (&v)[8]) {
  const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
// the bits of the largest magnitude
__device__ __forceinline__ uint32_t magnitude_bits(const float (&v)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
  return m;
}
// What a row's codes are computed with: 127 v (scaled by a power of two where it could overflow) divided by amax and rounded
// as a division is, so that the code is the one that the format names also where the quotient is half a code or next to it.  The
// quotient is the product with the reciprocal, corrected once by what it leaves of 127 v: with a reciprocal that is itself
// refined, which costs a row two instructions, that is the nearest fp32 number.  (A division of the compiler's is ten
// instructions per value: 201 million values 158 -> 118 us.  Without the correction one code of h in four million is another.)
struct RowQuant {
  float times, by, inverse, scale;
  bool finite;
};
__device__ __forceinline__ RowQuant row_quant(uint32_t amax_bits) {
  RowQuant q;
  q.finite = amax_bits < 0x7f800000u;
  const float amax = q.finite ? fmaxf(__uint_as_float(amax_bits), I8_MIN_AMAX) : 1.0f;
  const float down = amax > 0x1p100f ? 0x1p-10f : 1.0f;
  q.times = 127.0f * down;
  q.by = amax * down;
  const float near = __builtin_amdgcn_rcpf(q.by);
  q.inverse = fmaf(fmaf(-near, q.by, 1.0f), near, near);
  q.scale = q.finite ? amax / 127.0f : __uint_as_float(0x7fc00000u);
  return q;
}
// The code of a value is the low byte of the value + 1.5 * 2^23, which has no bits behind the point (nearest even).
__device__ __forceinline__ uint2 codes_of(const float (&v)[8], const RowQuant& q) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 8; i += 4) {
    uint32_t b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float y = v[i + k] * q.times;
      const float s = y * q.inverse;
      b[k] = __float_as_uint(fmaf(fmaf(-s, q.by, y), q.inverse, s) + 12582912.0f);
    }
    w[i / 4] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u), __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), 0x05040100u);
  }
  return q.finite ? make_uint2(w[0], w[1]) : make_uint2(0, 0);
}

// Codes and scale of one row, by the whole block (64 NW threads).  HELD: pieces of 8 values that a thread keeps between the
// maximum and the codes; what is beyond them is read again.
template <int NW, int HELD, class T>
__device__ __forceinline__ void own_row_codes(const T* __restrict__ row, int K, int8_t* codes, float* scale, uint32_t* wave_max) {
  const int tid = threadIdx.x;
  float v[HELD][8];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    const int k = 8 * (i * 64 * NW + tid);
    if (k < K) {
      load_8(row + k, v[i]);
      m = max(m, magnitude_bits(v[i]));
    }
  }
  for (int k = 8 * (HELD * 64 * NW + tid); k < K; k += 8 * 64 * NW) {
    float far[8];
    load_8(row + k, far);
    m = max(m, magnitude_bits(far));
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, off));
  __syncthreads();  // the last row's maxima have been read
  if (tid % 64 == 0) wave_max[tid / 64] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) m = max(m, wave_max[w]);
  const RowQuant q = row_quant(m);
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    const int k = 8 * (i * 64 * NW + tid);
    if (k < K) *(uint2*)(codes + k) = codes_of(v[i], q);
  }
  for (int k = 8 * (HELD * 64 * NW + tid); k < K; k += 8 * 64 * NW) {
    float far[8];
    load_8(row + k, far);
    *(uint2*)(codes + k) = codes_of(far, q);
  }
  if (tid == 0) *scale = q.scale;
}

}  // namespace hmoe
