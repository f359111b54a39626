// Device-side helpers of the kernels that hold values in 8 bits: e4m3 with a
// power-of-two scale (E8M0: byte b stands for 2^(b - 127)) for each block of
// 128 values.
#pragma once

#include "hydra_device.h"
#include "hydra_elem.h"

namespace hydra {

constexpr int kFp8Block = 128;

typedef __attribute__((__vector_size__(8 * sizeof(int)))) int i32x8_t;

// The scale byte for a block whose largest finite magnitude is a: the least
// 2^e >= 2^-127 with a <= 448 2^e (448 = 1.75 * 2^8 is e4m3's largest value).
__device__ __forceinline__ int fp8_scale_byte(float a) {
  const uint32_t u = __float_as_uint(a);
  const int b = int(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return b > 0 ? b : 0;
}
// 2^-(b - 127), exact for every byte the function above returns (0 ... 247).
__device__ __forceinline__ float fp8_inverse(int b) { return __uint_as_float(uint32_t(254 - b) << 23); }

// |x|, and 0 for what is not finite.
__device__ __forceinline__ float fp8_magnitude(float x) {
  const float a = fabsf(x);
  return a <= 3.4028235e38f ? a : 0.f;
}

// Four values times p as e4m3 bytes, nearest, ties to even; NaN and infinities
// become NaN.  The product is exact (p a power of two; what fp32 cannot hold of
// it is far below e4m3's least value), so every value is rounded once.
__device__ __forceinline__ uint32_t fp8_pack4(const float* x, float p) {
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = fabsf(x[i]) <= 3.4028235e38f ? x[i] * p : __uint_as_float(0x7FC00000u);
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], w, true);
  return (uint32_t)w;
}

// D = A * B + C on one 32x32 tile with a K = 64 step, e4m3 inputs times the
// scales.  The matrix cores add the products of each group of eight consecutive k
// with about 13 bits below the largest of them, and the groups in fp32: sums of
// typical rows are 2e-5 off (1.3e-5 of 64 values of a normal distribution; the
// unscaled fp8 instructions are the same), a two-hundredth of a step of bf16.  Lane l supplies 32 values of row (l % 32) of A
// and of column (l % 32) of B (k-group l / 32, the same k in both) and, in the
// low byte of sa and sb, their scale bytes; D as in mfma32.
__device__ __forceinline__ f32x16_t mfma32_fp8(const uint4& a0, const uint4& a1, const uint4& b0, const uint4& b1,
                                               const f32x16_t& c, int sa, int sb) {
  const i32x8_t a = {(int)a0.x, (int)a0.y, (int)a0.z, (int)a0.w, (int)a1.x, (int)a1.y, (int)a1.z, (int)a1.w};
  const i32x8_t b = {(int)b0.x, (int)b0.y, (int)b0.z, (int)b0.w, (int)b1.x, (int)b1.y, (int)b1.z, (int)b1.w};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, sa, 0, sb);
}

// Sixteen e4m3 bytes times the scale of byte b as bf16 (exact but for results below
// 2^-126, four fraction bits of eight): v[0] the first eight, v[1] the others.
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2_t;
__device__ __forceinline__ void fp8_to_bf16(const uint4& q, int b, uint4 (&v)[2]) {
  const float s = __uint_as_float((uint32_t)b << 23);
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
  uint32_t o[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], s, false));
    o[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], s, true));
  }
  v[0] = make_uint4(o[0], o[1], o[2], o[3]);
  v[1] = make_uint4(o[4], o[5], o[6], o[7]);
}

}  // namespace hydra
