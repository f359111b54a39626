// Device-side helpers of the kernels that take bf16 or fp32 tensors: elements of
// either type, 16-byte groups of them, and reductions over a wave.
#pragma once

#include "hydra_device.h"
#include "hydra_internal.h"

namespace hydra {

typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4_t;
typedef __attribute__((__vector_size__(2 * sizeof(uint32_t)))) uint32_t u32x2_t;

// float -> bf16 bits, round to nearest even, by the hardware's conversion (NaN
// stays NaN).
__device__ __forceinline__ uint16_t f32_to_bf16_any(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ __forceinline__ uint32_t f32_to_bf16_pair(float lo, float hi) {
  return (uint32_t)f32_to_bf16_any(lo) | ((uint32_t)f32_to_bf16_any(hi) << 16);
}

__device__ __forceinline__ float load_elem(const void* p, int type, size_t i) {
  return type == kF32 ? static_cast<const float*>(p)[i] : bf16_to_f32(static_cast<const uint16_t*>(p)[i]);
}

__device__ __forceinline__ void store_elem(void* p, int type, size_t i, float v) {
  if (type == kF32)
    static_cast<float*>(p)[i] = v;
  else
    static_cast<uint16_t*>(p)[i] = f32_to_bf16_any(v);
}

// Elements of 16 bytes.
template <int T>
constexpr int kVec = T == kF32 ? 4 : 8;

template <int T>
__device__ __forceinline__ void unpack(const uint4& u, float (&f)[kVec<T>]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (T == kF32) {
      f[i] = __uint_as_float(w[i]);
    } else {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
}

// Four bf16 elements (for results that are twice as wide: a lane that loads 16
// bytes and stores 32 leaves gaps of 16 bytes in each of its two stores).
__device__ __forceinline__ void unpack(const u32x2_t& u, float (&f)[4]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    f[2 * i] = __uint_as_float(u[i] << 16);
    f[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
  }
}

template <bool MAX>
__device__ __forceinline__ float combine(float a, float b) {
  return MAX ? fmaxf(a, b) : a + b;
}

// Maximum or sum over the wave's lanes in a fixed order, in every lane: each row
// of 16 lanes by shifts of 1, 2, 4 and 8, then the last lane of rows 0 and 2 into
// rows 1 and 3, and that of row 1 into rows 2 and 3.
template <bool MAX>
__device__ __forceinline__ float wave_all(float v) {
  const uint32_t none = __float_as_uint(MAX ? -INFINITY : 0.f);
#define HYDRA_DPP(ctrl, rows) \
  v = combine<MAX>(v, __uint_as_float(__builtin_amdgcn_update_dpp(none, __float_as_uint(v), ctrl, rows, 0xF, false)))
  HYDRA_DPP(0x111, 0xF);
  HYDRA_DPP(0x112, 0xF);
  HYDRA_DPP(0x114, 0xF);
  HYDRA_DPP(0x118, 0xF);
  HYDRA_DPP(0x142, 0xA);
  HYDRA_DPP(0x143, 0xC);
#undef HYDRA_DPP
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}
__device__ __forceinline__ float wave_sum(float v) { return wave_all<false>(v); }
__device__ __forceinline__ float wave_max(float v) { return wave_all<true>(v); }

}  // namespace hydra
