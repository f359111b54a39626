// bf16 or fp32 matrices to e4m3 with a power-of-two scale for each block of 128
// values of a row, or of 128 x 128 values (a frozen weight, with its transpose
// in the same pass).
//
// Per block: a = the largest finite magnitude, e = the least integer >= -127
// with a <= 448 2^e, q = e4m3(x 2^-e).  A power of two moves every value by its
// exponent alone, so a value is rounded once, and the matrix cores take the
// scale as it is.
//
// Bound: memory.  A block's values stay in registers between the maximum and
// the conversion, so x is read once; the transpose goes through LDS, so both
// copies are written in rows.  2048 x 4096 bf16 by rows 6.8 us (3.7 TB/s read and
// written); 11008 x 4096 by tiles, both copies, 45 us (4.0 TB/s).
#include "hydra_fp8.h"

namespace hydra {
namespace {

constexpr int QT = 256;  // threads

// Eight values from column c of a row of K: 16-byte loads (VEC: K % 8 == 0, rows
// 16-byte aligned), else one by one, zeros past the row.
template <int T, bool VEC>
__device__ __forceinline__ void load8(const void* row, int c, int K, float (&f)[8]) {
  if constexpr (VEC) {
    if (c >= K) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = 0.f;
    } else if constexpr (T == kF32) {
      const uint4* p = reinterpret_cast<const uint4*>(static_cast<const float*>(row) + c);
      float a[4], b[4];
      unpack<kF32>(p[0], a);
      unpack<kF32>(p[1], b);
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = a[i], f[4 + i] = b[i];
    } else {
      unpack<kBf16>(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(row) + c), f);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = c + i < K ? load_elem(row, T, c + i) : 0.f;
  }
}

// Eight bytes to column c of a row of K.
template <bool VEC>
__device__ __forceinline__ void store8(uint8_t* row, int c, int K, uint2 v) {
  if constexpr (VEC) {
    if (c < K) *reinterpret_cast<uint2*>(row + c) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < K) row[c + i] = (uint8_t)((i < 4 ? v.x : v.y) >> (8 * (i & 3)));
  }
}

__device__ __forceinline__ float max8(const float (&f)[8]) {
  float a = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) a = fmaxf(a, fp8_magnitude(f[i]));
  return a;
}

// Rows: a block is 16 lanes of 8 values, a workgroup 16 blocks.
template <int T, bool VEC>
__global__ __launch_bounds__(QT) void quantize_rows_kernel(Fp8QuantArgs g, int64_t blocks, int kb_n) {
  const int64_t b = (int64_t)blockIdx.x * (QT / 16) + threadIdx.x / 16;
  if (b >= blocks) return;
  const int64_t m = b / kb_n;
  const int kb = (int)(b - m * kb_n);
  const int c = kb * kFp8Block + (threadIdx.x & 15) * 8;
  float f[8];
  load8<T, VEC>(static_cast<const char*>(g.x) + (size_t)m * g.K * (T == kF32 ? 4 : 2), c, g.K, f);
  float a = max8(f);
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) a = fmaxf(a, __shfl_xor(a, d, 16));
  const int byte = fp8_scale_byte(a);
  const float p = fp8_inverse(byte);
  store8<VEC>(g.q + (size_t)m * g.K, c, g.K, make_uint2(fp8_pack4(f, p), fp8_pack4(f + 4, p)));
  if ((threadIdx.x & 15) == 0) g.scale[b] = (uint8_t)byte;
}

// One 128 x 128 block a workgroup: thread t holds rows 8 (t / 16) ... + 7 of
// columns 8 (t % 16) ... + 7, and with qt turns its 8 x 8 bytes in registers.
template <int T, bool VEC, bool VECT>
__global__ __launch_bounds__(QT) void quantize_tiles_kernel(Fp8QuantArgs g, int kb_n, int mb_n) {
  __shared__ float red[QT / 64];
  // rows of 128 bytes, 16 apart from the next: the eight-byte writes of a wave (four rows' groups of sixteen columns)
  // and the 16-byte reads both spread over the banks
  constexpr int LD = 144;
  __shared__ __align__(16) uint8_t turn[kFp8Block * LD];
  const int t = threadIdx.x;
  const int mb = blockIdx.x / kb_n, kb = blockIdx.x - mb * kb_n;
  const int m0 = mb * kFp8Block + (t / 16) * 8, lc = (t & 15) * 8, c = kb * kFp8Block + lc;
  float f[8][8];
  float a = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (m0 + i < g.M) {
      load8<T, VEC>(static_cast<const char*>(g.x) + (size_t)(m0 + i) * g.K * (T == kF32 ? 4 : 2), c, g.K, f[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[i][j] = 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) a = fmaxf(a, max8(f[i]));
  a = wave_max(a);
  if ((t & 63) == 0) red[t >> 6] = a;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < QT / 64; ++i) a = fmaxf(a, red[i]);
  const int byte = fp8_scale_byte(a);
  const float p = fp8_inverse(byte);
  if (t == 0) {
    g.scale[(size_t)mb * kb_n + kb] = (uint8_t)byte;
    if (g.qt) g.scale_t[(size_t)kb * mb_n + mb] = (uint8_t)byte;
  }
  uint2 q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    q[i] = make_uint2(fp8_pack4(f[i], p), fp8_pack4(f[i] + 4, p));
    if (m0 + i < g.M) store8<VEC>(g.q + (size_t)(m0 + i) * g.K, c, g.K, q[i]);
  }
  if (!g.qt) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint32_t lo = 0, hi = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo |= (((j < 4 ? q[i].x : q[i].y) >> (8 * (j & 3))) & 0xFFu) << (8 * i);
      hi |= (((j < 4 ? q[4 + i].x : q[4 + i].y) >> (8 * (j & 3))) & 0xFFu) << (8 * i);
    }
    *reinterpret_cast<uint2*>(turn + (lc + j) * LD + (t / 16) * 8) = make_uint2(lo, hi);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = i * 32 + t / 8, col = (t & 7) * 16;  // of the transposed block
    const int k = kb * kFp8Block + row, m = mb * kFp8Block + col;
    if (k >= g.K || m >= g.M) continue;
    const uint8_t* src = turn + row * LD + col;
    uint8_t* dst = g.qt + (size_t)k * g.M + m;
    if constexpr (VECT) {
      *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(src);
    } else {
      for (int j = 0; j < 16 && m + j < g.M; ++j) dst[j] = src[j];
    }
  }
}

bool at16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <int T, bool VEC>
void launch_tiles(const Fp8QuantArgs& a, int kb, int mb, hipStream_t stream) {
  const dim3 grid((unsigned)((int64_t)mb * kb)), block(QT);
  if (a.qt && a.M % 16 == 0 && at16(a.qt))
    hipLaunchKernelGGL((quantize_tiles_kernel<T, VEC, true>), grid, block, 0, stream, a, kb, mb);
  else
    hipLaunchKernelGGL((quantize_tiles_kernel<T, VEC, false>), grid, block, 0, stream, a, kb, mb);
}

template <int T, bool VEC>
void launch_type(const Fp8QuantArgs& a, hipStream_t stream) {
  const int kb = (a.K + kFp8Block - 1) / kFp8Block, mb = (a.M + kFp8Block - 1) / kFp8Block;
  if (a.tiles) return launch_tiles<T, VEC>(a, kb, mb, stream);
  const int64_t blocks = (int64_t)a.M * kb;
  hipLaunchKernelGGL((quantize_rows_kernel<T, VEC>), dim3((unsigned)((blocks + QT / 16 - 1) / (QT / 16))), dim3(QT), 0,
                     stream, a, blocks, kb);
}

}  // namespace

hipError_t launch_fp8_quantize(const Fp8QuantArgs& a, hipStream_t stream) {
  const bool vec = a.K % 8 == 0 && at16(a.x) && (reinterpret_cast<uintptr_t>(a.q) & 7) == 0;
  if (a.x_type == kF32)
    vec ? launch_type<kF32, true>(a, stream) : launch_type<kF32, false>(a, stream);
  else
    vec ? launch_type<kBf16, true>(a, stream) : launch_type<kBf16, false>(a, stream);
  return hipGetLastError();
}

}  // namespace hydra
