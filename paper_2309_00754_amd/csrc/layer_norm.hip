// Layer norm of M rows of K values and its backward, for gfx950 (OPT's layers;
// the update stage of Sec. 2 Stage 3 takes the linears' dx through it).
//
//   mean = sum x / K, var = sum (x - mean)^2 / K, rstd = 1 / sqrt(var + eps)
//   y = (x - mean) rstd w + b
//   g = dy w, xh = (x - mean) rstd
//   dx = rstd (g - sum g / K - xh sum (g xh) / K), dw = sum_m dy xh, db = sum_m dy
//
// Up to K = 16384 a row is held in the registers of 1 to 16 waves and read once:
//  * layer_norm_kernel: sum, centred squares and result from the registers; a
//    row group goes on to further rows with its w and b in registers.
//  * norm_back_kernel: the two sums of dx, dx, and each lane's columns of dw
//    and db added up over the group's rows; the groups of a workgroup meet in
//    LDS, the workgroups' parts in norm_back_sum_kernel, all in a fixed order.
// Longer rows:
//  * layer_norm_long_kernel: one workgroup per row, three passes over it.
//  * norm_back_rows_kernel: one workgroup per row, the two sums of dx; then
//    norm_back_cols_kernel, a thread per column over a chunk of rows, and
//    norm_back_sum_kernel.
// Statistics, products and sums are fp32; results are rounded once.
#include "hydra_elem.h"

#include <initializer_list>

namespace hydra {
namespace {

// VEC elements of type T at element `i` of a buffer (zeros where `i` is out of
// its range), as loaded and as fp32.
template <int T, int VEC>
struct Chunk {
  static constexpr int BYTES = VEC * (T == kF32 ? 4 : 2);
  uint32_t v[BYTES >= 4 ? BYTES / 4 : 1];
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, int byte_off) {
    if constexpr (BYTES >= 16) {
#pragma unroll
      for (int q = 0; q < BYTES / 16; ++q) {
        const uint4 u = buf_load16(r, byte_off + 16 * q);
        v[4 * q] = u.x, v[4 * q + 1] = u.y, v[4 * q + 2] = u.z, v[4 * q + 3] = u.w;
      }
    } else if constexpr (BYTES == 8) {
      const uint2 u = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(r, byte_off, 0, 0));
      v[0] = u.x, v[1] = u.y;
    } else if constexpr (BYTES == 4) {
      v[0] = __builtin_amdgcn_raw_buffer_load_b32(r, byte_off, 0, 0);
    } else {
      v[0] = __builtin_amdgcn_raw_buffer_load_b16(r, byte_off, 0, 0);
    }
  }
  __device__ __forceinline__ float at(int e) const {
    if constexpr (T == kF32)
      return __uint_as_float(v[e]);
    else
      return e & 1 ? __uint_as_float(v[e >> 1] & 0xFFFF0000u) : __uint_as_float(v[e >> 1] << 16);
  }
};

template <int VEC>
__device__ __forceinline__ void store_chunk(__amdgpu_buffer_rsrc_t r, int type, int k, const float (&f)[VEC]) {
  if (type == kF32) {
    if constexpr (VEC == 1) {
      __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(f[0]), r, k * 4, 0, 0);
    } else {
#pragma unroll
      for (int q = 0; q < VEC / 4; ++q)
        __builtin_amdgcn_raw_buffer_store_b128(
            u32x4_t{__float_as_uint(f[4 * q]), __float_as_uint(f[4 * q + 1]), __float_as_uint(f[4 * q + 2]),
                    __float_as_uint(f[4 * q + 3])},
            r, k * 4 + 16 * q, 0, 0);
    }
  } else if constexpr (VEC == 1) {
    __builtin_amdgcn_raw_buffer_store_b16((short)f32_to_bf16_any(f[0]), r, k * 2, 0, 0);
  } else {
    uint32_t u[VEC / 2];
#pragma unroll
    for (int e = 0; e < VEC / 2; ++e)
      u[e] = f32_to_bf16_pair(f[2 * e], f[2 * e + 1]);
    if constexpr (VEC == 8)
      __builtin_amdgcn_raw_buffer_store_b128(u32x4_t{u[0], u[1], u[2], u[3]}, r, k * 2, 0, 0);
    else
      __builtin_amdgcn_raw_buffer_store_b64(u32x2_t{u[0], u[1]}, r, k * 2, 0, 0);
  }
}

// The K values of a vector (w, b) that a lane's columns need, `none` where the
// vector is not there.
template <int VEC, int NCH>
__device__ __forceinline__ void load_vector(const void* p, int type, int K, int k0, int step, float none,
                                            float (&f)[NCH][VEC]) {
#pragma unroll
  for (int c = 0; c < NCH; ++c)
#pragma unroll
    for (int e = 0; e < VEC; ++e) f[c][e] = none;
  if (!p) return;
  const __amdgpu_buffer_rsrc_t r = make_rsrc(p, (uint32_t)K * (type == kF32 ? 4u : 2u));
  if (type == kF32) {
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int k = k0 + c * step;
      Chunk<kF32, VEC> u;
      u.load(r, k < K ? k * 4 : kOutOfRange);
#pragma unroll
      for (int e = 0; e < VEC; ++e) f[c][e] = u.at(e);
    }
  } else {
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int k = k0 + c * step;
      Chunk<kBf16, VEC> u;
      u.load(r, k < K ? k * 2 : kOutOfRange);
#pragma unroll
      for (int e = 0; e < VEC; ++e) f[c][e] = u.at(e);
    }
  }
}

constexpr int kMaxWaves = 16;  // of a row

// Sum over the `nw` waves of a row group (nw a power of two; this wave's group
// starts at wave w0), in every thread.  `red` is used by this call alone until
// the workgroup's next barrier but one.
__device__ __forceinline__ float group_sum(float v, float* red, int nw, int w0, int wave) {
  v = wave_sum(v);
  if (nw == 1) return v;
  if ((threadIdx.x & 63) == 0) red[wave] = v;
  __syncthreads();
  v = red[w0];
  for (int i = 1; i < nw; ++i) v += red[w0 + i];
  return v;
}

// A number that is the same in every lane, in a scalar register.
__device__ __forceinline__ float uniform(float v) {
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v)));
}

// s / count, from inv_k = 1 / count rounded: the product alone misses whole quotients by a
// step (a row of 1000 values of 1000 gets a mean of 1000.00006, and with a small
// eps its result is not the bias), and one correction by the remainder, which is
// exact, gives them.  16384 x 128 bf16 forward takes 7.4 us, 3552 x 9445 57.4 (the
// product alone: 7.2 and 56.4; a division, before both numbers were in scalar
// registers: 7.8 and 59.1).
__device__ __forceinline__ float quotient(float s, float count, float inv_k) {
  const float q = s * inv_k;
  const float c = fmaf(fmaf(-q, count, s), inv_k, q);
  return fabsf(q) < INFINITY ? c : q;  // (of an infinite sum the remainder is no number)
}

// Workgroups of THREADS threads hold THREADS / (64 nw) rows at a time, each in
// nw waves; a lane has NCH chunks of VEC columns, nw * 64 * VEC apart.
template <int TX, int VEC, int NCH, int THREADS>
__global__ __launch_bounds__(THREADS) void layer_norm_kernel(LayerNormArgs a, int nw) {
  __shared__ float red[2][kMaxWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int w0 = wave & -nw, groups = THREADS / 64 / nw, K = a.K;
  const int k0 = ((wave - w0) * 64 + lane) * VEC, step = nw * 64 * VEC;
  constexpr int XB = TX == kF32 ? 4 : 2;
  const int yb = a.y_type == kF32 ? 4 : 2;
  float w[NCH][VEC], b[NCH][VEC];
  load_vector<VEC, NCH>(a.w, a.w_type, K, k0, step, 1.f, w);
  load_vector<VEC, NCH>(a.b, a.w_type, K, k0, step, 0.f, b);
  const float count = uniform((float)K), inv_k = uniform(1.f / (float)K);
  const int per = gridDim.x * groups;
  // (the same number of rounds for every group of the workgroup: it has barriers)
  for (int r0 = blockIdx.x * groups; r0 < a.M; r0 += per) {
    const int row = r0 + (nw == 1 ? wave : w0 / nw);
    const bool live = row < a.M;
    const size_t at = (size_t)(live ? row : 0) * K;
    const __amdgpu_buffer_rsrc_t xr = make_rsrc(static_cast<const uint8_t*>(a.x) + at * XB, live ? (uint32_t)K * XB : 0u);
    Chunk<TX, VEC> x[NCH];
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int k = k0 + c * step;
      x[c].load(xr, k < K ? k * XB : kOutOfRange);
    }
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < VEC; ++e) s += x[c].at(e);
    const float mean = quotient(group_sum(s, red[0], nw, w0, wave), count, inv_k);
    s = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      float q = 0.f;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float d = x[c].at(e) - mean;
        q = fmaf(d, d, q);
      }
      s += k0 + c * step < K ? q : 0.f;
    }
    const float rstd = 1.f / sqrtf(quotient(group_sum(s, red[1], nw, w0, wave), count, inv_k) + a.eps);
    if (!live) continue;
    const __amdgpu_buffer_rsrc_t yr = make_rsrc(static_cast<uint8_t*>(a.y) + at * yb, (uint32_t)K * yb);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int k = k0 + c * step;
      float f[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) f[e] = fmaf((x[c].at(e) - mean) * rstd, w[c][e], b[c][e]);
      if (k < K) store_chunk<VEC>(yr, a.y_type, k, f);
    }
    if (k0 == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
}

// The same layout.  Workgroup i writes its part of dw at pw + i 2 K, of db at pb
// + i 2 K (either may be null).
template <int TD, int TX, int VEC, int NCH, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_back_kernel(LayerNormBackArgs a, float* pw, float* pb, int nw) {
  // the groups' columns of dw, then of db, by place in the group: no two lanes on one bank
  __shared__ float acc[THREADS * NCH * VEC];
  __shared__ float red[2][2][THREADS / 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int w0 = wave & -nw, groups = THREADS / 64 / nw, group = w0 / nw, K = a.K;
  const int k0 = ((wave - w0) * 64 + lane) * VEC, step = nw * 64 * VEC;
  constexpr int DB = TD == kF32 ? 4 : 2, XB = TX == kF32 ? 4 : 2;
  const int ob = a.dx_type == kF32 ? 4 : 2;
  float w[NCH][VEC], dw[NCH][VEC], db[NCH][VEC];
  load_vector<VEC, NCH>(a.w, a.w_type, K, k0, step, 1.f, w);
#pragma unroll
  for (int c = 0; c < NCH; ++c)
#pragma unroll
    for (int e = 0; e < VEC; ++e) dw[c][e] = db[c][e] = 0.f;
  const float count = uniform((float)K), inv_k = uniform(1.f / (float)K);
  // the next row's loads before this row's sums meet, where registers allow it: 4096
  // x 4096 bf16 27.2 us, 31.0 without; 4096 x 2048 fp32 24.9, 26.6 without; 2000 x 11008
  // bf16 38.8, 43.9 without (fp32 at 32 columns a lane spills with it: 122, 64.5 without)
  constexpr bool AHEAD = (NCH * VEC <= 16 || VEC == 8) && THREADS <= 512;
  const int per = gridDim.x * groups;
  int turn = 0;
  Chunk<TD, VEC> dn[AHEAD ? NCH : 1];
  Chunk<TX, VEC> xn[AHEAD ? NCH : 1];
  float mean_n = 0.f, rstd_n = 0.f;
  const auto fetch = [&](int row) __attribute__((always_inline)) {
    const bool live = row < a.M;
    const size_t at = (size_t)(live ? row : 0) * K;
    const __amdgpu_buffer_rsrc_t dr = make_rsrc(static_cast<const uint8_t*>(a.dy) + at * DB, live ? (uint32_t)K * DB : 0u);
    const __amdgpu_buffer_rsrc_t xr = make_rsrc(static_cast<const uint8_t*>(a.x) + at * XB, live ? (uint32_t)K * XB : 0u);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int k = k0 + c * step;
      dn[c].load(dr, k < K ? k * DB : kOutOfRange);
      xn[c].load(xr, k < K ? k * XB : kOutOfRange);
    }
    mean_n = live ? a.mean[row] : 0.f;
    rstd_n = live ? a.rstd[row] : 0.f;
  };
  if constexpr (AHEAD) fetch(blockIdx.x * groups + group);
  for (int r0 = blockIdx.x * groups; r0 < a.M; r0 += per, turn ^= 1) {
    const int row = r0 + group;
    const bool live = row < a.M;
    const size_t at = (size_t)(live ? row : 0) * K;
    Chunk<TD, VEC> d[NCH];
    Chunk<TX, VEC> x[NCH];
    float mean, rstd;
    if constexpr (AHEAD) {
#pragma unroll
      for (int c = 0; c < NCH; ++c) d[c] = dn[c], x[c] = xn[c];
      mean = mean_n, rstd = rstd_n;
      if (r0 + per < a.M) fetch(row + per);
    } else {
      // (not by fetch: 3552 x 9445 fp32 takes 116 us by a function, whose chunks' offsets are
      // formed anew for the stores, 107 here)
      const __amdgpu_buffer_rsrc_t dr = make_rsrc(static_cast<const uint8_t*>(a.dy) + at * DB, live ? (uint32_t)K * DB : 0u);
      const __amdgpu_buffer_rsrc_t xr = make_rsrc(static_cast<const uint8_t*>(a.x) + at * XB, live ? (uint32_t)K * XB : 0u);
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        const int k = k0 + c * step;
        d[c].load(dr, k < K ? k * DB : kOutOfRange);
        x[c].load(xr, k < K ? k * XB : kOutOfRange);
      }
      mean = live ? a.mean[row] : 0.f;
      rstd = live ? a.rstd[row] : 0.f;
    }
    // (columns past K have dy = 0)
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float dy = d[c].at(e), xh = (x[c].at(e) - mean) * rstd, g = dy * w[c][e];
        s0 += g;
        s1 = fmaf(g, xh, s1);
        dw[c][e] = fmaf(dy, xh, dw[c][e]);
        db[c][e] += dy;
      }
    if (!a.dx) continue;
    s0 = wave_sum(s0);
    s1 = wave_sum(s1);
    if (nw > 1) {
      if (lane == 0) {
        red[turn][0][wave] = s0;
        red[turn][1][wave] = s1;
      }
      __syncthreads();
      s0 = red[turn][0][w0];
      s1 = red[turn][1][w0];
      for (int i = 1; i < nw; ++i) {
        s0 += red[turn][0][w0 + i];
        s1 += red[turn][1][w0 + i];
      }
    }
    if (!live) continue;
    s0 = quotient(s0, count, inv_k);
    s1 = quotient(s1, count, inv_k);
    const __amdgpu_buffer_rsrc_t orr = make_rsrc(static_cast<uint8_t*>(a.dx) + at * ob, (uint32_t)K * ob);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int k = k0 + c * step;
      float f[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float xh = (x[c].at(e) - mean) * rstd;
        f[e] = rstd * (fmaf(d[c].at(e), w[c][e], -s0) - xh * s1);
      }
      if (k < K) store_chunk<VEC>(orr, a.dx_type, k, f);
    }
  }
  const int lanes = nw * 64, at0 = threadIdx.x - w0 * 64;
  for (int which = 0; which < 2; ++which) {
    float* const p = which ? pb : pw;
    if (!p) continue;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        acc[((group * NCH + c) * VEC + e) * lanes + at0] = which ? db[c][e] : dw[c][e];
    __syncthreads();
    const __amdgpu_buffer_rsrc_t pr = make_rsrc(p + (size_t)blockIdx.x * 2 * K, (uint32_t)K * 4u);
    const int shift = 31 - __builtin_clz(lanes);
    for (int i = threadIdx.x; i < lanes * NCH; i += THREADS) {  // a lane's place and chunk: whole chunks go out
      const int c = i >> shift, at = i & (lanes - 1), k = c * step + at * VEC;
      if (k >= K) continue;
      float f[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        f[e] = acc[(c * VEC + e) * lanes + at];
        for (int g = 1; g < groups; ++g) f[e] += acc[((g * NCH + c) * VEC + e) * lanes + at];
      }
      store_chunk<VEC>(pr, kF32, k, f);
    }
    __syncthreads();
  }
}

// dw and db from n parts of [2][K], in order: a workgroup takes 64 of the 2 K
// columns, each of its waves a run of the parts.
constexpr int SUM_WAVES = 16;
__global__ __launch_bounds__(SUM_WAVES * 64) void norm_back_sum_kernel(const float* part, int n, int K, float* dw,
                                                                      float* db) {
  __shared__ float red[SUM_WAVES][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t k = (int64_t)blockIdx.x * 64 + lane, K2 = 2 * (int64_t)K;
  const int run = (n + SUM_WAVES - 1) / SUM_WAVES, c0 = wave * run, c1 = min(n, c0 + run);
  float s = 0.f;
  if (k < K2) {
    constexpr int U = 8;
    int c = c0;
    for (; c + U <= c1; c += U) {
      float v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = part[(c + u) * K2 + k];
#pragma unroll
      for (int u = 0; u < U; ++u) s += v[u];
    }
    for (; c < c1; ++c) s += part[c * K2 + k];
  }
  red[wave][lane] = s;
  __syncthreads();
  if (wave != 0 || k >= K2) return;
#pragma unroll
  for (int i = 1; i < SUM_WAVES; ++i) s += red[i][lane];
  if (k < K) {
    if (dw) dw[k] = s;
  } else if (db) {
    db[k - K] = s;
  }
}

// ---- rows longer than the registers hold

constexpr int LONG_THREADS = 1024;

// Sum over the workgroup, in a fixed order, in every thread.
__device__ __forceinline__ float block_sum(float v) {
  __shared__ float part[LONG_THREADS / 64];
  v = wave_sum(v);
  __syncthreads();  // (the last call's parts have been read)
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
#pragma unroll
  for (int i = 1; i < LONG_THREADS / 64; ++i) v += part[i];
  return v;
}

__global__ __launch_bounds__(LONG_THREADS) void layer_norm_long_kernel(LayerNormArgs a) {
  const int row = blockIdx.x, t = threadIdx.x, K = a.K;
  const size_t r0 = (size_t)row * K;
  float s = 0.f;
  for (int k = t; k < K; k += LONG_THREADS) s += load_elem(a.x, a.x_type, r0 + k);
  const float mean = block_sum(s) / (float)K;
  s = 0.f;
  for (int k = t; k < K; k += LONG_THREADS) {
    const float c = load_elem(a.x, a.x_type, r0 + k) - mean;
    s = fmaf(c, c, s);
  }
  const float rstd = 1.f / sqrtf(block_sum(s) / (float)K + a.eps);
  for (int k = t; k < K; k += LONG_THREADS) {
    const float w = a.w ? load_elem(a.w, a.w_type, k) : 1.f, b = a.b ? load_elem(a.b, a.w_type, k) : 0.f;
    store_elem(a.y, a.y_type, r0 + k, fmaf((load_elem(a.x, a.x_type, r0 + k) - mean) * rstd, w, b));
  }
  if (t == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
}

__global__ __launch_bounds__(LONG_THREADS) void norm_back_rows_kernel(LayerNormBackArgs a, float2* sums) {
  const int row = blockIdx.x, t = threadIdx.x, K = a.K;
  const size_t r0 = (size_t)row * K;
  const float mean = a.mean[row], rstd = a.rstd[row];
  float s0 = 0.f, s1 = 0.f;
  for (int k = t; k < K; k += LONG_THREADS) {
    const float g = load_elem(a.dy, a.dy_type, r0 + k) * (a.w ? load_elem(a.w, a.w_type, k) : 1.f);
    s0 += g;
    s1 = fmaf(g, (load_elem(a.x, a.x_type, r0 + k) - mean) * rstd, s1);
  }
  s0 = block_sum(s0);
  s1 = block_sum(s1);
  if (t == 0) sums[row] = make_float2(s0 / (float)K, s1 / (float)K);
}

constexpr int COL_THREADS = 256;

// 256 columns of the rows blockIdx.y * rows ...
__global__ __launch_bounds__(COL_THREADS) void norm_back_cols_kernel(LayerNormBackArgs a, const float2* sums, float* part,
                                                                     int rows) {
  const int k = blockIdx.x * COL_THREADS + threadIdx.x, K = a.K;
  if (k >= K) return;
  const int m0 = blockIdx.y * rows, m1 = min(a.M, m0 + rows);
  const float w = a.w ? load_elem(a.w, a.w_type, k) : 1.f;
  float dw = 0.f, db = 0.f;
  for (int m = m0; m < m1; ++m) {
    const size_t i = (size_t)m * K + k;
    const float dy = load_elem(a.dy, a.dy_type, i), rstd = a.rstd[m];
    const float xh = (load_elem(a.x, a.x_type, i) - a.mean[m]) * rstd;
    dw = fmaf(dy, xh, dw);
    db += dy;
    if (a.dx) {
      const float2 s = sums[m];
      store_elem(a.dx, a.dx_type, i, rstd * (fmaf(dy, w, -s.x) - xh * s.y));
    }
  }
  float* p = part + (size_t)blockIdx.y * 2 * K;
  p[k] = dw;
  p[K + k] = db;
}

// ---- plans

// Columns per lane.  16 as far as 8 waves reach: 4096 x 4096 fp32 forward 26.6
// us (of 32: 28.6; of 8: 26.3), backward 44.1 (of 32: 50.7; of 8: 43.2); bf16
// forward 13.7 (of 32: 12.4; of 8: 18.3), backward 27.2 (of 32: 29.3; of 8: 27.7).
// 32 for rows of up to 16384.  Element by element (rows of odd length or alignment) 16 alone, in 16
// waves above 8192: a chunk's address takes a register too, and 32 spill.  (Of 16
// the backward keeps 20, with two types 35, in scratch memory there; yet 3552 x 9445
// fp32 takes 107 us, by the long rows' kernels 198; bf16 81, by those 251; the
// forward 66, by those 115.)
constexpr int kFew = 16, kMany = 32;
constexpr int kFewK = 8 * 64 * kFew, kManyK = 8 * 64 * kMany;
constexpr int FWD_THREADS = 256, BACK_THREADS = 512, ODD_THREADS = kMaxWaves * 64;

// Waves per row: enough for `lane` columns a lane.
int row_waves(int K, int lane) {
  int nw = 1;
  while (nw * 64 * lane < K) nw *= 2;
  return nw;
}

// Workgroups of the backward.  Each writes a part of dw and db that
// norm_back_sum_kernel reads again: one a CU, or half as many where the rows are
// few, M K up to 2^22.  Small side, with 128 (with 256): K = 2048, 700 rows of bf16
// 10.8 us (11.0), 1500 12.6 (12.8), of fp32 11.0 (11.2) and 13.5 (14.0); K = 4096,
// 333 rows of bf16 11.1 (11.5), 700 12.4 (12.8), of fp32 11.7 (11.7) and 13.9
// (14.5).  Large side, with 256 (with 128): 3000 x 2048 bf16 14.6 (16.4), fp32 18.5
// (19.5); 1500 x 4096 14.8 (16.4) and 19.1 (20.1).  A single one, which needs no
// second launch, where that takes it two rounds of rows at most (8 x 2048 bf16 7.3
// us, 8.5 with the launch; but 16 x 2048, four rounds, 9.6 and 8.5).
int back_blocks(int M, int K, int nw) {
  const int groups = nw < BACK_THREADS / 64 ? BACK_THREADS / 64 / nw : 1, want = (M + groups - 1) / groups;
  if (want <= 2) return 1;
  const int most = (int64_t)M * K <= (1 << 22) ? 128 : 256;
  return want < most ? want : most;
}

// Row chunks of the backward of long rows: about 1024 workgroups over columns and rows.
void long_plan(int M, int K, int& nch, int& rows) {
  const int cols = (K + COL_THREADS - 1) / COL_THREADS;
  nch = (1024 + cols - 1) / cols;
  rows = (M + nch - 1) / nch;
  nch = (M + rows - 1) / rows;
}

size_t sums_bytes(int M) { return ((size_t)M * sizeof(float2) + 15) & ~size_t(15); }

bool aligned16(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (reinterpret_cast<uintptr_t>(p) & 15) return false;
  return true;
}

// At most 1024 workgroups, which then take several rows each: 8192 x 2048 fp32 to
// bf16 22.0 us (2048 of them: 22.5; one for each row group at 32 columns a lane: 24.5).
template <int TX, int VEC, int LANE>
void forward_of(const LayerNormArgs& a, hipStream_t stream) {
  const int nw = row_waves(a.K, LANE);
  if constexpr (LANE == kFew) {  // (of 32 columns a lane rows have 8 waves)
    if (nw <= FWD_THREADS / 64) {
      const int groups = FWD_THREADS / 64 / nw, want = (a.M + groups - 1) / groups;
      hipLaunchKernelGGL((layer_norm_kernel<TX, VEC, LANE / VEC, FWD_THREADS>), dim3(want < 1024 ? want : 1024),
                         dim3(FWD_THREADS), 0, stream, a, nw);
      return;
    }
  }
  hipLaunchKernelGGL((layer_norm_kernel<TX, VEC, LANE / VEC, 512>), dim3(a.M < 512 ? a.M : 512), dim3(512), 0, stream, a, nw);
}

template <int TX, int VEC>
bool forward(const LayerNormArgs& a, hipStream_t stream) {
  if (a.K <= kFewK) {
    forward_of<TX, VEC, kFew>(a, stream);
    return true;
  }
  if (a.K > kManyK) return false;
  if constexpr (VEC > 1)
    forward_of<TX, VEC, kMany>(a, stream);
  else
    hipLaunchKernelGGL((layer_norm_kernel<TX, 1, kFew, ODD_THREADS>), dim3(a.M < 512 ? a.M : 512), dim3(ODD_THREADS), 0, stream,
                       a, kMaxWaves);
  return true;
}

// The number of parts written (1: straight to dw and db), 0 where the row does
// not fit.
template <int TD, int TX, int VEC>
int backward(const LayerNormBackArgs& a, float* part, hipStream_t stream) {
  const bool few = a.K <= kFewK;
  if (a.K > kManyK) return 0;
  const int nw = row_waves(a.K, few || VEC == 1 ? kFew : kMany), blocks = back_blocks(a.M, a.K, nw);
  float* const pw = blocks > 1 ? part : a.dw;
  float* const pb = blocks > 1 && part ? part + a.K : a.db;
  if (few) {
    hipLaunchKernelGGL((norm_back_kernel<TD, TX, VEC, kFew / VEC, BACK_THREADS>), dim3(blocks), dim3(BACK_THREADS), 0, stream,
                       a, pw, pb, nw);
  } else if constexpr (VEC > 1) {
    hipLaunchKernelGGL((norm_back_kernel<TD, TX, VEC, kMany / VEC, BACK_THREADS>), dim3(blocks), dim3(BACK_THREADS), 0,
                       stream, a, pw, pb, nw);
  } else {
    hipLaunchKernelGGL((norm_back_kernel<TD, TX, 1, kFew, ODD_THREADS>), dim3(blocks), dim3(ODD_THREADS), 0, stream, a, pw, pb,
                       nw);
  }
  return blocks;
}

template <int VEC>
int backward_of(const LayerNormBackArgs& a, float* part, hipStream_t stream) {
  if (a.dy_type == kF32)
    return a.x_type == kF32 ? backward<kF32, kF32, VEC>(a, part, stream) : backward<kF32, kBf16, VEC>(a, part, stream);
  if (a.x_type == kF32) return backward<kBf16, kF32, VEC>(a, part, stream);
  return backward<kBf16, kBf16, VEC == 1 ? 1 : 8>(a, part, stream);
}

}  // namespace

size_t layer_norm_back_ws_bytes(int M, int K) {
  // (whatever the types and the alignment of the call)
  if (K <= kManyK) return (size_t)back_blocks(M, K, row_waves(K, K <= kFewK ? kFew : kMany)) * 2 * K * sizeof(float);
  int nch, rows;
  long_plan(M, K, nch, rows);
  return sums_bytes(M) + (size_t)nch * 2 * K * sizeof(float);
}

hipError_t launch_layer_norm(const LayerNormArgs& a, hipStream_t stream) {
  const bool al = aligned16({a.x, a.y, a.w, a.b});
  bool done;
  if (a.x_type == kF32)
    done = al && a.K % 4 == 0 ? forward<kF32, 4>(a, stream) : forward<kF32, 1>(a, stream);
  else
    done = al && a.K % 8 == 0 ? forward<kBf16, 8>(a, stream) : forward<kBf16, 1>(a, stream);
  if (!done) hipLaunchKernelGGL(layer_norm_long_kernel, dim3(a.M), dim3(LONG_THREADS), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_layer_norm_back(const LayerNormBackArgs& a, void* ws, hipStream_t stream) {
  const bool sums = a.dw || a.db, al = aligned16({a.dy, a.x, a.w, a.dx});
  float* part = static_cast<float*>(ws);
  float* const p = sums ? part : nullptr;
  // 16 bytes of bf16 per lane and load where both are bf16, of fp32 where one is
  const bool vec = al && a.K % (a.dy_type == kBf16 && a.x_type == kBf16 ? 8 : 4) == 0;
  int n = vec ? backward_of<4>(a, p, stream) : backward_of<1>(a, p, stream);
  bool add = sums && n > 1;
  if (n == 0) {
    add = sums;
    int rows;
    long_plan(a.M, a.K, n, rows);
    float2* rs = static_cast<float2*>(ws);
    part = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + sums_bytes(a.M));
    const int cols = (a.K + COL_THREADS - 1) / COL_THREADS;
    if (a.dx) hipLaunchKernelGGL(norm_back_rows_kernel, dim3(a.M), dim3(LONG_THREADS), 0, stream, a, rs);
    hipLaunchKernelGGL(norm_back_cols_kernel, dim3(cols, n), dim3(COL_THREADS), 0, stream, a, rs, part, rows);
  }
  if (add)
    hipLaunchKernelGGL(norm_back_sum_kernel, dim3((2 * a.K + 63) / 64), dim3(SUM_WAVES * 64), 0, stream, part, n, a.K, a.dw,
                       a.db);
  return hipGetLastError();
}

}  // namespace hydra
