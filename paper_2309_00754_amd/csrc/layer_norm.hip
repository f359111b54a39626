// Layer norm of M rows of K values and its backward, for gfx950 (OPT's layers;
// the update stage of Sec. 2 Stage 3 takes the linears' dx through it).
//
//   mean = sum x / K, var = sum (x - mean)^2 / K, rstd = 1 / sqrt(var + eps)
//   y = (x - mean) rstd w + b
//   g = dy w, xh = (x - mean) rstd
//   dx = rstd (g - sum g / K - xh sum (g xh) / K), dw = sum_m dy xh, db = sum_m dy
//
//  * layer_norm_kernel: one workgroup per row, three passes over it (the sum,
//    the centred squares, the result).
//  * norm_back_rows_kernel: one workgroup per row, the two sums of dx.
//  * norm_back_kernel: a thread per column over a chunk of rows: dx and the
//    chunk's part of dw and db.
//  * norm_back_sum_kernel: adds the chunks' parts in chunk order.
// Statistics, products and sums are fp32; results are rounded once.
#include "hydra_device.h"
#include "hydra_internal.h"

namespace hydra {
namespace {

__device__ __forceinline__ float load1(const void* p, int type, size_t i) {
  return type == kF32 ? static_cast<const float*>(p)[i] : bf16_to_f32(static_cast<const uint16_t*>(p)[i]);
}

__device__ __forceinline__ void store1(void* p, int type, size_t i, float v) {
  if (type == kF32)
    static_cast<float*>(p)[i] = v;
  else
    static_cast<uint16_t*>(p)[i] = f32_to_bf16_any(v);
}

constexpr int LN_THREADS = 256;

// Sum over the workgroup, in a fixed order, in every thread.
__device__ __forceinline__ float block_sum(float v) {
  __shared__ float part[LN_THREADS / 64];
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
  __syncthreads();  // (the last call's parts have been read)
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
#pragma unroll
  for (int i = 1; i < LN_THREADS / 64; ++i) v += part[i];
  return v;
}

__global__ __launch_bounds__(LN_THREADS) void layer_norm_kernel(LayerNormArgs a) {
  const int row = blockIdx.x, t = threadIdx.x, K = a.K;
  const size_t r0 = (size_t)row * K;
  float s = 0.f;
  for (int k = t; k < K; k += LN_THREADS) s += load1(a.x, a.x_type, r0 + k);
  const float mean = block_sum(s) / (float)K;
  s = 0.f;
  for (int k = t; k < K; k += LN_THREADS) {
    const float c = load1(a.x, a.x_type, r0 + k) - mean;
    s = fmaf(c, c, s);
  }
  const float rstd = 1.f / sqrtf(block_sum(s) / (float)K + a.eps);
  for (int k = t; k < K; k += LN_THREADS) {
    const float w = a.w ? load1(a.w, a.w_type, k) : 1.f, b = a.b ? load1(a.b, a.w_type, k) : 0.f;
    store1(a.y, a.y_type, r0 + k, fmaf((load1(a.x, a.x_type, r0 + k) - mean) * rstd, w, b));
  }
  if (t == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
}

__global__ __launch_bounds__(LN_THREADS) void norm_back_rows_kernel(LayerNormBackArgs a, float2* sums) {
  const int row = blockIdx.x, t = threadIdx.x, K = a.K;
  const size_t r0 = (size_t)row * K;
  const float mean = a.mean[row], rstd = a.rstd[row];
  float s0 = 0.f, s1 = 0.f;
  for (int k = t; k < K; k += LN_THREADS) {
    const float g = load1(a.dy, a.dy_type, r0 + k) * (a.w ? load1(a.w, a.w_type, k) : 1.f);
    s0 += g;
    s1 = fmaf(g, (load1(a.x, a.x_type, r0 + k) - mean) * rstd, s1);
  }
  s0 = block_sum(s0);
  s1 = block_sum(s1);
  if (t == 0) sums[row] = make_float2(s0 / (float)K, s1 / (float)K);
}

// Columns of one workgroup; rows are split into nch chunks of `rows`.
__global__ __launch_bounds__(LN_THREADS) void norm_back_kernel(LayerNormBackArgs a, const float2* sums, float* part,
                                                               int rows) {
  const int k = blockIdx.x * LN_THREADS + threadIdx.x, K = a.K;
  if (k >= K) return;
  const int m0 = blockIdx.y * rows, m1 = min(a.M, m0 + rows);
  const float w = a.w ? load1(a.w, a.w_type, k) : 1.f;
  float dw = 0.f, db = 0.f;
  for (int m = m0; m < m1; ++m) {
    const size_t i = (size_t)m * K + k;
    const float dy = load1(a.dy, a.dy_type, i), rstd = a.rstd[m];
    const float xh = (load1(a.x, a.x_type, i) - a.mean[m]) * rstd;
    dw = fmaf(dy, xh, dw);
    db += dy;
    if (a.dx) {
      const float2 s = sums[m];
      store1(a.dx, a.dx_type, i, rstd * (fmaf(dy, w, -s.x) - xh * s.y));
    }
  }
  float* p = part + (size_t)blockIdx.y * 2 * K;
  p[k] = dw;
  p[K + k] = db;
}

__global__ __launch_bounds__(LN_THREADS) void norm_back_sum_kernel(const float* part, int nch, int K, float* dw,
                                                                   float* db) {
  const int k = blockIdx.x * LN_THREADS + threadIdx.x;
  if (k >= 2 * K) return;
  float s = 0.f;
  for (int c = 0; c < nch; ++c) s += part[(size_t)c * 2 * K + k];
  if (k < K) {
    if (dw) dw[k] = s;
  } else if (db) {
    db[k - K] = s;
  }
}

// Row chunks of the backward: about 1024 workgroups over columns and rows, at
// most 256 chunks.
void back_plan(int M, int K, int& nch, int& rows) {
  const int cols = (K + LN_THREADS - 1) / LN_THREADS;
  const int want = (1024 + cols - 1) / cols;
  nch = want < 256 ? want : 256;
  rows = (M + nch - 1) / nch;
  nch = (M + rows - 1) / rows;
}

size_t sums_bytes(int M) { return ((size_t)M * sizeof(float2) + 15) & ~size_t(15); }

}  // namespace

size_t layer_norm_back_ws_bytes(int M, int K) {
  int nch, rows;
  back_plan(M, K, nch, rows);
  return sums_bytes(M) + (size_t)nch * 2 * K * sizeof(float);
}

hipError_t launch_layer_norm(const LayerNormArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(layer_norm_kernel, dim3(a.M), dim3(LN_THREADS), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_layer_norm_back(const LayerNormBackArgs& a, void* ws, hipStream_t stream) {
  int nch, rows;
  back_plan(a.M, a.K, nch, rows);
  float2* sums = static_cast<float2*>(ws);
  float* part = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + sums_bytes(a.M));
  const int cols = (a.K + LN_THREADS - 1) / LN_THREADS;
  if (a.dx) hipLaunchKernelGGL(norm_back_rows_kernel, dim3(a.M), dim3(LN_THREADS), 0, stream, a, sums);
  hipLaunchKernelGGL(norm_back_kernel, dim3(cols, nch), dim3(LN_THREADS), 0, stream, a, sums, part, rows);
  if (a.dw || a.db)
    hipLaunchKernelGGL(norm_back_sum_kernel, dim3((2 * a.K + LN_THREADS - 1) / LN_THREADS), dim3(LN_THREADS), 0, stream,
                       part, nch, a.K, a.dw, a.db);
  return hipGetLastError();
}

}  // namespace hydra
