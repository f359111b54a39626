// The norm over many gradient tensors, and the tensors scaled to a norm of at
// most max_norm, for gfx950 (the update stage's adapters: dA and dB of every
// linear, Sec. 2 Stage 3 and App. B's rank 128).
//
//   norm = sqrt(sum g^2), out = g c, c = max_norm / norm where norm > max_norm, else 1
//
//  * grad_sum_kernel: the tensors of a launch are cut into chunks; a workgroup
//    adds the squares of its chunks in 64 bits and writes its part.
//  * grad_norm_kernel: one workgroup adds the parts.
//  * grad_scale_kernel: every workgroup adds the parts itself (the same order:
//    the same c), then scales its chunks.
// Pointers and sizes travel as kernel arguments, kSegs tensors a launch.
// Squares are formed and added in 64 bits: an fp32 product of two gradients
// below 1e-19 or above 1e19 would leave the range, and the conversion and the
// 64-bit FMA run beside the loads.
#include "hydra_device.h"
#include "hydra_internal.h"

namespace hydra {
namespace {

constexpr int GN_THREADS = 256;
constexpr int GN_CHUNK = 16384;  // elements
constexpr int kSegs = 120;       // (28 bytes each: below the 4 KB of arguments of a launch)
constexpr int kMaxParts = 2048;

struct GradSegs {
  const void* g[kSegs];
  void* out[kSegs];
  int64_t numel[kSegs];
  int chunk0[kSegs];     // first chunk of the tensor
  uint8_t g_type[kSegs], out_type[kSegs];
  int n, chunks;
};

__device__ __forceinline__ float load1(const void* p, int type, int64_t i) {
  return type == kF32 ? static_cast<const float*>(p)[i] : bf16_to_f32(static_cast<const uint16_t*>(p)[i]);
}

// The tensor that chunk c belongs to.
__device__ __forceinline__ int seg_of(const GradSegs& s, int c) {
  int lo = 0, hi = s.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (s.chunk0[mid] <= c)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

// Sum over the workgroup in a fixed order, in every thread.
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double part[GN_THREADS / 64];
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
#pragma unroll
  for (int i = 1; i < GN_THREADS / 64; ++i) v += part[i];
  return v;
}

__global__ __launch_bounds__(GN_THREADS) void grad_sum_kernel(GradSegs s, double* part) {
  const int t = threadIdx.x;
  double sum = 0.0;
  for (int c = blockIdx.x; c < s.chunks; c += gridDim.x) {
    const int i = seg_of(s, c);
    const int64_t e0 = (int64_t)(c - s.chunk0[i]) * GN_CHUNK;
    const int64_t e1 = min(s.numel[i], e0 + GN_CHUNK);
    for (int64_t e = e0 + t; e < e1; e += GN_THREADS) {
      const double v = (double)load1(s.g[i], s.g_type[i], e);
      sum = fma(v, v, sum);
    }
  }
  sum = block_sum(sum);
  if (t == 0) part[blockIdx.x] = sum;
}

__device__ __forceinline__ double norm_of(const double* part, int parts) {
  double v = 0.0;
  for (int i = threadIdx.x; i < parts; i += GN_THREADS) v += part[i];
  return sqrt(block_sum(v));
}

__global__ __launch_bounds__(GN_THREADS) void grad_norm_kernel(const double* part, int parts, float* norm) {
  const double v = norm_of(part, parts);
  if (threadIdx.x == 0) *norm = (float)v;
}

__global__ __launch_bounds__(GN_THREADS) void grad_scale_kernel(GradSegs s, const double* part, int parts,
                                                                float max_norm, float* norm, int32_t* err) {
  const int t = threadIdx.x;
  const double v = norm_of(part, parts);
  const bool finite = (float)v <= 3.4028235e38f;
  const float c = finite && v > (double)max_norm ? (float)((double)max_norm / v) : 1.f;
  if (norm && blockIdx.x == 0 && t == 0) {
    *norm = (float)v;
    if (!finite && err) atomicOr(err, 1);
  }
  for (int k = blockIdx.x; k < s.chunks; k += gridDim.x) {
    const int i = seg_of(s, k);
    if (c == 1.f && s.out[i] == s.g[i]) continue;
    const int64_t e0 = (int64_t)(k - s.chunk0[i]) * GN_CHUNK;
    const int64_t e1 = min(s.numel[i], e0 + GN_CHUNK);
    for (int64_t e = e0 + t; e < e1; e += GN_THREADS) {
      const float v = load1(s.g[i], s.g_type[i], e) * c;
      if (s.out_type[i] == kF32)
        static_cast<float*>(s.out[i])[e] = v;
      else
        static_cast<uint16_t*>(s.out[i])[e] = f32_to_bf16_any(v);
    }
  }
}

// The next tensors of the list, from i on (empty ones left out).
int64_t take(const GradArgs& a, int64_t i, GradSegs& s) {
  s.n = s.chunks = 0;
  for (; i < a.n && s.n < kSegs; ++i) {
    if (a.numels[i] == 0) continue;
    const int64_t chunks = (a.numels[i] + GN_CHUNK - 1) / GN_CHUNK;
    s.g[s.n] = a.g[i];
    s.out[s.n] = a.clip ? (a.outs ? a.outs[i] : const_cast<void*>(a.g[i])) : nullptr;
    s.numel[s.n] = a.numels[i];
    s.g_type[s.n] = (uint8_t)a.types[i];
    s.out_type[s.n] = (uint8_t)(a.outs ? a.out_types[i] : a.types[i]);
    s.chunk0[s.n] = s.chunks;
    s.chunks += (int)chunks;
    ++s.n;
  }
  return i;
}

}  // namespace

size_t grad_ws_bytes() { return kMaxParts * sizeof(double); }

hipError_t launch_grad_norm(const GradArgs& a, void* ws, hipStream_t stream) {
  double* part = static_cast<double*>(ws);
  const int launches = (int)((a.n + kSegs - 1) / kSegs);
  const int most = kMaxParts / launches < 1024 ? kMaxParts / launches : 1024;
  GradSegs s;
  int parts = 0;
  for (int64_t i = 0; i < a.n;) {
    i = take(a, i, s);
    if (s.chunks == 0) continue;
    const int grid = s.chunks < most ? s.chunks : most;
    hipLaunchKernelGGL(grad_sum_kernel, dim3(grid), dim3(GN_THREADS), 0, stream, s, part + parts);
    parts += grid;
  }
  if (!a.clip || parts == 0) {
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(GN_THREADS), 0, stream, part, parts, a.norm);
    return hipGetLastError();
  }
  bool first = true;
  for (int64_t i = 0; i < a.n;) {
    i = take(a, i, s);
    if (s.chunks == 0) continue;
    const int grid = s.chunks < 2048 ? s.chunks : 2048;
    hipLaunchKernelGGL(grad_scale_kernel, dim3(grid), dim3(GN_THREADS), 0, stream, s, part, parts, a.max_norm,
                       first ? a.norm : nullptr, a.err);
    first = false;
  }
  return hipGetLastError();
}

}  // namespace hydra
