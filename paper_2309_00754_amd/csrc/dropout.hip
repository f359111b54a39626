// Dropout whose mask is never stored: whether an element is kept follows from
// its index, a seed and an offset by a counter-based generator, so the backward
// makes the same mask again:
//   y = residual + m x,  m = 65536 / (65536 - drop) where the element's sixteen
//   random bits are `drop` or more, else 0.
//
// A thread takes one block of the generator: eight elements.
// Bound: memory, with the generator's twenty 32 x 32 -> 64 bit products a block
// close behind.  4096 x 2048 fp32 onto fp32 17.8 us (5.7 TB/s read and written), 2048 x
// 4096 bf16 6.3 us (5.3 TB/s).
#include "hydra_elem.h"
#include "hydra_philox.h"

namespace hydra {
namespace {

constexpr int DT = 256;

template <int T>
__device__ __forceinline__ void load8(const void* p, size_t i, float (&f)[8]) {
  if constexpr (T == kF32) {
    const uint4* q = reinterpret_cast<const uint4*>(static_cast<const float*>(p) + i);
    float a[4], b[4];
    unpack<kF32>(q[0], a);
    unpack<kF32>(q[1], b);
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = a[j], f[4 + j] = b[j];
  } else {
    unpack<kBf16>(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i), f);
  }
}

// R: the residual's type, -1: none.
template <int X, int R, int Y>
__global__ __launch_bounds__(DT) void dropout_kernel(DropoutArgs a) {
  const size_t group = (size_t)blockIdx.x * DT + threadIdx.x, i = group * 8;
  if (i + 8 > (size_t)a.n) return;
  float x[8], r[8];
  load8<X>(a.x, i, x);
  if constexpr (R >= 0) load8<R>(a.res, i, r);
  const uint4 w = dropout_words(a.rng[0], a.rng[1], group);
  float y[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float v = dropout_keeps(w, j, a.drop) ? x[j] * a.keep : 0.f;
    y[j] = R >= 0 ? v + r[j] : v;
  }
  if constexpr (Y == kF32) {
    f32x4_t* o = reinterpret_cast<f32x4_t*>(static_cast<float*>(a.y) + i);
    o[0] = f32x4_t{y[0], y[1], y[2], y[3]};
    o[1] = f32x4_t{y[4], y[5], y[6], y[7]};
  } else {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.y) + i) =
        make_uint4(f32_to_bf16_pair(y[0], y[1]), f32_to_bf16_pair(y[2], y[3]), f32_to_bf16_pair(y[4], y[5]),
                   f32_to_bf16_pair(y[6], y[7]));
  }
}

// Element by element from group `from` on: buffers off their 16-byte boundaries,
// and the last, partial block.
__global__ __launch_bounds__(DT) void dropout_any_kernel(DropoutArgs a, size_t from) {
  const size_t group = from + (size_t)blockIdx.x * DT + threadIdx.x;
  const size_t n = (size_t)a.n;
  if (group * 8 >= n) return;
  const uint4 w = dropout_words(a.rng[0], a.rng[1], group);
  for (int j = 0; j < 8; ++j) {
    const size_t i = group * 8 + j;
    if (i >= n) return;
    float v = dropout_keeps(w, j, a.drop) ? load_elem(a.x, a.x_type, i) * a.keep : 0.f;
    if (a.res) v += load_elem(a.res, a.res_type, i);
    store_elem(a.y, a.y_type, i, v);
  }
}

template <int X, int R>
void launch_xr(const DropoutArgs& a, dim3 grid, hipStream_t stream) {
  if (a.y_type == kF32)
    hipLaunchKernelGGL((dropout_kernel<X, R, kF32>), grid, dim3(DT), 0, stream, a);
  else
    hipLaunchKernelGGL((dropout_kernel<X, R, kBf16>), grid, dim3(DT), 0, stream, a);
}

template <int X>
void launch_x(const DropoutArgs& a, dim3 grid, hipStream_t stream) {
  if (!a.res)
    launch_xr<X, -1>(a, grid, stream);
  else if (a.res_type == kF32)
    launch_xr<X, kF32>(a, grid, stream);
  else
    launch_xr<X, kBf16>(a, grid, stream);
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t stream) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.res) | reinterpret_cast<uintptr_t>(a.y);
  const size_t whole = (at & 15) == 0 ? (size_t)a.n / 8 : 0, all = ((size_t)a.n + 7) / 8;
  if (whole > 0) {
    const dim3 grid((unsigned)((whole + DT - 1) / DT));
    a.x_type == kF32 ? launch_x<kF32>(a, grid, stream) : launch_x<kBf16>(a, grid, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (all > whole) {
    hipLaunchKernelGGL(dropout_any_kernel, dim3((unsigned)((all - whole + DT - 1) / DT)), dim3(DT), 0, stream, a, whole);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace hydra
