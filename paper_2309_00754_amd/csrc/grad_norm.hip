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
//    the same c), then scales its share.  The shares run backwards, so that the
//    first to be read are what the sums read last and the memory-side cache
//    (256 MB) still holds, and neither these last reads nor the results take
//    its place.  Every adapter of OPT-1.3b at rank 128 (453 MB) in place: 223 us,
//    forwards 235, with the reads through the cache 281, with the results 276;
//    into others 222, 222, 254 and 275; of Llama-7B at rank 16 into bf16 (160 MB,
//    which the cache holds) 70, 66, 72 and 89.  The sums alone run at 5.1 TB/s
//    (those 160 MB) to 5.6 (453 MB).
// Pointers and sizes travel as kernel arguments, 256 runs a launch of the sums
// and 176 of the scaling; tensors that lie side by side, as views of one buffer
// do, are one run.  A workgroup
// takes an equal share of a launch's chunks, one stretch of them: chunks dealt
// in turn, each with its own search for the tensor and its own wait, took the 453
// MB 7% longer.
// Squares are formed and added in 64 bits: an fp32 square of a gradient below
// 1e-19 or above 1e19 would leave the range, and the conversion and the 64-bit
// FMA run beside the loads.
#include "hydra_elem.h"

#include <type_traits>

namespace hydra {
namespace {

constexpr int GN_THREADS = 256;
constexpr int kMaxParts = 2048;  // of all launches of a call
constexpr int kWorkgroups = 1024;  // of a launch at most
constexpr int kLogChunk = 11;    // elements of a chunk

// Tensors side by side in memory, as one.
struct Run {
  const void* g;
  void* out;
  int64_t numel;
  int g_type, out_type;
};

// The runs of a launch.  `last` holds the elements of a run's last chunk less
// one, and above them its two types.
template <int N, bool OUT>
struct GradSegs {
  static constexpr int kMost = N;
  const void* g[N];
  void* out[OUT ? N : 1];
  int chunk0[N + 1];  // first chunk of each run, and the end
  uint16_t last[N];
  int n;
  __device__ __forceinline__ int64_t numel(int i) const {
    return ((int64_t)(chunk0[i + 1] - chunk0[i] - 1) << kLogChunk) + (last[i] & ((1 << kLogChunk) - 1)) + 1;
  }
  __device__ __forceinline__ int g_type(int i) const { return (last[i] >> kLogChunk) & 1; }
  __device__ __forceinline__ int out_type(int i) const { return (last[i] >> (kLogChunk + 1)) & 1; }
  // Run n.
  void add(const Run& r) {
    g[n] = r.g;
    if constexpr (OUT) out[n] = r.out;
    chunk0[n + 1] = chunk0[n] + (int)((r.numel + (int64_t(1) << kLogChunk) - 1) >> kLogChunk);
    last[n] = (uint16_t)(((r.numel - 1) & ((1 << kLogChunk) - 1)) | r.g_type << kLogChunk |
                         r.out_type << (kLogChunk + 1));
  }
  __host__ __device__ int chunks() const { return chunk0[n]; }
};
using SumSegs = GradSegs<256, false>;
using ScaleSegs = GradSegs<176, true>;
static_assert(sizeof(SumSegs) <= 4000 && sizeof(ScaleSegs) <= 4000, "kernel arguments");

// The run that chunk c belongs to: every lane compares the starts of some.
template <class Segs>
__device__ __forceinline__ int seg_of(const Segs& s, int c) {
  const int lane = threadIdx.x & 63;
  int n = 0;
  for (int i = 0; i < s.n; i += 64) n += __popcll(__ballot(i + lane < s.n && s.chunk0[i + lane] <= c));
  return __builtin_amdgcn_readfirstlane(n - 1);
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

// Chunks [c0, c1) of a run of type T: elements [e0, e1), of which the whole groups
// of VEC from b0, a 16-byte boundary of g, on are taken together.
struct Piece {
  int64_t e0, e1, b0, groups;
};
template <int T, int VEC>
__device__ __forceinline__ Piece piece_of(const void* g, int64_t numel, int64_t c0, int64_t c1) {
  constexpr int BYTES = T == kF32 ? 4 : 2;
  const int64_t head = (int64_t)((-reinterpret_cast<uintptr_t>(g)) & 15) / BYTES;  // before the first boundary
  Piece p;
  p.b0 = head + (c0 << kLogChunk);
  p.e0 = c0 == 0 ? 0 : p.b0;
  p.e1 = min(numel, head + (c1 << kLogChunk));
  p.groups = p.e1 > p.b0 ? (p.e1 - p.b0) / VEC : 0;
  return p;
}

// f(run, first chunk, end) for this workgroup's chunks: an equal share of all of
// them, in order (k: which share).
template <class Segs, class F>
__device__ __forceinline__ void each_piece(const Segs& s, int k, F f) {
  const int64_t all = s.chunks();
  int c = (int)(all * k / gridDim.x);
  const int end = (int)(all * (k + 1) / gridDim.x);
  for (int i = seg_of(s, c); c < end; ++i) {
    const int stop = min(end, s.chunk0[i + 1]);
    f(i, (int64_t)(c - s.chunk0[i]), (int64_t)(stop - s.chunk0[i]));
    c = stop;
  }
}

constexpr int GN_U = 8;  // loads of a thread under way

// The elements of a piece that are in no whole group: those before b0 and those
// after the last group, fewer than 16 of each.
template <int VEC, class F>
__device__ __forceinline__ void edges(const Piece& p, F f) {
  const int t = threadIdx.x;
  const int64_t front = min(p.b0, p.e1) - p.e0, back = p.groups > 0 || p.e1 > p.b0 ? p.b0 + p.groups * VEC : p.e1;
  if (t < front) f(p.e0 + t);
  if (t < p.e1 - back) f(back + t);
}

template <int T>
__device__ __forceinline__ void sum_piece(const void* g, int64_t numel, int64_t c0, int64_t c1, double (&sum)[4]) {
  constexpr int VEC = kVec<T>;
  const Piece p = piece_of<T, VEC>(g, numel, c0, c1);
  const uint4* const v = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(g) + p.b0 * (16 / VEC));
  for (int64_t i = threadIdx.x; i < p.groups; i += GN_THREADS * GN_U) {
    uint4 u[GN_U];
#pragma unroll
    for (int q = 0; q < GN_U; ++q) u[q] = i + q * GN_THREADS < p.groups ? v[i + q * GN_THREADS] : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int q = 0; q < GN_U; ++q) {
      float f[VEC];
      unpack<T>(u[q], f);
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum[e & 3] = fma((double)f[e], (double)f[e], sum[e & 3]);
    }
  }
  edges<VEC>(p, [&](int64_t e) {
    const double x = (double)load_elem(g, T, e);
    sum[0] = fma(x, x, sum[0]);
  });
}

__global__ __launch_bounds__(GN_THREADS) void grad_sum_kernel(SumSegs s, double* part) {
  double sum[4] = {0.0, 0.0, 0.0, 0.0};
  each_piece(s, blockIdx.x, [&](int i, int64_t c0, int64_t c1) __attribute__((always_inline)) {
    if (s.g_type(i) == kF32)
      sum_piece<kF32>(s.g[i], s.numel(i), c0, c1, sum);
    else
      sum_piece<kBf16>(s.g[i], s.numel(i), c0, c1, sum);
  });
  const double v = block_sum((sum[0] + sum[1]) + (sum[2] + sum[3]));
  if (threadIdx.x == 0) part[blockIdx.x] = v;
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

// A group is 16 bytes of g, or where the results are wider 16 bytes of them: with
// 32 bytes of results in two stores every adapter of OPT-1.3b at rank 128, bf16
// into fp32, took 249 us, not 145.
template <int TG, int TO>
__device__ __forceinline__ void scale_piece(const void* g, void* out, int64_t numel, int64_t c0, int64_t c1,
                                            float c) {
  constexpr bool WIDER = TG == kBf16 && TO == kF32;
  constexpr int VEC = WIDER ? 4 : kVec<TG>, GB = TG == kF32 ? 4 : 2, OB = TO == kF32 ? 4 : 2;
  using in_t = typename std::conditional<WIDER, u32x2_t, u32x4_t>::type;
  using out_t = typename std::conditional<VEC * OB == 8, u32x2_t, u32x4_t>::type;
  const Piece p = piece_of<TG, VEC>(g, numel, c0, c1);
  if ((reinterpret_cast<uintptr_t>(out) + p.b0 * OB) % sizeof(out_t) != 0) {  // (the same for every chunk of a run)
    for (int64_t e = p.e0 + threadIdx.x; e < p.e1; e += GN_THREADS) store_elem(out, TO, e, load_elem(g, TG, e) * c);
    return;
  }
  const in_t* const v = reinterpret_cast<const in_t*>(static_cast<const uint8_t*>(g) + p.b0 * GB);
  out_t* const o = reinterpret_cast<out_t*>(static_cast<uint8_t*>(out) + p.b0 * OB);
  for (int64_t i = threadIdx.x; i < p.groups; i += GN_THREADS * GN_U) {
    in_t u[GN_U];
#pragma unroll
    for (int q = 0; q < GN_U; ++q)
      u[q] = i + q * GN_THREADS < p.groups ? __builtin_nontemporal_load(v + i + q * GN_THREADS) : in_t{};
#pragma unroll
    for (int q = 0; q < GN_U; ++q) {
      const int64_t k = i + q * GN_THREADS;
      float f[VEC];
      if constexpr (WIDER)
        unpack(u[q], f);
      else
        unpack<TG>(__builtin_bit_cast(uint4, u[q]), f);
      out_t w;
#pragma unroll
      for (int e = 0; e < VEC * OB / 4; ++e) {
        if constexpr (TO == kF32)
          w[e] = __float_as_uint(f[e] * c);
        else
          w[e] = f32_to_bf16_pair(f[2 * e] * c, f[2 * e + 1] * c);
      }
      if (k < p.groups) __builtin_nontemporal_store(w, o + k);
    }
  }
  edges<VEC>(p, [&](int64_t e) { store_elem(out, TO, e, load_elem(g, TG, e) * c); });
}

__global__ __launch_bounds__(GN_THREADS) void grad_scale_kernel(ScaleSegs s, const double* part, int parts,
                                                                float max_norm, float* norm, int32_t* err) {
  const double v = norm_of(part, parts);
  const bool finite = (float)v <= 3.4028235e38f;
  const float c = finite && v > (double)max_norm ? (float)((double)max_norm / v) : 1.f;
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) {
    *norm = (float)v;
    if (!finite && err) atomicOr(err, 1);
  }
  each_piece(s, gridDim.x - 1 - blockIdx.x, [&](int i, int64_t c0, int64_t c1) __attribute__((always_inline)) {
    const void* const g = s.g[i];
    void* const out = s.out[i];
    const int64_t numel = s.numel(i);
    if (c == 1.f && out == g) return;
    if (s.g_type(i) == kF32) {
      if (s.out_type(i) == kF32)
        scale_piece<kF32, kF32>(g, out, numel, c0, c1, c);
      else
        scale_piece<kF32, kBf16>(g, out, numel, c0, c1, c);
    } else {
      if (s.out_type(i) == kF32)
        scale_piece<kBf16, kF32>(g, out, numel, c0, c1, c);
      else
        scale_piece<kBf16, kBf16>(g, out, numel, c0, c1, c);
    }
  });
}

// The list as runs: empty tensors left out, tensors side by side joined.  Kept as
// the runs' first tensors, 8 KB of the caller's stack (the library allocates
// nothing; the runs themselves would be 128 KB).
struct Runs {
  const GradArgs& a;
  int n = 0;
  uint16_t first[kMaxGrads];

  explicit Runs(const GradArgs& args) : a(args) {
    Run p{};
    for (int64_t i = 0; i < a.n; ++i) {
      if (a.numels[i] == 0) continue;
      const Run t = tensor(i);
      if (n > 0 && p.g_type == t.g_type && p.out_type == t.out_type &&
          static_cast<const uint8_t*>(p.g) + p.numel * type_bytes(p.g_type) == t.g &&
          static_cast<uint8_t*>(p.out) + p.numel * type_bytes(p.out_type) == t.out) {
        p.numel += t.numel;
        continue;
      }
      p = t;
      first[n++] = (uint16_t)i;
    }
  }
  Run tensor(int64_t i) const {
    const int gt = a.types[i];
    return Run{a.g[i], a.outs ? a.outs[i] : const_cast<void*>(a.g[i]), a.numels[i], gt, a.outs ? a.out_types[i] : gt};
  }
  Run operator[](int r) const {
    Run p = tensor(first[r]);
    for (int64_t i = first[r] + 1, end = r + 1 < n ? first[r + 1] : a.n; i < end; ++i) p.numel += a.numels[i];
    return p;
  }
};
static_assert(kMaxGrads <= 1 << 16, "tensors by 16-bit numbers");

// The launch's runs, from run `r0` on; returns how many.
template <class Segs>
int fill(Segs& s, const Runs& runs, int r0) {
  s.chunk0[0] = 0;
  for (s.n = 0; s.n < Segs::kMost && r0 + s.n < runs.n; ++s.n) s.add(runs[r0 + s.n]);
  return s.n;
}

}  // namespace

size_t grad_ws_bytes() { return kMaxParts * sizeof(double); }

hipError_t launch_grad_norm(const GradArgs& a, void* ws, hipStream_t stream) {
  double* part = static_cast<double*>(ws);
  const Runs runs(a);
  const int n = runs.n;
  const int sums = (n + SumSegs::kMost - 1) / SumSegs::kMost;
  const int most = sums > 2 ? kMaxParts / sums : kWorkgroups;
  int parts = 0;
  SumSegs s;
  for (int r = 0; r < n;) {
    r += fill(s, runs, r);
    const int grid = s.chunks() < most ? s.chunks() : most;
    hipLaunchKernelGGL(grad_sum_kernel, dim3(grid), dim3(GN_THREADS), 0, stream, s, part + parts);
    parts += grid;
  }
  if (!a.clip || n == 0) {
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(GN_THREADS), 0, stream, part, parts, a.norm);
    return hipGetLastError();
  }
  ScaleSegs o;
  for (int l = (n - 1) / ScaleSegs::kMost; l >= 0; --l) {
    fill(o, runs, l * ScaleSegs::kMost);
    const int grid = o.chunks() < kWorkgroups ? o.chunks() : kWorkgroups;
    hipLaunchKernelGGL(grad_scale_kernel, dim3(grid), dim3(GN_THREADS), 0, stream, o, part, parts, a.max_norm,
                       l == 0 ? a.norm : nullptr, a.err);
  }
  return hipGetLastError();
}

}  // namespace hydra
