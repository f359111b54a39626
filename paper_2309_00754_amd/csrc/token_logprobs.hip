// Log-probabilities of given tokens over materialised logits, the entropy and
// the most likely alternatives, and their gradient with respect to the logits,
// for gfx950 (Sec. 2 Stage 3: the policy ratio's log-probabilities and what the
// update takes back through the CLM head).
//
//   lse = m + ln S, S = sum_j e^(z_j - m), m = max z
//   H = ln S - W / S,  W = sum_j e^(z_j - m) (z_j - m)
//   dz_j = d_lp ([j == token] - p_j) - d_H p_j (ln p_j + H), p_j = e^(z_j - lse)
//
//  * token_logp_kernel: one workgroup per row keeps a running (m, S, W) per
//    thread and joins them in a fixed tree; the alternatives are extracted one
//    after the other, each by a maximum over the workgroup.
//  * token_logp_back_kernel: a workgroup per row; a row without a gradient is
//    filled with zeros unread.
#include "hydra_device.h"
#include "hydra_internal.h"

namespace hydra {
namespace {

constexpr int TL_THREADS = 512;
constexpr int TL_WAVES = TL_THREADS / 64;

__device__ __forceinline__ float load_z(const void* p, int type, size_t i) {
  return type == kF32 ? static_cast<const float*>(p)[i] : bf16_to_f32(static_cast<const uint16_t*>(p)[i]);
}

// A whole number that orders logits by value, then by index (the lower one the
// greater): NaN first, then +inf.  +0 and -0 are one value.
__device__ __forceinline__ uint64_t order_key(float z, int idx) {
  const uint32_t u = __float_as_uint(z + 0.f);
  const uint32_t o = z != z ? 0xFFFFFFFEu : (int)u < 0 ? ~u : u | 0x80000000u;
  return ((uint64_t)o << 32) | (uint32_t)~idx;
}

// The statistics of a part of a row.  Differences to the maximum are formed
// before anything else is done with them, so that logits up to the type's
// largest and lowest values (masks) keep their meaning.
struct Stat {
  float m, s, w;  // max z, sum e^(z - m), sum e^(z - m) (z - m)
};

constexpr float kFar = -1000.f;  // e^kFar is 0, and a product of the two is (with -inf it would not be)

__device__ __forceinline__ void rescale(Stat& a, float m) {
  // (nothing so far: s = w = 0; and a NaN sum stays one)
  if (a.m != -INFINITY && a.m != m) {
    const float d = a.m - m, e = exp_e(d);
    a.w = fmaf(a.s, fmaxf(d, kFar), a.w) * e;
    a.s *= e;
  }
  a.m = m;
}

__device__ __forceinline__ void absorb(Stat& a, float z) {
  rescale(a, fmaxf(a.m, z));
  if (z == -INFINITY) return;
  const float d = z - a.m, e = exp_e(d);
  a.s += e;
  a.w = fmaf(e, fmaxf(d, kFar), a.w);
}

__device__ __forceinline__ Stat block_stat(Stat a) {
  __shared__ float red[3][TL_WAVES];
  const int t = threadIdx.x;
  float m = a.m;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  if ((t & 63) == 0) red[0][t >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < TL_WAVES; ++i) m = fmaxf(m, red[0][i]);
  rescale(a, m);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    a.s += __shfl_xor(a.s, o);
    a.w += __shfl_xor(a.w, o);
  }
  if ((t & 63) == 0) {
    red[1][t >> 6] = a.s;
    red[2][t >> 6] = a.w;
  }
  __syncthreads();
  a.s = red[1][0];
  a.w = red[2][0];
#pragma unroll
  for (int i = 1; i < TL_WAVES; ++i) {
    a.s += red[1][i];
    a.w += red[2][i];
  }
  return a;
}

__device__ __forceinline__ uint64_t block_max(uint64_t v) {
  __shared__ uint64_t red[TL_WAVES];
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    const uint64_t u = __shfl_xor((unsigned long long)v, o);
    v = u > v ? u : v;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int i = 1; i < TL_WAVES; ++i) v = red[i] > v ? red[i] : v;
  return v;
}

// lp of a logit, by way of the maximum: of the rounding of lse that of ln S
// alone remains.
__device__ __forceinline__ float logp_of(float z, const Stat& a, float ln_s) { return (z - a.m) - ln_s; }

__global__ __launch_bounds__(TL_THREADS) void token_logp_kernel(TokenLogpArgs a) {
  const int row = blockIdx.x, t = threadIdx.x, V = a.V;
  const size_t r0 = (size_t)row * a.ld;
  Stat st{-INFINITY, 0.f, 0.f};
  for (int j = t; j < V; j += TL_THREADS) absorb(st, load_z(a.z, a.type, r0 + j));
  st = block_stat(st);
  const float ln_s = log_e(st.s);
  if (t == 0) {
    if (a.lse) a.lse[row] = st.m + ln_s;
    if (a.entropy) a.entropy[row] = ln_s - st.w / st.s;
    if (a.lp) {
      const int tk = a.tokens[row];
      const bool ok = tk >= 0 && tk < V;
      a.lp[row] = ok ? logp_of(load_z(a.z, a.type, r0 + tk), st, ln_s) : __builtin_nanf("");
      if (!ok && a.err) atomicOr(a.err, 1);
    }
  }
  uint64_t last = ~0ull;
  for (int r = 0; r < a.top; ++r) {
    uint64_t best = 0;
    for (int j = t; j < V; j += TL_THREADS) {
      const uint64_t k = order_key(load_z(a.z, a.type, r0 + j), j);
      best = k < last && k > best ? k : best;
    }
    last = block_max(best);
    if (t == 0) {
      const int id = (int)~(uint32_t)last;
      a.ids[(size_t)row * a.top + r] = id;
      if (a.top_lp) a.top_lp[(size_t)row * a.top + r] = logp_of(load_z(a.z, a.type, r0 + id), st, ln_s);
    }
  }
}

__global__ __launch_bounds__(TL_THREADS) void token_logp_back_kernel(TokenLogpBackArgs a) {
  const int row = blockIdx.x, t = threadIdx.x, V = a.V;
  const size_t r0 = (size_t)row * a.ld, d0 = (size_t)row * a.ld_d;
  const float d_lp = a.d_lp ? a.d_lp[row] : 0.f, d_h = a.d_entropy ? a.d_entropy[row] : 0.f;
  const bool live = d_lp != 0.f || d_h != 0.f;
  int tk = -1;
  float lse = 0.f, h = 0.f, scale = 1.f;
  if (live) {
    lse = a.lse[row];
    h = d_h != 0.f ? a.entropy[row] : 0.f;
    if (d_lp != 0.f) {
      tk = a.tokens[row];
      if (tk < 0 || tk >= V) {
        scale = __builtin_nanf("");
        if (t == 0 && a.err) atomicOr(a.err, 1);
      }
    }
  }
  for (int j = t; j < V; j += TL_THREADS) {
    float d = 0.f;
    if (live) {
      const float lp = load_z(a.z, a.type, r0 + j) - lse, p = exp_e(lp);
      // (p = 0 where lp is -inf)
      d = scale * fmaf(-p, fmaf(d_h, fmaxf(lp, kFar) + h, d_lp), j == tk ? d_lp : 0.f);
    }
    if (a.d_type == kF32)
      static_cast<float*>(a.dz)[d0 + j] = d;
    else
      static_cast<uint16_t*>(a.dz)[d0 + j] = f32_to_bf16_any(d);
  }
}

}  // namespace

size_t token_logp_ws_bytes(int, int, int) { return 0; }

hipError_t launch_token_logp(const TokenLogpArgs& a, void*, hipStream_t stream) {
  hipLaunchKernelGGL(token_logp_kernel, dim3(a.M), dim3(TL_THREADS), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_token_logp_back(const TokenLogpBackArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(token_logp_back_kernel, dim3(a.M), dim3(TL_THREADS), 0, stream, a);
  return hipGetLastError();
}

}  // namespace hydra
