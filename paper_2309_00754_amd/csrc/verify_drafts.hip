// Drafted tokens against the target's probabilities, and the token after them
// (speculative sampling, Leviathan, Kalman and Matias 2023; Chen et al. 2023):
// with p = softmax(z / T) and q = softmax(zd / T) at a position, a draft t is
// accepted where u q(t) < p(t); at the first that is not, the next token is drawn
// from max(p - q, 0), after the last from p, by the inverse of the running sum at
// one more u.  The tokens are distributed as the target's own samples.
//
// Exponentials and sums are 64-bit: a sample's place among tens of thousands of
// running sums is lost in 32 bits (their errors, 1e-7 each, against steps of
// 1e-5: one sample in a hundred another token).
//
// Bound: memory for many rows (every logit once), launches for few.
//  * verify_stats_kernel: maximum and sum of exponentials of every segment of
//    every row that a sequence has;
//  * verify_left_kernel: the rows' totals, the acceptances, and what the
//    distribution of the next token has left in every segment;
//  * verify_sample_kernel: the segment in which the sample lies, and its place.
#include "hydra_elem.h"

namespace hydra {
namespace {

constexpr int VT = 256;            // threads
constexpr int kSeg = 4096;         // logits of a segment
constexpr int kPer = kSeg / VT;    // ... of a thread
constexpr int kMaxRows = 2 * kMaxDrafts + 1;

struct Part {   // of one segment of one row
  double sum;   // of e^((z - most) / T)
  float most;   // -inf: masked out whole; NaN: the row holds NaN or +inf
  int pad;
};
struct Decision {  // of one sequence
  double p_sum, q_sum;
  float p_most, q_most;
  int accepted;
  int kind;  // kPlain: from p; kMinus: from max(p - q, 0); kWithout: from p without token; kNone: no distribution
  int token;
  int pad;
};
enum Kind : int { kPlain = 0, kMinus = 1, kWithout = 2, kNone = 3 };

// e^x for x <= 0 to about 1e-14: 2^k P(r), x = k ln 2 + r, |r| <= ln 2 / 2, with
// the exponential series to r^11 / 11! (the rest is below 1e-14).
__device__ __forceinline__ double exp64(double x) {
  x = fmax(x, -800.0);  // (below it e^x is 0 in 64 bits)
  const double k = rint(x * 0x1.71547652b82fep+0);
  double r = fma(-k, 0x1.62e42feep-1, x);  // ln 2 in two parts, the first of 32 bits
  r = fma(-k, 0x1.a39ef35793c76p-33, r);
  double s = 1.0 / 39916800;
  s = fma(s, r, 1.0 / 3628800);
  s = fma(s, r, 1.0 / 362880);
  s = fma(s, r, 1.0 / 40320);
  s = fma(s, r, 1.0 / 5040);
  s = fma(s, r, 1.0 / 720);
  s = fma(s, r, 1.0 / 120);
  s = fma(s, r, 1.0 / 24);
  s = fma(s, r, 1.0 / 6);
  s = fma(s, r, 0.5);
  s = fma(s, r, 1.0);
  s = fma(s, r, 1.0);
  return ldexp(s, (int)k);
}
// e^((z - most) / T) of a logit that is no NaN, 0 for -inf.
__device__ __forceinline__ double weight(float z, float most, double inv_t) {
  return exp64(((double)z - (double)most) * inv_t);
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// Four logits from column c of a row of V, -inf past it.  VEC: 16-byte (bf16:
// 8-byte) loads.
template <int T, bool VEC>
__device__ __forceinline__ void load4(const void* row, int64_t c, int V, float (&f)[4]) {
  if (VEC && c + 4 <= V) {
    if constexpr (T == kF32)
      unpack<kF32>(*reinterpret_cast<const uint4*>(static_cast<const float*>(row) + c), f);
    else
      unpack(*reinterpret_cast<const u32x2_t*>(static_cast<const uint16_t*>(row) + c), f);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = c + i < V ? load_elem(row, T, c + i) : -INFINITY;
  }
}

template <int T>
__device__ __forceinline__ const void* row_of(const void* z, int64_t row, int64_t ld) {
  return static_cast<const char*>(z) + row * ld * (T == kF32 ? 4 : 2);
}

__device__ __forceinline__ int length_of(const VerifyArgs& a, int b) {
  if (!a.lens) return a.k;
  const int n = a.lens[b];
  return n < 0 ? 0 : n > a.k ? a.k : n;
}

template <int T, bool VEC>
__device__ __forceinline__ void stats(const void* row, const VerifyArgs& a, int seg, Part* out) {
  __shared__ float rm[VT / 64];
  __shared__ double rs[VT / 64];
  __shared__ int rb[VT / 64];
  const int t = threadIdx.x;
  float f[kPer];
  float most = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < kPer / 4; ++i) {
    float v[4];
    load4<T, VEC>(row, (int64_t)seg * kSeg + i * (VT * 4) + t * 4, a.V, v);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f[4 * i + j] = v[j];
      most = fmaxf(most, v[j]);
      bad = bad || !(v[j] < INFINITY);
    }
  }
  most = wave_max(most);
  if ((t & 63) == 0) rm[t >> 6] = most;
  const bool any = __any(bad);
  if ((t & 63) == 0) rb[t >> 6] = any;
  __syncthreads();
  most = fmaxf(fmaxf(rm[0], rm[1]), fmaxf(rm[2], rm[3]));
  const bool none = most == -INFINITY, odd = rb[0] || rb[1] || rb[2] || rb[3];
  double sum = 0;
  if (!none && !odd) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) sum += weight(f[i], most, a.inv_t);
  }
  sum = wave_sum64(sum);
  if ((t & 63) == 0) rs[t >> 6] = sum;
  __syncthreads();
  if (t == 0) *out = Part{(rs[0] + rs[1]) + (rs[2] + rs[3]), odd ? __uint_as_float(0x7FC00000u) : most, 0};
}

// Rows [0, n (k + 1)) are the target's, the rest the draft's.
template <int TZ, int TD, bool VEC>
__global__ __launch_bounds__(VT) void verify_stats_kernel(VerifyArgs a, Part* parts, int nseg) {
  const int64_t row = blockIdx.x / nseg;
  const int seg = (int)(blockIdx.x - row * nseg);
  const int64_t nt = (int64_t)a.n * (a.k + 1);
  Part* out = parts + row * nseg + seg;
  if (row < nt) {
    const int b = (int)(row / (a.k + 1)), j = (int)(row - (int64_t)b * (a.k + 1));
    if (j > length_of(a, b)) return;
    stats<TZ, VEC>(row_of<TZ>(a.z, row, a.ld), a, seg, out);
  } else {
    const int64_t d = row - nt;
    const int b = (int)(d / a.k), j = (int)(d - (int64_t)b * a.k);
    if (j >= length_of(a, b)) return;
    stats<TD, VEC>(row_of<TD>(a.zd, d, a.ld_d), a, seg, out);
  }
}

// The weight of a logit in the next token's distribution, relative to p's or (kMinus) as a probability.
__device__ __forceinline__ double left_of(const Decision& d, float z, float zd, int64_t v, double inv_t, double p_inv,
                                          double q_inv) {
  double p = weight(z, d.p_most, inv_t) * p_inv;
  if (d.kind == kMinus) p = fmax(p - weight(zd, d.q_most, inv_t) * q_inv, 0.0);
  if (d.kind == kWithout && v == d.token) p = 0;
  return p;
}

template <int TZ, int TD, bool VEC>
__global__ __launch_bounds__(VT) void verify_left_kernel(VerifyArgs a, const Part* parts, int nseg, Decision* decisions,
                                                         double* left) {
  __shared__ float most[kMaxRows];
  __shared__ double sum[kMaxRows];
  __shared__ int accept[kMaxDrafts];
  __shared__ Decision sd;
  __shared__ double rs[VT / 64];
  const int t = threadIdx.x;
  const int b = blockIdx.x / nseg, seg = blockIdx.x - b * nseg;
  const int len = length_of(a, b);
  const int64_t nt = (int64_t)a.n * (a.k + 1);
  // rows 0 ... len are the target's, then the draft's: 16 lanes each
  const int rows = len + 1 + (a.zd ? len : 0);
  for (int r = t / 16; r < rows; r += VT / 16) {
    const int64_t row = r <= len ? (int64_t)b * (a.k + 1) + r : nt + (int64_t)b * a.k + (r - len - 1);
    const Part* p = parts + row * nseg;
    float m = -INFINITY;
    bool bad = false;
    for (int s = t & 15; s < nseg; s += 16) {
      m = fmaxf(m, p[s].most);
      bad = bad || p[s].most != p[s].most;
    }
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) {
      m = fmaxf(m, __shfl_xor(m, d, 16));
      bad = __shfl_xor((int)bad, d, 16) || bad;
    }
    double v = 0;
    if (m > -INFINITY && !bad)
      for (int s = t & 15; s < nseg; s += 16)
        if (p[s].most > -INFINITY) v += p[s].sum * weight(p[s].most, m, a.inv_t);
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) v += __shfl_xor(v, d, 16);
    if ((t & 15) == 0) {
      most[r] = m;
      sum[r] = bad ? 0.0 : v;  // 0: no distribution
    }
  }
  __syncthreads();
  // 1: accepted, 0: not, 2: no draft that can be one (its token, its row), 3: no distribution of the target
  for (int i = t; i < len; i += VT) {
    const int tok = a.drafts[(int64_t)b * a.k + i];
    int what = 0;
    if (!(sum[i] > 0)) {
      what = 3;
    } else if (tok < 0 || tok >= a.V || (a.zd && !(sum[len + 1 + i] > 0))) {
      what = 2;
    } else {
      const float z = load_elem(row_of<TZ>(a.z, (int64_t)b * (a.k + 1) + i, a.ld), TZ, tok);
      const double p = weight(z, most[i], a.inv_t) / sum[i];
      double q = 1;
      if (a.zd) {
        const float zd = load_elem(row_of<TD>(a.zd, (int64_t)b * a.k + i, a.ld_d), TD, tok);
        q = weight(zd, most[len + 1 + i], a.inv_t) / sum[len + 1 + i];
      }
      what = (double)a.u[(int64_t)b * (a.k + 1) + i] * q < p;
    }
    accept[i] = what;
  }
  __syncthreads();
  if (t == 0) {
    int at = 0;
    while (at < len && accept[at] == 1) ++at;
    Decision d{};
    d.accepted = at;
    d.token = -1;
    d.p_most = most[at];
    d.p_sum = sum[at];
    d.kind = kPlain;
    if (!(sum[at] > 0)) {
      d.kind = kNone;
    } else if (at < len && accept[at] == 0) {
      d.kind = a.zd ? kMinus : kWithout;
      d.token = a.drafts[(int64_t)b * a.k + at];
      if (a.zd) {
        d.q_most = most[len + 1 + at];
        d.q_sum = sum[len + 1 + at];
      }
    }
    sd = d;
    if (seg == 0) {
      decisions[b] = d;
      const bool odd = d.kind == kNone || (at < len && accept[at] == 2) || (a.lens && a.lens[b] != len);
      if (odd && a.err) atomicOr(a.err, 1);
    }
  }
  __syncthreads();
  const Decision d = sd;
  double v = 0;
  if (d.kind != kNone) {
    const void* zr = row_of<TZ>(a.z, (int64_t)b * (a.k + 1) + d.accepted, a.ld);
    const void* dr = d.kind == kMinus ? row_of<TD>(a.zd, (int64_t)b * a.k + d.accepted, a.ld_d) : nullptr;
    const double p_inv = 1.0 / d.p_sum, q_inv = d.kind == kMinus ? 1.0 / d.q_sum : 0.0;
#pragma unroll
    for (int i = 0; i < kPer / 4; ++i) {
      const int64_t c = (int64_t)seg * kSeg + i * (VT * 4) + t * 4;
      float z[4], zd[4] = {0.f, 0.f, 0.f, 0.f};
      load4<TZ, VEC>(zr, c, a.V, z);
      if (dr) load4<TD, VEC>(dr, c, a.V, zd);
#pragma unroll
      for (int j = 0; j < 4; ++j) v += left_of(d, z[j], zd[j], c + j, a.inv_t, p_inv, q_inv);
    }
  }
  v = wave_sum64(v);
  if ((t & 63) == 0) rs[t >> 6] = v;
  __syncthreads();
  if (t == 0) left[(int64_t)b * nseg + seg] = (rs[0] + rs[1]) + (rs[2] + rs[3]);
}

template <int TZ, int TD, bool VEC>
__global__ __launch_bounds__(VT) void verify_sample_kernel(VerifyArgs a, const Part* parts, int nseg,
                                                           const Decision* decisions, const double* left) {
  __shared__ double wsum[VT / 64];
  __shared__ int found, last;
  __shared__ double before;
  __shared__ int sseg;
  __shared__ int skind;
  __shared__ double goal;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int b = blockIdx.x;
  Decision d = decisions[b];
  const int64_t base = (int64_t)b * (a.k + 1);
  // the accepted drafts, their log-probabilities, and what lies past the new token
  for (int j = t; j <= a.k; j += VT) {
    if (j == d.accepted) continue;
    const bool in = j < d.accepted;
    const int tok = in ? a.drafts[(int64_t)b * a.k + j] : -1;
    a.tokens[base + j] = tok;
    if (a.lp) {
      float lp = 0.f;
      if (in) {
        const Part* p = parts + (base + j) * nseg;
        float m = -INFINITY;
        for (int s = 0; s < nseg; ++s) m = fmaxf(m, p[s].most);
        double v = 0;
        for (int s = 0; s < nseg; ++s)
          if (p[s].most > -INFINITY) v += p[s].sum * weight(p[s].most, m, a.inv_t);
        const float z = load_elem(row_of<TZ>(a.z, base + j, a.ld), TZ, tok);
        lp = (float)(((double)z - (double)m) * a.inv_t - log(v));
      }
      a.lp[base + j] = lp;
    }
  }
  if (t == 0) {
    a.accepted[b] = d.accepted;
    if (d.kind == kNone) {
      a.tokens[base + d.accepted] = -1;
      if (a.lp) a.lp[base + d.accepted] = __uint_as_float(0x7FC00000u);
    }
  }
  if (d.kind == kNone) return;
  if (t == 0) {
    // the segment in which the running sum passes u of the total
    const double* l = left + (int64_t)b * nseg;
    double all = 0;
    for (int s = 0; s < nseg; ++s) all += l[s];
    int kind = d.kind;
    const Part* p = parts + (base + d.accepted) * nseg;
    // nothing left (p and q the same but for rounding): from p
    if (!(all > 0)) {
      kind = kPlain;
      all = 0;
      for (int s = 0; s < nseg; ++s)
        if (p[s].most > -INFINITY) all += p[s].sum * weight(p[s].most, d.p_most, a.inv_t) / d.p_sum;
    }
    const double g = (double)a.u[base + a.k] * all;
    double run = 0, at = 0;
    int seg = -1;
    for (int s = 0; s < nseg; ++s) {
      const double v = kind == d.kind ? l[s]
                       : p[s].most > -INFINITY ? p[s].sum * weight(p[s].most, d.p_most, a.inv_t) / d.p_sum : 0.0;
      if (v > 0) {
        seg = s;  // (the last with anything in it, where rounding or u leaves none)
        at = run;
        if (run + v > g) break;
      }
      run += v;
    }
    sseg = seg;
    before = at;
    skind = kind;
    goal = g;
    found = 0x7FFFFFFF;
    last = -1;
  }
  __syncthreads();
  d.kind = skind;
  const void* zr = row_of<TZ>(a.z, base + d.accepted, a.ld);
  const void* dr = d.kind == kMinus ? row_of<TD>(a.zd, (int64_t)b * a.k + d.accepted, a.ld_d) : nullptr;
  const double p_inv = 1.0 / d.p_sum, q_inv = d.kind == kMinus ? 1.0 / d.q_sum : 0.0;
  double run = before;
  const double g = goal;
  for (int i = 0; i < kPer / 4; ++i) {
    const int64_t c = (int64_t)sseg * kSeg + i * (VT * 4) + t * 4;
    float z[4], zd[4] = {0.f, 0.f, 0.f, 0.f};
    load4<TZ, VEC>(zr, c, a.V, z);
    if (dr) load4<TD, VEC>(dr, c, a.V, zd);
    double w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = left_of(d, z[j], zd[j], c + j, a.inv_t, p_inv, q_inv);
    double mine = (w[0] + w[1]) + (w[2] + w[3]), scan = mine;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const double o = __shfl_up(scan, s);
      if (lane >= s) scan += o;
    }
    if (lane == 63) wsum[wave] = scan;
    __syncthreads();
    double to = run + (scan - mine);
    for (int k = 0; k < wave; ++k) to += wsum[k];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      to += w[j];
      if (w[j] > 0) {
        atomicMax(&last, (int)(c + j));
        if (to > g) atomicMin(&found, (int)(c + j));
      }
    }
    run += (wsum[0] + wsum[1]) + (wsum[2] + wsum[3]);
    __syncthreads();
  }
  if (t == 0) {
    const int tok = found != 0x7FFFFFFF ? found : last;
    a.tokens[base + d.accepted] = tok;
    if (a.lp) {
      const float z = load_elem(zr, TZ, tok);
      a.lp[base + d.accepted] = (float)(((double)z - (double)d.p_most) * a.inv_t - log(d.p_sum));
    }
  }
}

size_t up256(size_t v) { return (v + 255) / 256 * 256; }
int segments(int V) { return (V + kSeg - 1) / kSeg; }
size_t part_bytes(const int64_t rows, int V) { return up256((size_t)rows * segments(V) * sizeof(Part)); }

template <int TZ, int TD, bool VEC>
hipError_t launch_all(const VerifyArgs& a, void* ws, hipStream_t stream) {
  const int nseg = segments(a.V);
  const int64_t rows = (int64_t)a.n * (a.k + 1) + (a.zd ? (int64_t)a.n * a.k : 0);
  uint8_t* w = static_cast<uint8_t*>(ws);
  Part* parts = reinterpret_cast<Part*>(w);
  w += part_bytes((int64_t)a.n * (2 * a.k + 1), a.V);
  Decision* decisions = reinterpret_cast<Decision*>(w);
  w += up256((size_t)a.n * sizeof(Decision));
  double* left = reinterpret_cast<double*>(w);
  hipLaunchKernelGGL((verify_stats_kernel<TZ, TD, VEC>), dim3((unsigned)(rows * nseg)), dim3(VT), 0, stream, a, parts, nseg);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((verify_left_kernel<TZ, TD, VEC>), dim3((unsigned)((int64_t)a.n * nseg)), dim3(VT), 0, stream, a, parts,
                     nseg, decisions, left);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL((verify_sample_kernel<TZ, TD, VEC>), dim3(a.n), dim3(VT), 0, stream, a, parts, nseg, decisions, left);
  return hipGetLastError();
}

template <int TZ, int TD>
hipError_t launch_types(const VerifyArgs& a, void* ws, hipStream_t stream) {
  // four logits a load: rows on boundaries of four elements
  const auto whole = [](const void* p, int64_t ld, int type) {
    return (reinterpret_cast<uintptr_t>(p) & (type == kF32 ? 15 : 7)) == 0 && ld % 4 == 0;
  };
  const bool vec = whole(a.z, a.ld, TZ) && (!a.zd || whole(a.zd, a.ld_d, TD));
  return vec ? launch_all<TZ, TD, true>(a, ws, stream) : launch_all<TZ, TD, false>(a, ws, stream);
}

}  // namespace

size_t verify_ws_bytes(int n, int k, int V) {
  return part_bytes((int64_t)n * (2 * k + 1), V) + up256((size_t)n * sizeof(Decision)) +
         up256((size_t)n * segments(V) * sizeof(double));
}

hipError_t launch_verify(const VerifyArgs& a, void* ws, hipStream_t stream) {
  if (a.z_type == kF32)
    return a.d_type == kF32 ? launch_types<kF32, kF32>(a, ws, stream) : launch_types<kF32, kBf16>(a, ws, stream);
  return a.d_type == kF32 ? launch_types<kBf16, kF32>(a, ws, stream) : launch_types<kBf16, kBf16>(a, ws, stream);
}

}  // namespace hydra
