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
// Bound: vector instructions for many rows (64 sequences of up to 7: 35 for each logit of the
// sums, the tables below among them, which keep the vector units busy for 24 of that launch's 33
// us; its logits are 16 us of memory), launches for few.
//  * verify_stats_kernel: maximum and sum of exponentials of every segment of
//    every row that a sequence has;
//  * verify_left_kernel: the rows' totals, the acceptances (every workgroup of a
//    sequence forms them itself), the accepted tokens, and what the distribution of
//    the next token has in every segment;
//  * verify_sample_kernel: the segment in which the sample lies, and its place.
// 1 sequence of 5 drafts, V 32000, 16 us: three launches of dependent steps; 64 of up to 7,
// V 50272, 52 us: some 30 of them for the sums over 26 million logits.
#include "hydra_elem.h"

namespace hydra {
namespace {

constexpr int VT = 256;            // threads
// Logits of a segment.  us with 4096, 2048 and 1024, target fp32, draft bf16: 1 sequence of 4
// drafts, V 32000, 19.5, 15.2, 14.0 (the exponentials of a segment are one CU's); 64 of
// 7, V 50272, 69.1, 71.4, 93.9 (the maxima's and sums' exchange is a workgroup's).
constexpr int kSeg = 2048;
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

// e^((z - most) / T) for z <= most: with y = (z - most) 64 / (T ln 2) = k + f, k whole and
// |f| <= 1/2, it is 2^(k / 64) e^(f ln 2 / 64): 2^(j / 64) from a table (put_table), the
// exponential series to its fourth power (the rest is below 4e-14).  Eleven 64-bit
// operations and four others; the series alone, to x^11, took twenty and nine.
constexpr int kTable = 64;
__device__ __forceinline__ void put_table(double* table) {
  if (threadIdx.x < kTable) table[threadIdx.x] = exp2(threadIdx.x * (1.0 / kTable));
}
// 64 / (T ln 2)
__device__ __forceinline__ double scale_of(double inv_t) { return inv_t * 0x1.71547652b82fep+6; }
constexpr double kFloor = -700 * 0x1.71547652b82fep+6;  // y of e^-700
__device__ __forceinline__ double power_of(double y, const double* table) {
  constexpr double L = 0x1.62e42fefa39efp-7, big = 0x1.8p52;  // ln 2 / 64; a sum whose last place is 1
  const double t = y + big, f = y - (t - big);
  double v = fma(L * L * L * L / 24, f, L * L * L / 6);
  v = fma(v, f, L * L / 2);
  v = fma(v, f, L);
  v = fma(v, f, 1.0);
  const int k = (int)__double2loint(t);
  return ldexp(v * table[k & (kTable - 1)], k >> 6);
}
// For sums: what is below e^-700, -inf too, is e^-700.
__device__ __forceinline__ double weight_in_sum(float z, float most, double scale, const double* table) {
  return power_of(fmax(((double)z - (double)most) * scale, kFloor), table);
}
// ... is 0; z is no NaN.
__device__ __forceinline__ double weight(float z, float most, double scale, const double* table) {
  const double y = ((double)z - (double)most) * scale, v = power_of(fmax(y, kFloor), table);
  return y <= kFloor ? 0.0 : v;
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
__device__ __forceinline__ void stats(const void* row, const VerifyArgs& a, int seg, Part* out, double* table) {
  __shared__ float rm[VT / 64];
  __shared__ double rs[VT / 64];
  __shared__ int rb[VT / 64];
  const int t = threadIdx.x;
  put_table(table);
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
  const bool any = __any(bad);
  if ((t & 63) == 0) {
    rm[t >> 6] = most;
    rb[t >> 6] = any;
  }
  __syncthreads();
  most = fmaxf(fmaxf(rm[0], rm[1]), fmaxf(rm[2], rm[3]));
  const bool none = most == -INFINITY, odd = rb[0] || rb[1] || rb[2] || rb[3];
  double sum = 0;
  if (!none && !odd) {
    const double sc = scale_of(a.inv_t);
#pragma unroll
    for (int i = 0; i < kPer; ++i) sum += weight_in_sum(f[i], most, sc, table);
  }
  sum = wave_sum64(sum);
  if ((t & 63) == 0) rs[t >> 6] = sum;
  __syncthreads();
  if (t == 0) *out = Part{(rs[0] + rs[1]) + (rs[2] + rs[3]), odd ? __uint_as_float(0x7FC00000u) : most, 0};
}

// Rows [0, n (k + 1)) are the target's, the rest the draft's.
template <int TZ, int TD, bool VEC>
__global__ __launch_bounds__(VT) void verify_stats_kernel(VerifyArgs a, Part* parts, int nseg) {
  __shared__ double table[kTable];
  const int64_t row = blockIdx.x / nseg;
  const int seg = (int)(blockIdx.x - row * nseg);
  const int64_t nt = (int64_t)a.n * (a.k + 1);
  Part* out = parts + row * nseg + seg;
  if (row < nt) {
    const int b = (int)(row / (a.k + 1)), j = (int)(row - (int64_t)b * (a.k + 1));
    if (j > length_of(a, b)) return;
    stats<TZ, VEC>(row_of<TZ>(a.z, row, a.ld), a, seg, out, table);
  } else {
    const int64_t d = row - nt;
    const int b = (int)(d / a.k), j = (int)(d - (int64_t)b * a.k);
    if (j >= length_of(a, b)) return;
    stats<TD, VEC>(row_of<TD>(a.zd, d, a.ld_d), a, seg, out, table);
  }
}

// What a logit has in the next token's distribution, as a probability.
__device__ __forceinline__ double left_of(const Decision& d, float z, float zd, int64_t v, double sc,
                                          double p_inv, double q_inv, const double* table) {
  double p = weight(z, d.p_most, sc, table) * p_inv;
  if (d.kind == kMinus) p = fmax(p - weight(zd, d.q_most, sc, table) * q_inv, 0.0);
  if (d.kind == kWithout && v == d.token) p = 0;
  return p;
}

// ... and of a thread's logits of a segment, four at a time.
template <int TZ, int TD, bool VEC>
__device__ __forceinline__ void left_in(const VerifyArgs& a, const Decision& d, int b, int seg, const double* table,
                                        double (&w)[kPer]) {
  const void* zr = row_of<TZ>(a.z, (int64_t)b * (a.k + 1) + d.accepted, a.ld);
  const bool minus = d.kind == kMinus;
  const void* dr = minus ? row_of<TD>(a.zd, (int64_t)b * a.k + d.accepted, a.ld_d) : nullptr;
  const double p_inv = 1.0 / d.p_sum, q_inv = minus ? 1.0 / d.q_sum : 0.0;
  const double sc = scale_of(a.inv_t);
  float z[kPer / 4][4], zd[kPer / 4][4];
#pragma unroll
  for (int i = 0; i < kPer / 4; ++i) {
    const int64_t c = (int64_t)seg * kSeg + i * (VT * 4) + threadIdx.x * 4;
    load4<TZ, VEC>(zr, c, a.V, z[i]);
    if (minus) load4<TD, VEC>(dr, c, a.V, zd[i]);
  }
#pragma unroll
  for (int i = 0; i < kPer / 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t c = (int64_t)seg * kSeg + i * (VT * 4) + threadIdx.x * 4 + j;
      w[4 * i + j] = left_of(d, z[i][j], zd[i][j], c, sc, p_inv, q_inv, table);
    }
}

template <int TZ, int TD, bool VEC>
__global__ __launch_bounds__(VT) void verify_left_kernel(VerifyArgs a, const Part* parts, int nseg, Decision* decisions,
                                                         double* left) {
  __shared__ double table[kTable];
  __shared__ float most[kMaxRows];
  __shared__ double sum[kMaxRows];
  __shared__ int accept[kMaxDrafts];
  __shared__ int stop;
  __shared__ double rs[VT / 64];
  const int t = threadIdx.x;
  const int b = blockIdx.x / nseg, seg = blockIdx.x - b * nseg;
  const int len = length_of(a, b);
  const int64_t nt = (int64_t)a.n * (a.k + 1), base = (int64_t)b * (a.k + 1);
  put_table(table);
  const double sc = scale_of(a.inv_t);
  // a thread's own draft (k <= VT) and its logits, requested ahead
  static_assert(kMaxDrafts <= VT, "a draft a thread");
  int tok = -1;
  float z = 0.f, zd = 0.f, u = 0.f;
  if (t < len) {
    tok = a.drafts[(int64_t)b * a.k + t];
    u = a.u[base + t];
    if (tok >= 0 && tok < a.V) {
      z = load_elem(row_of<TZ>(a.z, base + t, a.ld), TZ, tok);
      if (a.zd) zd = load_elem(row_of<TD>(a.zd, (int64_t)b * a.k + t, a.ld_d), TD, tok);
    }
  }
  __syncthreads();
  // rows 0 ... len are the target's, then the draft's: 16 lanes each
  const int rows = len + 1 + (a.zd ? len : 0);
  for (int r = t / 16; r < rows; r += VT / 16) {
    const int64_t row = r <= len ? base + r : nt + (int64_t)b * a.k + (r - len - 1);
    const Part* p = parts + row * nseg;
    float m = -INFINITY;
    double v = 0;
    bool bad = false;
    for (int s = t & 15; s < nseg; s += 16) {
      const Part q = p[s];
      bad = bad || q.most != q.most;
      const float to = fmaxf(m, q.most);
      if (to > -INFINITY && q.most == q.most)
        v = (m > -INFINITY ? v * weight(m, to, sc, table) : 0.0) +
            (q.most > -INFINITY ? q.sum * weight(q.most, to, sc, table) : 0.0);
      m = to;
    }
    float all = m;
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) {
      all = fmaxf(all, __shfl_xor(all, d, 16));
      bad = __shfl_xor((int)bad, d, 16) || bad;
    }
    v = m > -INFINITY ? v * weight(m, all, sc, table) : 0.0;
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) v += __shfl_xor(v, d, 16);
    if ((t & 15) == 0) {
      most[r] = all;
      sum[r] = bad ? 0.0 : v;  // 0: no distribution
    }
  }
  __syncthreads();
  // 1: accepted, 0: not, 2: no draft that can be one (its token, its row), 3: no distribution of the target
  double at_z = 0;  // ln p + ln sum of the draft
  if (t < len) {
    int what = 0;
    if (!(sum[t] > 0)) {
      what = 3;
    } else if (tok < 0 || tok >= a.V || (a.zd && !(sum[len + 1 + t] > 0))) {
      what = 2;
    } else {
      at_z = ((double)z - (double)most[t]) * a.inv_t;
      const double p = weight(z, most[t], sc, table) / sum[t];
      const double q = a.zd ? weight(zd, most[len + 1 + t], sc, table) / sum[len + 1 + t] : 1.0;
      what = (double)u * q < p;
    }
    accept[t] = what;
  }
  __syncthreads();
  if (t < 64) {  // the first that is not accepted
    int first = len;
    for (int i = t; i < len; i += 64)
      if (accept[i] != 1 && i < first) first = i;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) first = min(first, __shfl_xor(first, d));
    if (t == 0) stop = first;
  }
  __syncthreads();
  Decision d{};
  d.accepted = stop;
  d.token = -1;
  d.p_most = most[stop];
  d.p_sum = sum[stop];
  d.kind = !(d.p_sum > 0) ? kNone : kPlain;
  const int what = stop < len ? accept[stop] : 1;
  if (d.kind != kNone && what == 0) {
    d.kind = a.zd ? kMinus : kWithout;
    d.token = a.drafts[(int64_t)b * a.k + stop];
    if (a.zd) {
      d.q_most = most[len + 1 + stop];
      d.q_sum = sum[len + 1 + stop];
    }
  }
  if (seg == 0) {
    if (t == 0) {
      decisions[b] = d;
      a.accepted[b] = stop;
      if (a.err && (d.kind == kNone || what == 2 || (a.lens && a.lens[b] != len))) atomicOr(a.err, 1);
    }
    // the accepted drafts and what lies past the next token (and that one, where it has no distribution)
    if (t <= a.k && (t != stop || d.kind == kNone)) {
      a.tokens[base + t] = t < stop ? tok : -1;
      if (a.lp) a.lp[base + t] = t < stop ? (float)(at_z - log(sum[t])) : t == stop ? __uint_as_float(0x7FC00000u) : 0.f;
    }
  }
  double v = 0;
  if (d.kind != kNone) {
    double w[kPer];
    left_in<TZ, TD, VEC>(a, d, b, seg, table, w);
#pragma unroll
    for (int i = 0; i < kPer; ++i) v += w[i];
  }
  v = wave_sum64(v);
  if ((t & 63) == 0) rs[t >> 6] = v;
  __syncthreads();
  if (t == 0) left[(int64_t)b * nseg + seg] = (rs[0] + rs[1]) + (rs[2] + rs[3]);
}

__device__ __forceinline__ double wave_scan64(double v, int lane) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const double o = __shfl_up(v, s);
    if (lane >= s) v += o;
  }
  return v;
}

template <int TZ, int TD, bool VEC>
__global__ __launch_bounds__(VT) void verify_sample_kernel(VerifyArgs a, const Part* parts, int nseg,
                                                           const Decision* decisions, const double* left) {
  constexpr int R = kPer / 4;  // rounds of four logits a thread
  __shared__ double table[kTable];
  __shared__ double wsum[R][VT / 64];
  __shared__ int wfirst[VT / 64], wlast[VT / 64];
  __shared__ double before, goal;
  __shared__ int sseg, skind;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int b = blockIdx.x;
  Decision d = decisions[b];
  const int64_t base = (int64_t)b * (a.k + 1);
  if (d.kind == kNone) return;
  const double u = a.u[base + a.k], sc = scale_of(a.inv_t);
  put_table(table);
  __syncthreads();
  if (wave == 0) {
    // the segment in which the running sum passes u of the total
    const double* l = left + (int64_t)b * nseg;
    const Part* p = parts + (base + d.accepted) * nseg;
    int kind = d.kind;
    const auto mass = [&](int s) {
      if (s >= nseg) return 0.0;
      if (kind == d.kind) return l[s];
      return p[s].most > -INFINITY ? p[s].sum * weight(p[s].most, d.p_most, sc, table) / d.p_sum : 0.0;
    };
    double all = 0;
    for (int s0 = 0; s0 < nseg; s0 += 64) all += wave_sum64(mass(s0 + lane));
    if (!(all > 0)) {  // nothing left (p and q the same but for rounding): from p
      kind = kPlain;
      all = 0;
      for (int s0 = 0; s0 < nseg; s0 += 64) all += wave_sum64(mass(s0 + lane));
    }
    const double g = u * all;
    double run = 0, at = 0;
    int seg = -1;
    for (int s0 = 0; s0 < nseg; s0 += 64) {
      const double v = mass(s0 + lane), to = run + wave_scan64(v, lane);
      const uint64_t some = __ballot(v > 0), past = __ballot(v > 0 && to > g);
      if (some) {  // the first that passes, or the last with anything in it, where rounding or u leaves none
        const int src = past ? __ffsll((unsigned long long)past) - 1 : 63 - __clzll((long long)some);
        seg = s0 + src;
        at = __shfl(to - v, src);
      }
      if (past) break;
      run = __shfl(to, 63);
    }
    if (lane == 0) {
      sseg = seg;
      before = at;
      goal = g;
      skind = kind;
    }
  }
  __syncthreads();
  d.kind = skind;
  const int seg = sseg;
  const double g = goal;
  double w[kPer], scan[R];
  left_in<TZ, TD, VEC>(a, d, b, seg, table, w);
#pragma unroll
  for (int i = 0; i < R; ++i) {
    scan[i] = wave_scan64((w[4 * i] + w[4 * i + 1]) + (w[4 * i + 2] + w[4 * i + 3]), lane);
    if (lane == 63) wsum[i][wave] = scan[i];
  }
  __syncthreads();
  int first = 0x7FFFFFFF, last = -1;
  double run = before;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    double to = run + (scan[i] - ((w[4 * i] + w[4 * i + 1]) + (w[4 * i + 2] + w[4 * i + 3])));
#pragma unroll
    for (int k = 0; k < VT / 64; ++k) {
      if (k < wave) to += wsum[i][k];
      run += wsum[i][k];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = seg * kSeg + i * (VT * 4) + t * 4 + j;
      to += w[4 * i + j];
      if (w[4 * i + j] > 0) {
        last = c;
        if (to > g && c < first) first = c;
      }
    }
  }
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) {
    first = min(first, __shfl_xor(first, s));
    last = max(last, __shfl_xor(last, s));
  }
  if (lane == 0) {
    wfirst[wave] = first;
    wlast[wave] = last;
  }
  __syncthreads();
  if (t == 0) {
    first = min(min(wfirst[0], wfirst[1]), min(wfirst[2], wfirst[3]));
    last = max(max(wlast[0], wlast[1]), max(wlast[2], wlast[3]));
    const int tok = first != 0x7FFFFFFF ? first : last;
    a.tokens[base + d.accepted] = tok;
    if (a.lp) {
      const float z = load_elem(row_of<TZ>(a.z, base + d.accepted, a.ld), TZ, tok);
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
  hipLaunchKernelGGL((verify_sample_kernel<TZ, TD, VEC>), dim3(a.n), dim3(VT), 0, stream, a, parts, nseg, decisions,
                     left);
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
