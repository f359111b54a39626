// Log-probabilities of given tokens over materialised logits, the entropy and
// the most likely alternatives, and their gradient with respect to the logits,
// for gfx950 (Sec. 2 Stage 3: the policy ratio's log-probabilities and what the
// update takes back through the CLM head).
//
//   lse = m + ln S, S = sum_j e^(z_j - m), m = max z
//   H = ln S - W / S,  W = sum_j e^(z_j - m) (z_j - m)
//   dz_j = d_lp ([j == token] - p_j) - d_H p_j (ln p_j + H), p_j = e^(z_j - lse)
//
//  * token_logp_kernel: a workgroup of 128 to 512 threads per row, or per segment
//    of a long one, reads it once in 16-byte groups, each thread with running sums
//    relative to a power of two that follows its maximum; the threads meet in a
//    fixed tree.  For the alternatives it keeps the maximum of every group in LDS.
//  * token_logp_join_kernel: one wave per row joins the segments.
//  * token_logp_back_kernel: a workgroup per stretch of a row; rows without a
//    gradient are filled with zeros unread.
//
// The k largest of a row: every wave finds the j-th largest of its threads'
// maxima, j = k over the waves, or a number between it and the next; the smallest
// of these is a bound that at least k logits reach.  The groups whose maximum
// reaches it are read again (from the cache), and what reaches it there, some tens
// of logits, is ranked by counting.
// Ties, masks of one value and sorted rows can leave too many for that.  Then
// the k greatest groups by (maximum, lower index) are found exactly, by their
// maxima's bits from the highest down: they hold the k largest logits, since any
// logit in another group has one in each of these before it.  (32000 zeros or
// sorted logits, 32 alternatives, one row: extracting them one after the other
// took 335 us.)
#include "hydra_elem.h"

#include <type_traits>

namespace hydra {
namespace {

// 16-byte loads of a thread under way: 900 x 40000 fp32 with 16 alternatives 33.2
// us (2: 38.3; 8: 31.6), 1500 x 50272 bf16 with 8 alternatives 34.4 (2: 37.3; 8: 38.6).
constexpr int TL_U = 4;
constexpr int kSegMost = 57344;     // elements of a segment (its groups' maxima, 4 bytes each, beside 7 KB in 64 KB of LDS)
constexpr int kSegs = 64;           // segments of a row at most
constexpr int kCand = 576;          // logits ranked by counting at most

template <int T>
__device__ __forceinline__ float load_z(const void* p, size_t i) {
  return load_elem(p, T, i);
}

// Elements before the first 16-byte boundary of a row.
template <int T>
__device__ __forceinline__ int head_of(const void* row, int V) {
  return min(V, (int)((-reinterpret_cast<uintptr_t>(row)) & 15) / (16 / kVec<T>));
}

// A whole number that orders logits by value, then by index (the lower one the
// greater): NaN first, then +inf.  +0 and -0 are one value.  No logit gives 0.
__device__ __forceinline__ uint32_t order_bits(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return z != z ? 0xFFFFFFFEu : (int)u < 0 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t order_key(float z, int idx) {
  return ((uint64_t)order_bits(z) << 32) | (uint32_t)~idx;
}
__device__ __forceinline__ int index_of(uint64_t key) { return (int)~(uint32_t)key; }
__device__ __forceinline__ float logit_of(uint64_t key) {  // (of -0: +0)
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float((int)o < 0 ? o & 0x7FFFFFFFu : ~o);
}
// (of -inf and below: masked out, or no logit)
__device__ __forceinline__ bool masked_out(uint64_t key) { return (uint32_t)(key >> 32) <= 0x007FFFFFu; }

// A thread's running statistics: the largest logit m, and relative to a whole
// exponent r (that of the largest so far, kLow before) s = sum 2^t and w = sum
// 2^t t, t = z log2 e - r in one FMA.  A change of r scales by a power of two.
// Logits below -2^21 (masks) add nothing beside others; a row or segment whose
// largest lies outside +-2^21, where t would lose its fraction, is summed again
// relative to that logit itself.  (Bound by these instructions, not by memory,
// where few rows or 16-bit ones are read: with the sums relative to the maximum
// of every 16 bytes, twice the instructions, 32000 logits of one row took 5.7 us
// in place of 4.8, 900 rows of 40000 with 16 alternatives 36.8 in place of 33.0.)
constexpr float kLow = -4194304.f, kRange = 2097152.f;
constexpr float kFar = -1000.f;  // 2^kFar is 0, and a product of the two is (with -inf it would not be)

struct Run {
  float m = -INFINITY, r = kLow;
  float s[4] = {0.f, 0.f, 0.f, 0.f}, w[4] = {0.f, 0.f, 0.f, 0.f};  // (four chains of additions)
};

__device__ __forceinline__ float exponent_of(float m) { return fminf(fmaxf(rintf(m * kLog2e), kLow), -kLow); }

__device__ __forceinline__ void rescale(Run& a, float r) {
  if (r > a.r) {
    const float d = a.r - r, e = __builtin_amdgcn_exp2f(d);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a.w[i] = fmaf(a.s[i], fmaxf(d, kFar), a.w[i]) * e;
      a.s[i] *= e;
    }
    a.r = r;
  }
}

// Logits up to `most` are to be added.
__device__ __forceinline__ void make_room(Run& a, float most) {
  a.m = fmaxf(a.m, most);
  rescale(a, exponent_of(most));
}
template <int N>
__device__ __forceinline__ void add(Run& a, const float* z) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float t = fmaf(z[i], kLog2e, -a.r), e = __builtin_amdgcn_exp2f(t);
    a.s[i & 3] += e;
    a.w[i & 3] = fmaf(e, fmaxf(t, kFar), a.w[i & 3]);
  }
}

// The statistics of a row or segment: lse = hi + lo + ln s, the sum s = sum
// e^(z - hi - lo) and w = sum e^(z - hi - lo) (z - hi - lo).  hi is -inf where
// there is nothing but -inf.
struct Stat {
  float hi, lo, s, w;
};
constexpr float kLn2 = 0.693147182464599609375f, kLn2Rest = -1.904654299957767e-9f;  // ln 2 as two floats
constexpr float kLog2eRest = 1.3349759e-8f;  // (log2 e - kLog2e) ln 2: the base is off by m times that
__device__ __forceinline__ Stat stat_of(float m, float r, float s, float w) {
  Stat st;
  st.hi = r * kLn2;
  st.lo = fmaf(r, kLn2, -st.hi) + fmaf(r, kLn2Rest, m * kLog2eRest);
  if (m == -INFINITY) st.hi = -INFINITY, st.lo = 0.f;
  st.s = s;
  st.w = w * kLn2;
  return st;
}
// Relative to another base.
__device__ __forceinline__ void rebase(Stat& a, float hi, float lo) {
  const float d = a.hi == -INFINITY ? -INFINITY : (a.hi - hi) + (a.lo - lo);
  const float e = exp_e(d);
  a.w = fmaf(a.s, fmaxf(d, kFar), a.w) * e;
  a.s *= e;
  a.hi = hi;
  a.lo = lo;
}

// The waves' maxima, then their sums, met by the workgroup.
template <int WAVES>
struct Meet {
  float m[WAVES], s[WAVES], w[WAVES];
};
template <int WAVES>
__device__ __forceinline__ void meet_max(Run& a, const Meet<WAVES>& meet) {
  float m = meet.m[0];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) m = fmaxf(m, meet.m[i]);
  a.m = m;
  rescale(a, exponent_of(m));
}
template <int WAVES>
__device__ __forceinline__ void meet_sums(float& s, float& w, const Meet<WAVES>& meet) {
  s = meet.s[0];
  w = meet.w[0];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) {
    s += meet.s[i];
    w += meet.w[i];
  }
}

// How many of n numbers (LDS) are at least `bound` (> 0), in every thread.  `tally`:
// this call's alone until the workgroup's next barrier but one.
template <int WAVES>
__device__ __forceinline__ int count_from(const uint32_t* v, int n, uint32_t bound, int* tally) {
  constexpr int U = 8;
  int c = 0;
  for (int i0 = 0; i0 < n; i0 += WAVES * 64 * U) {
    uint32_t x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * WAVES * 64 + threadIdx.x;
      x[u] = i < n ? v[i] : 0;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) c += __popcll(__ballot(x[u] >= bound));
  }
  if ((threadIdx.x & 63) == 0) tally[threadIdx.x >> 6] = c;
  __syncthreads();
  c = tally[0];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) c += tally[i];
  return c;
}

// The `want` greatest of n > want numbers (LDS), the lower index first among
// equals: their indices to `slot`, in any order (*count of them, 0 before);
// returns a bound that they and no others but equals of it reach.  `start`: a
// bound to try first (where ties are what made this necessary it is mostly the
// one); if fewer than `want` reach it, those alone are taken.
template <int WAVES>
__device__ __forceinline__ uint32_t greatest(const uint32_t* v, int n, int want, uint32_t start, int* slot, int* count,
                                             int (*tally)[WAVES]) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  uint32_t bound = start;
  int have = n, turn = 1, above = count_from<WAVES>(v, n, start + 1, tally[0]);
  if (above >= want) {
    bound = 0;
    for (int bit = 31; bit >= 0 && have > want; --bit, turn ^= 1) {
      const int c = count_from<WAVES>(v, n, bound | (1u << bit), tally[turn]);
      if (c >= want) {
        bound |= 1u << bit;
        have = c;
      }
    }
    if (have > want) {
      above = count_from<WAVES>(v, n, bound + 1, tally[turn]);
      turn ^= 1;
    }
  }
  // all above the bound; of its equals (where they are too many) the first
  int left = want - above;
  for (int i0 = 0; i0 < n; i0 += WAVES * 64, turn ^= 1) {
    const int i = i0 + t;
    const uint32_t x = i < n ? v[i] : 0;
    bool take = i < n && x > bound;
    const bool equal = i < n && x == bound;
    const uint64_t equals = __ballot(equal);
    if (have > want) {
      if (lane == 0) tally[turn][wave] = __popcll(equals);
      __syncthreads();
      int before = __popcll(equals & ((1ull << lane) - 1)), all = 0;
      for (int w = 0; w < WAVES; ++w) {
        before += w < wave ? tally[turn][w] : 0;
        all += tally[turn][w];
      }
      take = take || (equal && before < left);
      left -= all < left ? all : left;
    } else {
      take = take || equal;
    }
    if (take) slot[atomicAdd(count, 1)] = i;
  }
  __syncthreads();
  return bound;
}

// lp of a logit, by way of the base: of the rounding of lse that of ln s alone
// remains.
__device__ __forceinline__ float logp_of(float z, const Stat& st, float ln_s) { return ((z - st.hi) - st.lo) - ln_s; }

// The token of a row and its logit, loaded ahead of the row (by one thread).
struct Token {
  int tk;
  float z;
};
template <int T>
__device__ __forceinline__ Token token_of(const TokenLogpArgs& a, int row) {
  Token k{0, 0.f};
  if (a.lp) {
    k.tk = a.tokens[row];
    if (k.tk >= 0 && k.tk < a.V) k.z = load_z<T>(a.z, (size_t)row * a.ld + k.tk);
  }
  return k;
}

// One thread: the row's statistics.
__device__ __forceinline__ void finish_row(const TokenLogpArgs& a, int row, const Stat& st, const Token& k) {
  const float ln_s = log_e(st.s);
  if (a.lse) a.lse[row] = st.hi + (st.lo + ln_s);
  if (a.entropy) a.entropy[row] = ln_s - st.w / st.s;
  if (a.lp) {
    const bool ok = k.tk >= 0 && k.tk < a.V;
    a.lp[row] = ok ? logp_of(k.z, st, ln_s) : __builtin_nanf("");
    if (!ok && a.err) atomicOr(a.err, 1);
  }
}

// One wave: f(rank, key) for each of the n keys at `key` (LDS, 16-byte aligned,
// room for a multiple of 16), the rank counted over all of them; 128 keys at a
// time, two to a lane.  (One to a lane, 8 keys loaded at a time: 85 rows of 3186
// with 32 alternatives 10.0 us, not 9.0.)
template <class F>
__device__ __forceinline__ void each_ranked(uint64_t* key, int n, F f) {
  constexpr int U = 16;
  const int lane = threadIdx.x & 63, padded = (n + U - 1) / U * U;
  if (lane < padded - n) key[n + lane] = 0;
  __builtin_amdgcn_wave_barrier();
  for (int i = lane; i - lane < n; i += 128) {
    const uint64_t a = i < n ? key[i] : ~0ull, b = i + 64 < n ? key[i + 64] : ~0ull;
    int rank_a = 0, rank_b = 0;
    for (int j = 0; j < padded; j += U) {
      uint64_t other[U];
#pragma unroll
      for (int q = 0; q < U; ++q) other[q] = key[j + q];
#pragma unroll
      for (int q = 0; q < U; ++q) rank_a += other[q] > a;
      if (n - i + lane > 64) {
#pragma unroll
        for (int q = 0; q < U; ++q) rank_b += other[q] > b;
      }
    }
    if (i < n) f(rank_a, a);
    if (i + 64 < n) f(rank_b, b);
  }
}

// One wave: the row's alternatives from n keys, which hold all logits of the
// first k that are not masked out.
template <int T>
__device__ __forceinline__ void finish_top(const TokenLogpArgs& a, int row, const Stat& st, uint64_t* key, int n) {
  const int lane = threadIdx.x & 63, k = a.top;
  const size_t o0 = (size_t)row * k;
  const float ln_s = log_e(st.s);
  const auto put = [&](int rank, int id, float z) __attribute__((always_inline)) {
    if (rank >= k) return;
    a.ids[o0 + rank] = id;
    if (a.top_lp) a.top_lp[o0 + rank] = logp_of(z, st, ln_s);
  };
  each_ranked(key, n, [&](int rank, uint64_t mine) __attribute__((always_inline)) { put(rank, index_of(mine), logit_of(mine)); });
  if (n >= k) return;
  // Fewer than k <= 32 logits are not masked out: of the first 64 entries (or of
  // all, at least k) enough are.
  const bool out = lane < a.V && load_z<T>(a.z, (size_t)row * a.ld + lane) == -INFINITY;
  const uint64_t outs = __ballot(out);
  if (out) put(n + __popcll(outs & ((1ull << lane) - 1)), lane, -INFINITY);
}

// Partial results of a segment in the workspace: all statistics [M][nseg], then
// all keys [M][nseg][top], the greatest first, 0 behind the last.
struct Parts {
  Stat* stat;
  uint64_t* key;
};

// The groups (of kVec elements from the first boundary on) of a segment.
struct Span {
  int head, g0, g1;    // elements before the first group; the segment's groups
  int tail0;           // elements [tail0, V) behind the last group
  bool first, last;
};
template <int T>
__device__ __forceinline__ Span span_of(const void* row, int V, int seg, int nseg) {
  constexpr int VEC = kVec<T>;
  Span s;
  s.head = head_of<T>(row, V);
  const int groups = (V - s.head) / VEC, per = (groups + nseg - 1) / nseg;
  s.g0 = min(groups, seg * per);
  s.g1 = min(groups, s.g0 + per);
  s.tail0 = s.head + groups * VEC;
  s.first = seg == 0;
  s.last = seg == nseg - 1;
  return s;
}

// Grid: M * nseg workgroups.
template <int T, bool TOP, int THREADS>
__global__ __launch_bounds__(THREADS) void token_logp_kernel(TokenLogpArgs a, int nseg, Parts parts) {
  constexpr int VEC = kVec<T>, WAVES = THREADS / 64;
  extern __shared__ float most_of[];  // TOP: the maxima of the segment's groups
  __shared__ Meet<WAVES> meet;
  // TOP: the waves' bounds, the groups that reach the bound, the logits that do
  __shared__ float bound_of[TOP ? WAVES : 1];
  __shared__ int slot[TOP ? kCand : 1], count[2], tally[TOP ? 2 : 1][WAVES];
  __shared__ __align__(16) uint64_t cand[TOP ? kCand : 1];
  const int row = blockIdx.x / nseg, seg = blockIdx.x - row * nseg, t = threadIdx.x, V = a.V;
  const uint8_t* const z = static_cast<const uint8_t*>(a.z) + (size_t)row * a.ld * (16 / VEC);
  const Span sp = span_of<T>(z, V, seg, nseg);
  const uint4* const v = reinterpret_cast<const uint4*>(z + (size_t)sp.head * (16 / VEC));
  Token token{0, 0.f};
  if (t == 0 && nseg == 1) token = token_of<T>(a, row);
  if (TOP && t < 2) count[t] = 0;
  const int groups = sp.g1 - sp.g0;
  const __amdgpu_buffer_rsrc_t rs = make_rsrc(v + sp.g0, (uint32_t)groups * 16u);
  const int first_of_wave = __builtin_amdgcn_readfirstlane(t & ~63);
  Run run;
  constexpr int ROUND = THREADS * TL_U;
  for (int g0 = 0; g0 < groups; g0 += ROUND) {
    uint4 u[TL_U];
#pragma unroll
    for (int q = 0; q < TL_U; ++q) {
      const int g = g0 + q * THREADS + t;
      u[q] = buf_load16(rs, g < groups ? g * 16 : kOutOfRange);
    }
    if (g0 + ROUND > groups) {  // the last round: -inf where there is no group
      constexpr uint32_t none = T == kF32 ? 0xFF800000u : 0xFF80FF80u;
#pragma unroll
      for (int q = 0; q < TL_U; ++q)
        if (g0 + q * THREADS + t >= groups) u[q] = make_uint4(none, none, none, none);
    }
    float f[TL_U * VEC], most = -INFINITY;
#pragma unroll
    for (int q = 0; q < TL_U; ++q) {
      float x[VEC];
      unpack<T>(u[q], x);
      float m = x[0];
#pragma unroll
      for (int e = 1; e < VEC; ++e) m = fmaxf(m, x[e]);
#pragma unroll
      for (int e = 0; e < VEC; ++e) f[q * VEC + e] = x[e];
      if constexpr (TOP) {
        const int g = g0 + q * THREADS + t;
        if (g < groups) most_of[g] = m;
      }
      most = fmaxf(most, m);
    }
    make_room(run, most);
#pragma unroll
    for (int q = 0; q < TL_U; ++q)
      if (g0 + q * THREADS + first_of_wave < groups) add<VEC>(run, f + q * VEC);
  }
  // the elements in no group: a thread each
  float edge = -INFINITY;
  int edge_at = -1;
  if (sp.first && t < sp.head) edge_at = t;
  if (sp.last && t >= 64 && t - 64 < V - sp.tail0) edge_at = sp.tail0 + t - 64;
  if (edge_at >= 0) {
    edge = load_z<T>(z, edge_at);
    make_room(run, edge);
    add<1>(run, &edge);
  }
  // First meeting: the maxima, and (TOP) each wave's bound.
  const float mine = run.m;
  const int lane = t & 63, wave = t >> 6;
  const float wave_most = wave_max(mine);
  if (lane == 0) meet.m[wave] = wave_most;
  // whole waves of groups, or the only one (where the last wave's few threads cannot
  // bound anything, and what is left to others is few)
  const int waves = groups >= 64 ? min(WAVES, groups / 64) : groups > 0;
  if constexpr (TOP) {
    float bound = -INFINITY;
    if (wave < waves) {
      const int j = (a.top + waves - 1) / waves;
      bound = wave_most;
      if (j >= 5) {
        // bit by bit, until j lanes reach it (what lies between the j-th and the
        // next is as good a bound) or it is found; extracted one by one, 3361 rows
        // of 1508 bf16 with 32 alternatives 16.5 us, not 12.3
        const uint32_t key = order_bits(mine);
        uint32_t least = 0;
        for (int bit = 31; bit >= 0; --bit) {
          const uint32_t next = least | (1u << bit);
          const int c = __popcll(__ballot(key >= next));
          if (c >= j) least = next;
          if (c == j) break;
        }
        bound = least > 0x007FFFFFu ? logit_of((uint64_t)least << 32) : -INFINITY;  // (0x007FFFFF: -inf)
      } else {
        float left = mine;
        for (int i = 1; i < j; ++i) {
          const uint64_t have = __ballot(left == bound);
          if (lane == __ffsll((unsigned long long)have) - 1) left = -INFINITY;
          bound = wave_max(left);
        }
      }
    }
    if (lane == 0) bound_of[wave] = bound;
  }
  __syncthreads();
  meet_max(run, meet);
  float sum = wave_sum((run.s[0] + run.s[1]) + (run.s[2] + run.s[3]));
  float mean = wave_sum((run.w[0] + run.w[1]) + (run.w[2] + run.w[3]));
  if (lane == 0) {
    meet.s[wave] = sum;
    meet.w[wave] = mean;
  }
  // Second meeting: the sums, and (TOP) the groups that reach the bound.
  float bound = -INFINITY;
  const auto reaches = [&](float x) __attribute__((always_inline)) { return x >= bound && x != -INFINITY; };
  if constexpr (TOP) {
    if (waves > 0) bound = bound_of[0];
    for (int i = 1; i < waves; ++i) bound = fminf(bound, bound_of[i]);
    constexpr int U = 4;  // (loads from LDS under way; with 8, 4000 x 5000 fp32 with 8 alternatives 21.1 us, not 20.8)
    for (int g0 = t; g0 < groups; g0 += THREADS * U) {
      float x[U];
#pragma unroll
      for (int q = 0; q < U; ++q) x[q] = g0 + q * THREADS < groups ? most_of[g0 + q * THREADS] : -INFINITY;
#pragma unroll
      for (int q = 0; q < U; ++q)
        if (reaches(x[q])) {
          const int i = atomicAdd(&count[0], 1);
          if (i < kCand) slot[i] = g0 + q * THREADS;
        }
    }
    if (edge_at >= 0 && reaches(edge)) cand[atomicAdd(&count[1], 1)] = order_key(edge, edge_at);
  }
  __syncthreads();
  meet_sums(sum, mean, meet);
  Stat st = stat_of(run.m, run.r, sum, mean);
  if (run.m != -INFINITY && !(fabsf(run.m) <= kRange)) {
    // far from zero: the sums relative to the largest logit itself
    sum = mean = 0.f;
    const auto add = [&](float x) __attribute__((always_inline)) {
      const float d = x - run.m, e = exp_e(d);
      sum += e;
      mean = fmaf(e, fmaxf(d, kFar), mean);
    };
    for (int e = sp.head + sp.g0 * VEC + t; e < sp.head + sp.g1 * VEC; e += THREADS) add(load_z<T>(z, e));
    if (edge_at >= 0) add(edge);
    __syncthreads();
    sum = wave_sum(sum);
    mean = wave_sum(mean);
    if (lane == 0) {
      meet.s[wave] = sum;
      meet.w[wave] = mean;
    }
    __syncthreads();
    st.hi = run.m;
    st.lo = 0.f;
    meet_sums(st.s, st.w, meet);
  }
  if (t == 0) {
    if (nseg == 1)
      finish_row(a, row, st, token);
    else
      parts.stat[blockIdx.x] = st;
  }
  if constexpr (TOP) {
    const int k = a.top, slots = count[0];
    int n = kCand + 1;  // too many
    if (slots <= kCand && st.s >= 0.f) {  // (no NaN and no +inf)
      for (int i = t; i < slots * VEC; i += THREADS) {
        const int e = sp.head + (sp.g0 + slot[i / VEC]) * VEC + i % VEC;
        const float x = load_z<T>(z, e);
        if (reaches(x)) {
          const int p = atomicAdd(&count[1], 1);
          if (p < kCand) cand[p] = order_key(x, e);
        }
      }
      __syncthreads();
      n = count[1];
    }
    if (n > kCand) {
      // by the groups' maxima as whole numbers; of a row with NaN they are formed again
      __syncthreads();
      uint32_t* const key = reinterpret_cast<uint32_t*>(most_of);
      const bool again = !(st.s >= 0.f);
      for (int g = t; g < groups; g += THREADS) {
        uint32_t most = 0;
        if (again) {
          float f[VEC];
          unpack<T>(v[sp.g0 + g], f);
#pragma unroll
          for (int e = 0; e < VEC; ++e) most = max(most, order_bits(f[e]));
        } else {
          most = order_bits(most_of[g]);
        }
        key[g] = most;
      }
      if (t < 2) count[t] = 0;
      __syncthreads();
      uint32_t least = 0;
      if (groups > k) {
        // (logits in no group can be among those that reach the waves' bound)
        least = greatest(key, groups, k, again ? 0 : order_bits(bound), slot, &count[0], tally);
      } else {
        if (t < groups) slot[t] = t;
        if (t == 0) count[0] = groups;
        __syncthreads();
      }
      for (int i = t; i < count[0] * VEC; i += THREADS) {
        const int e = sp.head + (sp.g0 + slot[i / VEC]) * VEC + i % VEC;
        const uint64_t x = order_key(load_z<T>(z, e), e);
        if ((uint32_t)(x >> 32) >= least && !masked_out(x)) cand[atomicAdd(&count[1], 1)] = x;
      }
      if (edge_at >= 0) {
        const uint64_t x = order_key(edge, edge_at);
        if (!masked_out(x)) cand[atomicAdd(&count[1], 1)] = x;
      }
      __syncthreads();
      n = count[1];
    }
    if (wave != 0) return;
    if (nseg == 1) {
      finish_top<T>(a, row, st, cand, n);
      return;
    }
    uint64_t* const out = parts.key + (size_t)blockIdx.x * k;
    each_ranked(cand, n, [&](int rank, uint64_t me) __attribute__((always_inline)) {
      if (rank < k) out[rank] = me;
    });
    for (int i = n + lane; i < k; i += 64) out[i] = 0;
  }
}

// One wave per row.
template <int T>
__global__ __launch_bounds__(64) void token_logp_join_kernel(TokenLogpArgs a, int nseg, Parts parts) {
  __shared__ __align__(16) uint64_t cand[kSegs * kMaxTop];
  const int row = blockIdx.x, lane = threadIdx.x, k = a.top;
  Token token{0, 0.f};
  if (lane == 0) token = token_of<T>(a, row);
  const Stat* const ps = parts.stat + (size_t)row * nseg;
  const uint64_t* const pk = parts.key + (size_t)row * nseg * k;
  const uint64_t early = lane < nseg * k ? pk[lane] : 0;
  Stat st{-INFINITY, 0.f, 0.f, 0.f};
  if (lane < nseg) st = ps[lane];
  // relative to the greatest base; its lo goes with it
  const float hi = wave_max(st.hi);
  const float lo = wave_max(st.hi == hi ? st.lo : -INFINITY);
  if (hi != -INFINITY) rebase(st, hi, lo);
  st.s = wave_sum(st.s);
  st.w = wave_sum(st.w);
  if (lane == 0) finish_row(a, row, st, token);
  if (k == 0) return;
  uint64_t bound = 0;
  if (nseg * k > 64) {
    // of many, what reaches a bound that k keys reach: the greatest of the
    // segments' k-th keys or the least of their j-th, j = k over the segments
    // (6 x 50272 fp32, 8 segments of 32 keys: 12.1 us; by the first alone 20.0)
    const int j = (k + nseg - 1) / nseg;
    uint64_t most = lane < nseg ? pk[lane * k + k - 1] : 0, least = lane < nseg ? pk[lane * k + j - 1] : ~0ull;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
      const uint64_t u = __shfl_xor((unsigned long long)most, o), v = __shfl_xor((unsigned long long)least, o);
      most = u > most ? u : most;
      least = v < least ? v : least;
    }
    bound = most > least ? most : least;
  }
  int n = 0;
  for (int i = lane; i - lane < nseg * k; i += 64) {
    const uint64_t key = i < 64 ? early : i < nseg * k ? pk[i] : 0;
    const bool in = key != 0 && key >= bound;
    const uint64_t ins = __ballot(in);
    if (in) cand[n + __popcll(ins & ((1ull << lane) - 1))] = key;
    n += __popcll(ins);
  }
  __syncthreads();
  finish_top<T>(a, row, st, cand, n);
}

// ---- gradient

constexpr int64_t kCacheBytes = int64_t(256) << 20;  // the memory-side cache
constexpr int TB_THREADS = 256;
constexpr int TB_U = 2;  // (2048 x 32000 fp32 into bf16 48.4 us, with 4 50.4; 250 x 50272 bf16 9.8 and 10.5)

template <bool FAR, class V>
__device__ __forceinline__ V fetch(const V* p) {
  return FAR ? __builtin_nontemporal_load(p) : *p;
}
template <bool FAR, class V>
__device__ __forceinline__ void put(V* p, V v) {
  if constexpr (FAR)
    __builtin_nontemporal_store(v, p);
  else
    *p = v;
}

// FAR: past the caches, for logits and gradient that they cannot hold together
// anyway (2048 x 32000 fp32 into bf16, 393 MB: 48.4 us, through them 55.2; but 250 x
// 50272 bf16, 50 MB: 11.2, through them 9.8).
// Stretches of `per` groups; workgroup b takes stretches b, b + gridDim.x, ...
// of the M * n of all rows.
template <int TZ, int TD>
struct BackGroup {
  // 16 bytes of logits, or of the gradient where it is wider: a lane that loads 16
  // bytes and stores 32 leaves gaps in each of its two stores (2048 x 32000 bf16
  // into fp32 with half of the rows live: 102 us that way, 64.5 this way)
  static constexpr bool WIDER = TZ == kBf16 && TD == kF32;
  static constexpr int VEC = WIDER ? 4 : kVec<TZ>, U = WIDER ? 2 * TB_U : TB_U;
};

template <int TZ, int TD, bool FAR>
__global__ __launch_bounds__(TB_THREADS) void token_logp_back_kernel(TokenLogpBackArgs a, int n, int per) {
  using G = BackGroup<TZ, TD>;
  constexpr bool WIDER = G::WIDER;
  constexpr int VEC = G::VEC, U = G::U, ZB = TZ == kF32 ? 4 : 2, DB = TD == kF32 ? 4 : 2;
  using in_t = typename std::conditional<WIDER, u32x2_t, u32x4_t>::type;
  using out_t = typename std::conditional<VEC * DB == 8, u32x2_t, u32x4_t>::type;
  const int t = threadIdx.x, V = a.V;
  for (int64_t b = blockIdx.x; b < (int64_t)a.M * n; b += gridDim.x) {
    const int row = (int)(b / n), part = (int)(b - (int64_t)row * n);
    const uint8_t* const z = static_cast<const uint8_t*>(a.z) + (size_t)row * a.ld * ZB;
    uint8_t* const d = static_cast<uint8_t*>(a.dz) + (size_t)row * a.ld_d * DB;
    float d_lp = a.d_lp ? a.d_lp[row] : 0.f;
    const float d_h = a.d_entropy ? a.d_entropy[row] : 0.f;
    const bool live = d_lp != 0.f || d_h != 0.f;
    const float lse = a.lse[row], h = d_h != 0.f ? a.entropy[row] : 0.f;
    int tk = -1;
    if (d_lp != 0.f) {
      tk = a.tokens[row];
      if (tk < 0 || tk >= V) {
        d_lp = __builtin_nanf("");  // (all of the row's gradient)
        if (part == 0 && t == 0 && a.err) atomicOr(a.err, 1);
      }
    }
    const auto gradient = [&](float x) __attribute__((always_inline)) {  // of every logit but the token's
      const float lp = x - lse, p = exp_e(lp);
      return -p * (d_h == 0.f ? d_lp : fmaf(d_h, fmaxf(lp, kFar) + h, d_lp));  // (p = 0 where lp is -inf)
    };
    const auto one = [&](int e) __attribute__((always_inline)) {
      const float f = live ? gradient(load_z<TZ>(z, e)) + (e == tk ? d_lp : 0.f) : 0.f;
      store_elem(d, TD, e, f);
    };
    const int head = head_of<TZ>(z, V), groups = (V - head) / VEC;
    const int g0 = min(groups, part * per), g1 = min(groups, g0 + per);
    if ((reinterpret_cast<uintptr_t>(d) + head * DB) % sizeof(out_t) != 0) {  // input and output never on a boundary together
      const int e0 = part == 0 ? 0 : head + g0 * VEC, e1 = part == n - 1 ? V : head + g1 * VEC;
      for (int e = e0 + t; e < e1; e += TB_THREADS) one(e);
      continue;
    }
    const in_t* const zv = reinterpret_cast<const in_t*>(z + (size_t)head * ZB);
    out_t* const dv = reinterpret_cast<out_t*>(d + (size_t)head * DB);
    for (int g = g0 + t; g < g1; g += TB_THREADS * U) {
      in_t u[U];
      if (live) {
#pragma unroll
        for (int q = 0; q < U; ++q)
          if (g + q * TB_THREADS < g1) u[q] = fetch<FAR>(zv + g + q * TB_THREADS);
      }
#pragma unroll
      for (int q = 0; q < U; ++q) {
        const int at = g + q * TB_THREADS;
        if (at >= g1) break;
        float f[VEC];
        if (live) {
          if constexpr (WIDER)
            unpack(u[q], f);
          else
            unpack<TZ>(__builtin_bit_cast(uint4, u[q]), f);
#pragma unroll
          for (int e = 0; e < VEC; ++e) f[e] = gradient(f[e]);
          const int mine = tk - head - at * VEC;  // the token's place in this group
          if ((unsigned)mine < (unsigned)VEC) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[e] += e == mine ? d_lp : 0.f;
          }
        } else {
#pragma unroll
          for (int e = 0; e < VEC; ++e) f[e] = 0.f;
        }
        out_t w;
#pragma unroll
        for (int e = 0; e < VEC * DB / 4; ++e) {
          if constexpr (TD == kF32)
            w[e] = __float_as_uint(f[e]);
          else
            w[e] = f32_to_bf16_pair(f[2 * e], f[2 * e + 1]);
        }
        put<FAR>(dv + at, w);
      }
    }
    if (part == 0 && t < head) one(t);
    if (part == n - 1 && t < V - head - groups * VEC) one(head + groups * VEC + t);
  }
}

// Segments of a row: none longer than kSegMost; more, of 24 KB, where a row is
// longer than 128 KB and there are few enough rows for three each on 256 workgroups
// (their join is a second launch).  50272 fp32 logits with 8 alternatives: 6 rows
// 8.6 us in eight segments, 9.9 in one; 64 rows 10.5 in four and 11.1; 100 rows 12.7
// in two and 11.8.  One row 6.2 and 6.4; of 32000 fp32 5.6 in five and 4.9.
int segments(int M, int V, int type) {
  const int64_t least = (V + kSegMost - 1) / kSegMost, bytes = V * (int64_t)type_bytes(type);
  int64_t n = bytes > (128 << 10) ? bytes / (24 << 10) : 1;
  n = n < 256 / M ? n : 256 / M;
  n = n < 3 ? 1 : n;
  n = n > least ? n : least;
  return (int)(n < kSegs ? n : kSegs);
}

// Threads of a row or segment.  128 for rows of up to five of their rounds of
// loads, where there are enough to fill the chip that way: 2000 fp32 logits, 400
// rows 3.4 us (with 512 threads 3.9); 5000 bf16 with 8 alternatives, 900 rows 7.4
// (9.5); 10000 fp32, 900 rows 8.2 (9.1), but 400 rows 6.9 (5.9).  256 for rows of up
// to five of theirs, or three where the logits are more than the caches turn over:
// 1000 rows of 32000 bf16 with 20 alternatives 17.9 us (with 512 threads 19.6), but
// 300 rows with 8 10.9 (10.3); 2000 rows of 12000 fp32 with 20 21.2 (25.4), but of
// 24000 with 8 41.6 (37.8).
int threads_of(int M, int groups) {
  if (groups <= 2560 && M >= 256 + groups / 4) return 128;
  const bool much = (int64_t)M * groups > (6 << 20);  // 96 MB
  return M >= 400 && groups <= (much ? 3200 : 5120) ? 256 : 512;
}

size_t stat_bytes(int M, int nseg) { return ((size_t)M * nseg * sizeof(Stat) + 15) & ~size_t(15); }

template <int T, int THREADS>
void rows_of(const TokenLogpArgs& a, int nseg, const Parts& p, hipStream_t stream) {
  const dim3 grid((unsigned)(a.M * nseg)), block(THREADS);
  if (a.top > 0) {
    const int groups = (a.V / kVec<T> + nseg - 1) / nseg + 1;
    hipLaunchKernelGGL((token_logp_kernel<T, true, THREADS>), grid, block, groups * sizeof(float), stream, a, nseg, p);
  } else {
    hipLaunchKernelGGL((token_logp_kernel<T, false, THREADS>), grid, block, 0, stream, a, nseg, p);
  }
}

template <int T>
void forward(const TokenLogpArgs& a, int nseg, const Parts& p, hipStream_t stream) {
  switch (nseg == 1 ? threads_of(a.M, a.V / kVec<T>) : 512) {
    case 128: rows_of<T, 128>(a, nseg, p, stream); break;
    case 256: rows_of<T, 256>(a, nseg, p, stream); break;
    default: rows_of<T, 512>(a, nseg, p, stream);
  }
  if (nseg > 1) hipLaunchKernelGGL((token_logp_join_kernel<T>), dim3(a.M), dim3(64), 0, stream, a, nseg, p);
}

}  // namespace

size_t token_logp_ws_bytes(int M, int V, int top) {
  const int nseg = segments(M, V, kF32);  // (the most of the two types)
  return nseg == 1 ? 0 : stat_bytes(M, nseg) + (size_t)M * nseg * top * sizeof(uint64_t);
}

hipError_t launch_token_logp(const TokenLogpArgs& a, void* ws, hipStream_t stream) {
  const int nseg = segments(a.M, a.V, a.type);
  Parts p{static_cast<Stat*>(ws), reinterpret_cast<uint64_t*>(static_cast<uint8_t*>(ws) + stat_bytes(a.M, nseg))};
  if (a.type == kF32)
    forward<kF32>(a, nseg, p, stream);
  else
    forward<kBf16>(a, nseg, p, stream);
  return hipGetLastError();
}

template <int TZ, int TD>
static void back_of(const TokenLogpBackArgs& a, hipStream_t stream) {
  // a stretch is one round of the workgroup's loads, or several where there are many
  using G = BackGroup<TZ, TD>;
  constexpr int ROUND = TB_THREADS * G::U;
  const int groups = a.V / G::VEC > 0 ? a.V / G::VEC : 1;
  const int64_t rounds = (int64_t)a.M * ((groups + ROUND - 1) / ROUND);
  int per = ROUND;
  while (per < 8 * ROUND && rounds * ROUND / per > 8192) per *= 2;
  const int n = (groups + per - 1) / per;
  const int64_t all = (int64_t)a.M * n;
  const dim3 grid((unsigned)(all < (1 << 20) ? all : 1 << 20)), block(TB_THREADS);
  if ((int64_t)a.M * a.V * (int64_t)(type_bytes(TZ) + type_bytes(TD)) > kCacheBytes)
    hipLaunchKernelGGL((token_logp_back_kernel<TZ, TD, true>), grid, block, 0, stream, a, n, per);
  else
    hipLaunchKernelGGL((token_logp_back_kernel<TZ, TD, false>), grid, block, 0, stream, a, n, per);
}

hipError_t launch_token_logp_back(const TokenLogpBackArgs& a, hipStream_t stream) {
  if (a.type == kF32)
    a.d_type == kF32 ? back_of<kF32, kF32>(a, stream) : back_of<kF32, kBf16>(a, stream);
  else
    a.d_type == kF32 ? back_of<kBf16, kF32>(a, stream) : back_of<kBf16, kBf16>(a, stream);
  return hipGetLastError();
}

}  // namespace hydra
