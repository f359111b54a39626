// The dual-output linear over a frozen weight held in e4m3 with power-of-two
// scales (128 values of a row of x, 128 x 128 of W):
//   y_off = xh Wh^T,  y_on = y_off + s (x A^T) B^T,
// xh and Wh what the bytes stand for.
//
// Two ways to form the base product, by where it ends:
//  * into bf16 (in fp8_gemm_kernel): the scaled 8-bit matrix instructions, which take
//    bytes and scales as they are at twice bf16's rate, and whose sums are 2e-5 off
//    (hydra_fp8.h);
//  * into fp32, and in fp8_stream_kernel, where reading W is what costs: bf16 matrix
//    instructions on the exact values (four fraction bits of bf16's eight), the
//    bytes converted in registers on the way in, sums in fp32.
// Kernels:
//  * fp8_prep_kernel reads x once: its bytes and scales, and partial sums of
//    T = x A^T for the update;
//  * fp8_t_finish_kernel adds those up once where many tiles would at a high rank;
//  * fp8_stream_kernel (up to 16 rows) is bound by reading W: every wave takes
//    blocks of 128 k values of 16 or more rows of W straight into registers (8 x 11008 x
//    4096 15.2 us, 3.0 TB/s, behind 3.8 us of x and T);
//  * fp8_gemm_kernel (more rows): tiles through LDS, four waves copying ahead of those that
//    multiply; K in parts where few rows leave CUs without a tile.  Bound by the matrix cores
//    from some 1000 rows on: 2048 x 11008 x 4096 into one bf16 output 118 to 124 us with all
//    launches, 1.5 PFLOP/s, into fp32 181, 1.0; below by the copies into LDS.
// Which tile, how many parts and how much room they take: hydra_fp8_plan.h.
#include <type_traits>

#include "hydra_fp8.h"
#include "hydra_fp8_plan.h"
#include "hydra_philox.h"

namespace hydra {
namespace {

// ------------------------------------------------------------------ before the product

constexpr int P_WAVES = 8;

// Two values as bf16 parts, a pair of each.  Two, rounded, are within 2^-17 of them (the
// first cut, not rounded, where rounding would make it infinite).  Three add up to them: the
// upper half of their bits, that of what it leaves, and what is left then (at most eight
// bits).  An infinity's other parts are zero.
__device__ __forceinline__ void two_parts(float a, float b, uint32_t& hi, uint32_t& lo) {
  const float f[2] = {a, b};
  uint32_t h[2];
  float rest[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    h[i] = f32_to_bf16_any(f[i]);
    if ((h[i] & 0x7FFF) == 0x7F80) h[i] = __float_as_uint(f[i]) >> 16;
    rest[i] = __builtin_isinf(f[i]) ? 0.f : f[i] - bf16_to_f32(h[i]);
  }
  hi = h[0] | h[1] << 16;
  lo = f32_to_bf16_pair(rest[0], rest[1]);
}
__device__ __forceinline__ void three_parts(float a, float b, uint32_t (&p)[3]) {
  const bool ia = __builtin_isinf(a), ib = __builtin_isinf(b);
#pragma unroll
  for (int n = 0; n < 3; ++n) {
    const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
    p[n] = __builtin_amdgcn_perm(ub, ua, 0x07060302u);
    a -= __uint_as_float(ua & 0xFFFF0000u);
    b -= __uint_as_float(ub & 0xFFFF0000u);
    if (n == 0) a = ia ? 0.f : a, b = ib ? 0.f : b;
  }
}

// The pieces of four lanes 16 apart, transposed: v[j] of lane group g becomes v[g] of
// lane group j.
__device__ __forceinline__ void transpose4(uint32_t (&v)[4]) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const auto r = __builtin_amdgcn_permlane32_swap(v[j], v[j + 2], false, false);
    v[j] = r[0];
    v[j + 2] = r[1];
  }
#pragma unroll
  for (int j = 0; j < 4; j += 2) {
    const auto r = __builtin_amdgcn_permlane16_swap(v[j], v[j + 1], false, false);
    v[j] = r[0];
    v[j + 1] = r[1];
  }
}

// 16 rows and one chunk of K a workgroup; a wave takes the chunk's blocks in turn.
// Lane l holds values 32 j + 8 (l / 16) ... + 7, j = 0 ... 3, of the block of row l % 16:
// four lanes read 64 consecutive bytes of a row, a block's maximum is over four
// lanes, and piece j of all lanes is one 16x16x32 product of T.  The bytes change lanes
// for stores of 128 consecutive bytes a row.  2048 x 4096 at rank 16, x quantized: 8.5 us
// (with each lane's eight bytes a store of their own 11.2; with 32 rows a workgroup, for
// half the reads of A, 10.2, with 64 12.9: fewer waves to hide the loads behind).
// QUANT: x's bytes and scales; OWN: the adapter has an input of its own.
template <int RP, bool QUANT, bool OWN>
__global__ __launch_bounds__(P_WAVES * 64) void fp8_prep_kernel(Fp8PrepArgs g) {
  constexpr int TJ = RP / 16, TJ1 = TJ > 0 ? TJ : 1;
  const int t = threadIdx.x, lane = t & 63, l16 = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int K = g.K, kb_n = (K + kFp8Block - 1) / kFp8Block;
  const int m0 = blockIdx.x * 16, rows = min(16, g.M - m0);
  const uint32_t bytes = (uint32_t)rows * K * 2u;
  const __amdgpu_buffer_rsrc_t xr = make_rsrc((QUANT ? g.x : g.xa) + (size_t)m0 * K, bytes);
  const __amdgpu_buffer_rsrc_t ar = make_rsrc(OWN ? g.xa + (size_t)m0 * K : nullptr, OWN ? bytes : 0u);
  const __amdgpu_buffer_rsrc_t Ar = make_rsrc(TJ > 0 ? g.A : nullptr, TJ > 0 ? (uint32_t)g.r * K * 2u : 0u);
  f32x4_t acc[TJ1];
#pragma unroll
  for (int j = 0; j < TJ1; ++j) acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const int kb1 = min(kb_n, (int)(blockIdx.y + 1) * g.kch);
  for (int kb = blockIdx.y * g.kch + wave; kb < kb1; kb += P_WAVES) {
    const int k = kb * kFp8Block + 8 * lg;
    uint4 v[4], a[4], w[4][TJ1];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool ok = k + 32 * j < K;
      v[j] = buf_load16(xr, ok ? (l16 * K + k + 32 * j) * 2 : kOutOfRange);
      if constexpr (OWN) a[j] = buf_load16(ar, ok ? (l16 * K + k + 32 * j) * 2 : kOutOfRange);
#pragma unroll
      for (int i = 0; i < TJ; ++i)
        w[j][i] = buf_load16(Ar, ok ? ((i * 16 + l16) * K + k + 32 * j) * 2 : kOutOfRange);
    }
    if constexpr (QUANT) {
      float f[4][8];
      float most = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        unpack<kBf16>(v[j], f[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) most = fmaxf(most, fp8_magnitude(f[j][i]));
      }
      most = fmaxf(most, __shfl_xor(most, 16));
      most = fmaxf(most, __shfl_xor(most, 32));
      const int byte = fp8_scale_byte(most);
      const float p = fp8_inverse(byte);
      uint32_t lo[4], hi[4];  // values 32 j + 8 lg ... + 3 and + 4 ... + 7; then 32 lg + 8 j ...
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        lo[j] = fp8_pack4(f[j], p);
        hi[j] = fp8_pack4(f[j] + 4, p);
      }
      transpose4(lo);
      transpose4(hi);
      const int kq = kb * kFp8Block + 32 * lg;
      if (l16 < rows) {
        uint8_t* q = g.xq + (size_t)(m0 + l16) * K + kq;
        if (kq < K) *reinterpret_cast<uint4*>(q) = make_uint4(lo[0], hi[0], lo[1], hi[1]);
        if (kq + 16 < K) *reinterpret_cast<uint4*>(q + 16) = make_uint4(lo[2], hi[2], lo[3], hi[3]);
        if (lg == 0) g.xs[(size_t)(m0 + l16) * kb_n + kb] = (uint8_t)byte;
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < TJ; ++i) acc[i] = mfma16(OWN ? a[j] : v[j], w[j][i], acc[i]);
  }
  if constexpr (TJ > 0) {
    // acc[j] of lane l: T[m0 + 4 lg + e][16 j + l16], to be added over the waves
    __shared__ float red[P_WAVES][16][RP];
#pragma unroll
    for (int j = 0; j < TJ; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) red[wave][4 * lg + e][16 * j + l16] = acc[j][e];
    __syncthreads();
    for (int e = t; e < rows * RP; e += P_WAVES * 64) {
      const int row = e / RP, j = e % RP;
      float sum = red[0][row][j];
#pragma unroll
      for (int w = 1; w < P_WAVES; ++w) sum += red[w][row][j];
      // (an infinity times the zeros of a row that A does not have is no number)
      g.part[((size_t)blockIdx.y * g.M + m0 + row) * RP + j] = j < g.r ? sum : 0.f;
    }
  }
}

// s T, which tiles at a rank above 16 read in place of the chunks' sums, as they hold it: in
// fp32, or (PARTS) as two bf16 parts [M][hi rp | lo rp].  Four values a thread.
template <bool PARTS>
__global__ __launch_bounds__(256) void fp8_t_finish_kernel(Fp8PrepArgs g, int lrp) {
  const size_t e = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4, all = (size_t)g.M << lrp;
  if (e >= all) return;
  f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int c = 0; c < g.nch; ++c) v += *reinterpret_cast<const f32x4_t*>(g.part + c * all + e);
  v *= g.s;
  if constexpr (PARTS) {
    uint2 hi, lo;
    two_parts(v[0], v[1], hi.x, lo.x);
    two_parts(v[2], v[3], hi.y, lo.y);
    const size_t row = e >> lrp;
    uint16_t* const o = static_cast<uint16_t*>(g.ts) + (row << (lrp + 1)) + (e - (row << lrp));
    *reinterpret_cast<uint2*>(o) = hi;
    *reinterpret_cast<uint2*>(o + g.rp) = lo;
  } else {
    *reinterpret_cast<f32x4_t*>(static_cast<float*>(g.ts) + e) = v;
  }
}

// ------------------------------------------------------------------ few rows

// 16 NB rows of W a workgroup, the blocks of K dealt to its waves; their partial
// sums meet in LDS in wave order.  U blocks a wave are requested before the first
// is used (two of them and three workgroups a CU: 0 to 15% slower).
template <int NB, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 4) void fp8_stream_kernel(Fp8LinearArgs a) {
  constexpr int U = 4, NT = WAVES * 64;
  __shared__ f32x4_t red[WAVES][NB][64];
  __shared__ __align__(16) float T[16][132];
  __shared__ uint16_t Bs[16 * NB][130];
  const int t = threadIdx.x, lane = t & 63, l16 = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int M = a.M, N = a.N, K = a.K, kb_n = (K + kFp8Block - 1) / kFp8Block;
  const int n0 = blockIdx.x * 16 * NB;
  const __amdgpu_buffer_rsrc_t xr = make_rsrc(a.xq, (uint32_t)M * K);
  const __amdgpu_buffer_rsrc_t wr = make_rsrc(a.wq + (size_t)n0 * K, (uint32_t)min(16 * NB, N - n0) * K);
  const uint8_t* xs = a.xs + (size_t)min(l16, M - 1) * kb_n;
  const uint8_t* ws = a.ws + (size_t)(n0 / kFp8Block) * kb_n;  // (16 NB rows lie in one block of 128)
  f32x4_t acc[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) acc[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  // T as the sum of its chunks in their order, and these rows of B: with 16 rows of W asked
  // for before W and put into LDS while W is on its way (8 x 11008 x 4096 22.3 -> 18.5 us, 1 x
  // 32000 x 4096 33.0 -> 30.6; 32 rows leave no registers for it)
  constexpr int UT = 4;
  const bool lora = a.y_on && a.rp > 0;
  const int lr = lora ? __builtin_ctz(a.rp) : 0, items = lora ? (M << lr) / 4 : 0;
  const int b_n = lora ? min(16 * NB, N - n0) << lr : 0;
  const float* const part = a.part + 4 * t;
  const uint32_t stride = (uint32_t)M << lr;
  f32x4_t tv[UT];
  uint16_t bv = 0;
  auto b_at = [&](int i) {
    const int n = i >> lr, j = i & (a.rp - 1);
    return j < a.r ? a.B[(size_t)(n0 + n) * a.ldb + j] : (uint16_t)0;
  };
  auto ask = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < UT; ++i)
      tv[i] = t < items && i < a.nch ? *reinterpret_cast<const f32x4_t*>(part + i * stride) : f32x4_t{0.f, 0.f, 0.f, 0.f};
    if (t < b_n) bv = b_at(t);
  };
  auto stage = [&]() __attribute__((always_inline)) {
    if (t < items) {
      f32x4_t v = tv[0];
#pragma unroll
      for (int i = 1; i < UT; ++i) v += tv[i];
#pragma unroll 4
      for (int c = UT; c < a.nch; ++c) v += *reinterpret_cast<const f32x4_t*>(part + c * stride);
      *reinterpret_cast<f32x4_t*>(&T[4 * t >> lr][4 * t & (a.rp - 1)]) = a.s * v;
    }
    if (t < b_n) Bs[t >> lr][t & (a.rp - 1)] = bv;
    for (int i = t + NT; i < b_n; i += NT) Bs[i >> lr][i & (a.rp - 1)] = b_at(i);
  };
  static_assert(NT >= 16 * 128 / 4, "a thread for every four values of T");
  if constexpr (NB == 1) {
    ask();
    __builtin_amdgcn_sched_barrier(0);
  }
  for (int kb0 = wave; kb0 < kb_n || kb0 == wave; kb0 += WAVES * U) {
    uint4 x[U][2], w[U][NB][2];
    int sx[U], sw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int kb = kb0 + u * WAVES, k = kb * kFp8Block + 32 * lg;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bool ok = k + 16 * h < K;
#pragma unroll
        for (int b = 0; b < NB; ++b)
          w[u][b][h] = buf_load16(wr, ok ? (b * 16 + l16) * K + k + 16 * h : kOutOfRange);
        x[u][h] = buf_load16(xr, ok ? l16 * K + k + 16 * h : kOutOfRange);
      }
      const int kc = min(kb, kb_n - 1);
      sx[u] = xs[kc];
      sw[u] = ws[kc];
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (NB == 1)
      if (kb0 == wave) stage();
    // lane l has values 32 (l / 16) ... + 31 of a block; the products take eight of
    // every lane at a time
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint4 xv[2], wv[2];
        fp8_to_bf16(x[u][h], sx[u], xv);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          fp8_to_bf16(w[u][b][h], sw[u], wv);
          acc[b] = mfma16(wv[0], xv[0], acc[b]);
          acc[b] = mfma16(wv[1], xv[1], acc[b]);
        }
      }
  }
#pragma unroll
  for (int b = 0; b < NB; ++b) red[wave][b][lane] = acc[b];
  if constexpr (NB > 1) {
    ask();
    stage();
  }
  __syncthreads();
  for (int e = t; e < 16 * NB * M; e += NT) {
    const int nl = e % (16 * NB), m = e / (16 * NB), n = n0 + nl;
    if (n >= N) continue;
    const int b = nl / 16, src = (nl % 16) / 4 * 16 + m, i = nl % 4;
    float v = red[0][b][src][i];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += red[w][b][src][i];
    const size_t at = (size_t)m * N + n;
    if (a.y_off) store_elem(a.y_off, a.y_type, at, v);
    if (!a.y_on) continue;
    if (lora) {
      float u = 0.f;
      for (int j = 0; j < a.r; ++j) u = fmaf(T[m][j], bf16_to_f32(Bs[nl][j]), u);
      v += u;
    }
    store_elem(a.y_on, a.y_type, at, v);
  }
}

template <int NB, int WAVES>
void launch_stream_as(const Fp8LinearArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL((fp8_stream_kernel<NB, WAVES>), dim3((a.N + 16 * NB - 1) / (16 * NB)), dim3(WAVES * 64), 0, stream, a);
}
// Sixteen rows of W a workgroup; thirty-two where that leaves two workgroups a CU and more
// than four rows of x, which every workgroup reads, count.  us at rank 16, x quantized in
// the call, <1, 8> and <2, 8>: 16 x 32000 x 4096 46.0 and 39.4, 8 x 32000 x 4096 37.7 and 34.9,
// 12 x 16400 x 4096 27.6 and 25.4; the product alone: 8 x 4096 x 4096 6.8 and 7.8, 8 x 11008 x
// 4096 13.4 and 15.4, 1 x 32000 x 4096 25.3 and 26.7.  Four waves or sixteen, or 64 rows:
// slower at most sizes, by up to a half.
void launch_stream(const Fp8LinearArgs& a, hipStream_t stream) {
  if (a.N > 16384 && a.M > 4)
    launch_stream_as<2, 8>(a, stream);
  else
    launch_stream_as<1, 8>(a, stream);
}

// ------------------------------------------------------------------ tiles

struct GemmArgs {
  Fp8LinearArgs a;
  int ntm, ntn, total;
  int vec;    // outputs in 16-byte stores
  int bvec;   // B in 16-byte loads
  int64_t xs_bytes, ws_bytes;
  int nsplit, per;  // K in nsplit parts of `per` slabs (PART, JOIN)
};

// WHOLE: a tile's outputs.  PART: the base product of one part of K (blockIdx.y) to
// a.split, [nsplit][M][N] fp32; JOIN: their sum in the order of K, and what WHOLE does
// after its own.
enum Phase { WHOLE, PART, JOIN };

// TM x TN tile, WM x WN sub-tile a wave, KS waves a sub-tile (each takes its share
// of every slab), slabs of BK values of K in a ring of NS; four more waves copy.
// WIDE: bf16 products, in steps of 32 values of K, into fp32 outputs; else 8-bit ones, in
// steps of 64, into bf16.  WPC workgroups share a CU.
template <bool WIDE_, int TM_, int TN_, int WM_, int WN_, int KS_, int BK_, int NS_, int WPC_ = 1>
struct Tile {
  static constexpr bool WIDE = WIDE_;
  static constexpr int WPC = WPC_;
  static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, KS = KS_, BK = BK_, NS = NS_;
  static constexpr int NWN = TN / WN, NMW = TM / WM * NWN * KS, NW = NMW + 4, NT = NW * 64;
  static constexpr int MT = WM / 32, NTL = WN / 32, NQ = MT * NTL;
  static constexpr int CPR = BK / 16;             // 16-byte chunks of an LDS row
  static constexpr int RPB = 64 / CPR;            // rows of a copy instruction
  static constexpr int XJ = TM / RPB / 4, WJ = TN / RPB / 4, DPW = XJ + WJ;  // copies per copy wave and slab
  static constexpr int STAGE = (TM + TN) * CPR;   // uint4
  static constexpr int STEP = WIDE ? 32 : 64;
  static constexpr int SPW = BK / STEP / KS;           // steps per wave and slab
  static constexpr int RD = STEP / 32;                 // 16-byte reads a lane and row in a step
  static constexpr int OLD = TN + 4;                   // row of the output tile in LDS (fp32, in values)
  static constexpr int OUT = KS * TM * OLD * 4;        // bytes of the KS partial sums of it
  // rows of s T (fp32, or two bf16 parts) and of B, 16 bytes apart from the next, at padded rank rp
  static constexpr int lora_bytes(int rp) { return TM * (4 * rp + 16) + TN * (2 * rp + 16); }
  static constexpr size_t cmax(size_t x, size_t y) { return x > y ? x : y; }
  static constexpr int MASK = TM * TN / 8;             // bytes of dropout's mask, after the rest
  static constexpr size_t LDS = cmax(cmax(size_t(NS) * STAGE * 16, OUT), lora_bytes(128));
  static_assert(TM % (RPB * 4) == 0 && TN % (RPB * 4) == 0 && SPW >= 1 && TN % 8 == 0, "whole copies, steps and groups");
  static_assert(SPW <= 4 && (SPW == 1 || SPW % 2 == 0), "steps listed below");
  static_assert(WN <= kFp8Block && LDS + MASK <= 160 * 1024 / WPC && (NS - 2) * DPW < 64, "one scale a sub-tile and slab; LDS; waits");
};

template <int V>
using IC = std::integral_constant<int, V>;

// s_waitcnt for at most N vector-memory operations in flight.
template <int N>
__device__ __forceinline__ void wait_vm() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (0xF << 8) | (((N >> 4) & 3) << 14));
  asm volatile("" ::: "memory");
}
// LDS operations of this wave complete, then the workgroup barrier.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Four scale bytes from `at` on (at < bytes); bytes past the array read as
// anything.
__device__ __forceinline__ uint32_t load_scales(const uint8_t* p, int64_t at, int64_t bytes) {
  if (bytes < 4) {
    uint32_t v = 0;
    for (int i = 0; i < 4; ++i)
      if (at + i < bytes) v |= (uint32_t)p[at + i] << (8 * i);
    return v;
  }
  const int64_t from = at < bytes - 4 ? at : bytes - 4;
  uint32_t v;
  __builtin_memcpy(&v, p + from, 4);
  return v >> (8 * (int)(at - from));
}

// MASK: the update goes through dropout's mask.
template <class G, bool MASK, Phase PH>
__global__ __launch_bounds__(G::NT, G::NT / 256 * G::WPC) void fp8_gemm_kernel(GemmArgs g) {
  constexpr int TM = G::TM, TN = G::TN, WM = G::WM, WN = G::WN, KS = G::KS, BK = G::BK, NS = G::NS;
  constexpr int MT = G::MT, NTL = G::NTL, NQ = G::NQ, SPW = G::SPW;
  constexpr int CPR = G::CPR, RPB = G::RPB, RD = G::RD;
  __shared__ uint4 sm[(G::LDS + (MASK ? G::MASK : 0)) / 16];
  const Fp8LinearArgs& a = g.a;
  const int M = a.M, N = a.N, K = a.K, kb_n = (K + kFp8Block - 1) / kFp8Block;
  const int t = threadIdx.x, lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int l32 = lane & 31, lh = lane >> 5;

  // Consecutive workgroups go to consecutive XCDs; each takes a contiguous range
  // of an order that walks up to 8 row tiles per column tile.
  int tmi, tni;
  {
    const int q = g.total >> 3, rem = g.total & 7, xcd = blockIdx.x & 7;
    const int lid = xcd * q + min(xcd, rem) + (blockIdx.x >> 3);
    const int per_group = 8 * g.ntn, group = lid / per_group, first_m = group * 8, gsize = min(g.ntm - first_m, 8);
    const int in = lid - group * per_group;
    tmi = first_m + in % gsize;
    tni = in / gsize;
  }
  const int m0 = __builtin_amdgcn_readfirstlane(tmi * TM), n0 = __builtin_amdgcn_readfirstlane(tni * TN);
  // slabs [kt0, nkt) of this workgroup
  const int kt0 = PH == PART ? (int)blockIdx.y * g.per : 0;
  const int nkt = PH == JOIN ? 0 : PH == PART ? min((K + BK - 1) / BK, kt0 + g.per) : (K + BK - 1) / BK;

  // LDS chunk of (row, 16-byte chunk c): c is XOR-ed with bits of the row, so that
  // 16 consecutive rows' chunks c lie in different banks.  W's rows follow x's.
  auto swz = [](int row) __attribute__((always_inline)) { return CPR == 8 ? (row >> 1) & 7 : row & 15; };
  auto lds_idx = [&](int row, int c) __attribute__((always_inline)) { return row * CPR + (c ^ swz(row)); };

  const int mw = wave < G::NMW ? wave : 0;
  const int kg = mw % KS, wt = mw / KS, wr = wt / G::NWN, wc = wt % G::NWN;

  // ---------------------------------------------------------------- epilogue
  // The accumulators go to LDS as fp32 rows, one copy for each of the KS waves of a
  // sub-tile; all waves then add the copies up and store whole rows (straight from
  // the accumulators a store writes 16-byte pieces of 32 rows: 2048 x 11008 x 4096 into
  // two bf16 outputs 153 us, this way 132).
  float* const out = reinterpret_cast<float*>(sm);
  // (this thread's number once more, as a value of the epilogue's own: addresses
  // formed from it are not kept in registers through the main loop)
  int te = t;
  constexpr int OLD = G::OLD;
  auto put = [&](const f32x16_t (&acc)[MT][NTL]) __attribute__((always_inline)) {
    // acc[mi][ni][4 i + e]: row mi 32 + l32, column ni 32 + 8 i + 4 lh + e
    const int l32 = te & 31, lh = te >> 5 & 1;
    float* o = out + (kg * TM + wr * WM + l32) * OLD + wc * WN + 4 * lh;
#pragma unroll
    for (int mi = 0; mi < MT; ++mi)
#pragma unroll
      for (int ni = 0; ni < NTL; ++ni)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x16_t& v = acc[mi][ni];
          *reinterpret_cast<f32x4_t*>(o + mi * 32 * OLD + ni * 32 + 8 * i) =
              f32x4_t{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
        }
  };
  // A thread's groups of consecutive columns, 16 bytes of the output: f(values, row, column).
  constexpr int w = G::WIDE ? 4 : 8, per_row = TN / w, groups = TM * per_row, rounds = (groups + G::NT - 1) / G::NT;
  // JOIN: the base product of these groups, from its parts (N % 4 == 0: four at a time)
  f32x4_t base[PH == JOIN ? rounds : 1][w / 4];
  if constexpr (PH == JOIN) {
    const size_t stride = (size_t)M * N;
#pragma unroll
    for (int i = 0; i < rounds; ++i) {
      const int at = i * G::NT + t, row = at / per_row, col = at % per_row * w;
      const bool ok = at < groups && m0 + row < M;
      const float* p = a.split + (size_t)(m0 + row) * N + n0 + col;
#pragma unroll
      for (int q = 0; q < w / 4; ++q) base[i][q] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
      for (int k = 0; k < g.nsplit; ++k, p += stride)
#pragma unroll
        for (int q = 0; q < w / 4; ++q) {
          if (N % 4 == 0) {
            if (ok && n0 + col + 4 * q < N) base[i][q] += *reinterpret_cast<const f32x4_t*>(p + 4 * q);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (ok && n0 + col + 4 * q + e < N) base[i][q][e] += p[4 * q + e];
          }
        }
    }
  }
  auto each = [&](auto f) __attribute__((always_inline)) {
    constexpr int un = PH == JOIN ? rounds : 4;
#pragma unroll un
    for (int i = 0; i < rounds; ++i) {
      const int at = i * G::NT + te;
      if (groups % G::NT != 0 && at >= groups) break;
      const int row = at / per_row, col = at % per_row * w;
      float v[w];
#pragma unroll
      for (int q = 0; q < w / 4; ++q) {
        f32x4_t s = *reinterpret_cast<const f32x4_t*>(out + row * OLD + col + 4 * q);
#pragma unroll
        for (int k = 1; k < KS; ++k)
          s += *reinterpret_cast<const f32x4_t*>(out + (k * TM + row) * OLD + col + 4 * q);
        if constexpr (PH == JOIN) s += base[i][q];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * q + e] = s[e];
      }
      f(v, row, col);
    }
  };
  auto store = [&](void* y, const float* v, int row, int col) __attribute__((always_inline)) {
    if (m0 + row >= M || n0 + col >= N) return;
    const size_t at = (size_t)(m0 + row) * N + n0 + col;
    if (g.vec) {
      if constexpr (w == 4)
        *reinterpret_cast<f32x4_t*>(static_cast<float*>(y) + at) = f32x4_t{v[0], v[1], v[2], v[3]};
      else
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(y) + at) =
            make_uint4(f32_to_bf16_pair(v[0], v[1]), f32_to_bf16_pair(v[2], v[3]), f32_to_bf16_pair(v[4], v[5]),
                       f32_to_bf16_pair(v[6], v[7]));
    } else {
#pragma unroll
      for (int e = 0; e < w; ++e)
        if (n0 + col + e < N) store_elem(y, w == 4 ? kF32 : kBf16, at + e, v[e]);
    }
  };
  // The rows of s T and those of B, zero padded to rp, to LDS: s T as it is where it goes
  // into fp32, else as its two parts [hi rp | lo rp].
  const int rp = a.rp, lrp = 31 - __builtin_clz(rp | 1), ldt = 2 * rp + 8, ldb = rp + 8;  // (in 16 bits)
  uint16_t* const Ts = reinterpret_cast<uint16_t*>(sm);
  uint16_t* const Bs = Ts + TM * ldt;
  // Four values of s T, of a tile's row.
  auto put_t = [&](int row, int j, const f32x4_t& v) __attribute__((always_inline)) {
    if constexpr (G::WIDE) {
      *reinterpret_cast<f32x4_t*>(Ts + row * ldt + 2 * j) = v;
    } else {
      uint2 hi, lo;
      two_parts(v[0], v[1], hi.x, lo.x);
      two_parts(v[2], v[3], hi.y, lo.y);
      *reinterpret_cast<uint2*>(Ts + row * ldt + j) = hi;
      *reinterpret_cast<uint2*>(Ts + row * ldt + rp + j) = lo;
    }
  };
  const int rows = min(TM, M - m0), cols = min(TN, N - n0);
  // By the 256 threads of the copy waves.  At padded rank 16, the usual one, the loads
  // come ahead (`ahead`), while the last products run and y_off is stored.
  struct Ahead {
    f32x4_t t[TM * 4 > 256 ? TM * 4 / 256 : 1][kStagedChunks];
    uint4 b[TN * 2 > 256 ? TN * 2 / 256 : 1];
  };
  const bool ahead = a.y_on && rp == 16 && !a.ts && g.bvec && a.nch <= kStagedChunks;
  auto load_ahead = [&](Ahead& u, int tc) __attribute__((always_inline)) {
    const size_t stride = (size_t)M * 16;
#pragma unroll
    for (int i = 0; i * 256 < TM * 4; ++i) {
      const int e = i * 256 + tc, row = e / 4, j = e % 4 * 4;
#pragma unroll
      for (int c = 0; c < kStagedChunks; ++c) {
        u.t[i][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (row < rows && c < a.nch)
          u.t[i][c] = *reinterpret_cast<const f32x4_t*>(a.part + (size_t)(m0 + row) * 16 + j + c * stride);
      }
    }
#pragma unroll
    for (int i = 0; i * 256 < TN * 2; ++i) {
      const int e = i * 256 + tc, row = e / 2, j = e % 2 * 8;
      u.b[i] = make_uint4(0, 0, 0, 0);
      if (row < cols && j < a.r) u.b[i] = *reinterpret_cast<const uint4*>(a.B + (size_t)(n0 + row) * a.ldb + j);
    }
  };
  auto put_ahead = [&](const Ahead& u, int tc) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i * 256 < TM * 4; ++i) {
      const int e = i * 256 + tc;
      f32x4_t v = u.t[i][0];
#pragma unroll
      for (int c = 1; c < kStagedChunks; ++c) v += u.t[i][c];
      if (TM * 4 % 256 == 0 || e < TM * 4) put_t(e / 4, e % 4 * 4, a.s * v);
    }
#pragma unroll
    for (int i = 0; i * 256 < TN * 2; ++i) {
      const int e = i * 256 + tc;
      if (TN * 2 % 256 == 0 || e < TN * 2) *reinterpret_cast<uint4*>(Bs + e / 2 * ldb + e % 2 * 8) = u.b[i];
    }
  };
  auto put_update = [&](int tc) __attribute__((always_inline)) {
    if (a.ts) {
      const uint16_t* const ts = static_cast<const uint16_t*>(a.ts);
#pragma unroll 8
      for (int e = tc; e < TM * rp / 4; e += 256) {  // 16 bytes each
        const int row = e >> (lrp - 2), c = (e & (rp / 4 - 1)) * 8;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (row < rows) v = *reinterpret_cast<const uint4*>(ts + (size_t)(m0 + row) * 2 * rp + c);
        *reinterpret_cast<uint4*>(Ts + row * ldt + c) = v;
      }
    } else {
      const size_t stride = (size_t)M * rp;
#pragma unroll 4
      for (int e = tc; e < TM * rp / 4; e += 256) {
        const int row = e >> (lrp - 2), j = (e & (rp / 4 - 1)) * 4;
        f32x4_t v = {0.f, 0.f, 0.f, 0.f};
        if (row < rows) {
          const float* p = a.part + (size_t)(m0 + row) * rp + j;
          for (int c = 0; c < a.nch; ++c) v += *reinterpret_cast<const f32x4_t*>(p + c * stride);
        }
        put_t(row, j, a.s * v);
      }
    }
    if (g.bvec) {
#pragma unroll 8
      for (int e = tc; e < TN * rp / 8; e += 256) {
        const int row = e >> (lrp - 3), j = (e & (rp / 8 - 1)) * 8;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (row < cols && j < a.r) v = *reinterpret_cast<const uint4*>(a.B + (size_t)(n0 + row) * a.ldb + j);
        *reinterpret_cast<uint4*>(Bs + row * ldb + j) = v;
      }
    } else {
#pragma unroll 8
      for (int e = tc; e < TN * rp; e += 256) {
        const int row = e >> lrp, j = e & (rp - 1);
        Bs[row * ldb + j] = row < cols && j < a.r ? a.B[(size_t)(n0 + row) * a.ldb + j] : (uint16_t)0;
      }
    }
  };
  // Dropout's mask of the update (N % 8 == 0 here): a bit a column, a byte a block of
  // the generator.  The copy waves make it while the products run.
  uint8_t* const mask = reinterpret_cast<uint8_t*>(sm) + G::LDS;
  // s T B^T onto the accumulators (of the first of a sub-tile's KS waves): rows of B
  // against those of the parts of s T: three into fp32, all that s T holds, made on the way
  // in; two into bf16, whose own rounding is two hundred times theirs.  us with two and
  // three into fp32: 333 x 4096 x 11008 at rank 16 56.0 and 56.2, 1024 x 4096 x 4096 at 128 60.9 and
  // 63.4; dx of 2048 x 4096 x 4096 under a mask, with dA and dB, at 16 100.8 and 102.0, at 128 176.6
  // and 180.5.  (Three planes in LDS, split as they are put there: 1 to 2% slower still at
  // rank 128, for the largest tile takes its columns in two halves then.)
  constexpr int NP = G::WIDE ? 3 : 2;
  auto add_update = [&](f32x16_t (&acc)[MT][NTL]) __attribute__((always_inline)) {
    if (KS > 1 && kg != 0) return;
    const int l32 = te & 31, lh = te >> 5 & 1;
    const uint16_t* const tr = Ts + (wr * WM + l32) * ldt + (G::WIDE ? 16 : 8) * lh;
    const uint16_t* const br = Bs + (wc * WN + l32) * ldb + 8 * lh;
    auto parts = [&](int mi, int k0, uint4 (&p)[NP]) __attribute__((always_inline)) {
      const uint16_t* const row = tr + mi * 32 * ldt;
      if constexpr (G::WIDE) {
        const f32x4_t a = *reinterpret_cast<const f32x4_t*>(row + 2 * k0);
        const f32x4_t b = *reinterpret_cast<const f32x4_t*>(row + 2 * k0 + 8);
        uint32_t v[4][3];
        three_parts(a[0], a[1], v[0]);
        three_parts(a[2], a[3], v[1]);
        three_parts(b[0], b[1], v[2]);
        three_parts(b[2], b[3], v[3]);
#pragma unroll
        for (int n = 0; n < NP; ++n) p[n] = make_uint4(v[0][n], v[1][n], v[2][n], v[3][n]);
      } else {
#pragma unroll
        for (int n = 0; n < NP; ++n) p[n] = *reinterpret_cast<const uint4*>(row + n * rp + k0);
      }
    };
    if constexpr (!MASK) {
      for (int k0 = 0; k0 < rp; k0 += 16) {
        uint4 bf[NTL];
#pragma unroll
        for (int ni = 0; ni < NTL; ++ni) bf[ni] = *reinterpret_cast<const uint4*>(br + ni * 32 * ldb + k0);
#pragma unroll
        for (int mi = 0; mi < MT; ++mi) {
          uint4 p[NP];
          parts(mi, k0, p);
#pragma unroll
          for (int n = 0; n < NP; ++n)
#pragma unroll
            for (int ni = 0; ni < NTL; ++ni) acc[mi][ni] = mfma32(bf[ni], p[n], acc[mi][ni]);
        }
      }
    } else {
      // blocks whose update is in registers at a time
      constexpr int PAIR = G::WIDE && NTL > 1 ? 2 : 1;
#pragma unroll
      for (int mi = 0; mi < MT; ++mi)
#pragma unroll
        for (int b0 = 0; b0 < NTL; b0 += PAIR) {
          f32x16_t L[PAIR];
#pragma unroll
          for (int q = 0; q < PAIR; ++q)
#pragma unroll
            for (int e = 0; e < 16; ++e) L[q][e] = 0.f;
          for (int k0 = 0; k0 < rp; k0 += 16) {
            uint4 p[NP];
            parts(mi, k0, p);
#pragma unroll
            for (int q = 0; q < PAIR; ++q) {
              const uint4 bf = *reinterpret_cast<const uint4*>(br + (b0 + q) * 32 * ldb + k0);
#pragma unroll
              for (int n = 0; n < NP; ++n) L[q] = mfma32(bf, p[n], L[q]);
            }
          }
          // a block's four bytes of this lane's row; elements 4 i + e: bit 4 lh + e of byte i
#pragma unroll
          for (int q = 0; q < PAIR; ++q) {
            const int at = ((wr * WM + mi * 32 + l32) * TN + wc * WN + (b0 + q) * 32) / 8;
            const uint32_t bits = *reinterpret_cast<const uint32_t*>(mask + at) >> (4 * lh);
#pragma unroll
            for (int e = 0; e < 16; ++e)
              acc[mi][b0 + q][e] += (bits >> (8 * (e / 4) + e % 4)) & 1 ? L[q][e] * a.keep : 0.f;
          }
          __builtin_amdgcn_sched_barrier(0);  // (PAIR blocks at a time)
        }
    }
  };
  // By the role of the wave: do_stage is a copy wave's, the others a matrix wave's.
  auto finish = [&](auto do_stage, auto do_put, auto do_add) __attribute__((always_inline)) {
    asm volatile("" : "+v"(te));
    if constexpr (PH == PART) {
      do_put();
      __syncthreads();
      float* const part = a.split + (size_t)blockIdx.y * M * N;
      each([&](const float* v, int row, int col) __attribute__((always_inline)) {
        if (m0 + row >= M) return;
        float* p = part + (size_t)(m0 + row) * N + n0 + col;
#pragma unroll
        for (int q = 0; q < w / 4; ++q) {
          if (N % 4 == 0) {
            if (n0 + col + 4 * q < N)
              *reinterpret_cast<f32x4_t*>(p + 4 * q) = f32x4_t{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (n0 + col + 4 * q + e < N) p[4 * q + e] = v[4 * q + e];
          }
        }
      });
      return;
    }
    const bool lora = a.y_on && rp > 0;
    if (a.y_off || !lora) {
      do_put();
      __syncthreads();
      each([&](const float* v, int row, int col) __attribute__((always_inline)) {
        if (a.y_off) store(a.y_off, v, row, col);
        if (a.y_on && !lora) store(a.y_on, v, row, col);
      });
      if (!lora) return;
      __syncthreads();
    }
    do_stage();
    __syncthreads();
    do_add();
    __syncthreads();
    do_put();
    __syncthreads();
    each([&](const float* v, int row, int col) __attribute__((always_inline)) { store(a.y_on, v, row, col); });
  };

  if (wave >= G::NMW) {
    // -------------------------------------------------------------- copy waves
    const int cw = wave - G::NMW;
    const int rl = lane / CPR;
    const int c = (lane % CPR) ^ swz(cw * RPB + rl);  // (the same for every block of rows cw + 4 j)
    const i32x4_t xr = make_rsrc_raw(a.xq + (size_t)m0 * K, (uint32_t)min(TM, M - m0) * K);
    const i32x4_t wrs = make_rsrc_raw(a.wq + (size_t)n0 * K, (uint32_t)min(TN, N - n0) * K);
    auto issue = [&](int stage, int kt) __attribute__((always_inline)) {
      const int k = kt * BK + c * 16;
      const bool ok = k < K && (PH != PART || kt < nkt);
#pragma unroll
      for (int j = 0; j < G::XJ; ++j) {
        const int row = (cw + 4 * j) * RPB;
        dma16(xr, sm + stage * G::STAGE + row * CPR, ok ? (row + rl) * K + k : kOutOfRange);
      }
#pragma unroll
      for (int j = 0; j < G::WJ; ++j) {
        const int row = (cw + 4 * j) * RPB;
        dma16(wrs, sm + stage * G::STAGE + (TM + row) * CPR, ok ? (row + rl) * K + k : kOutOfRange);
      }
    };
    const int tc = t - G::NMW * 64;
    int next = tc;  // of this thread's bytes of the mask
    const uint64_t seed = MASK ? a.rng[0] : 0, offset = MASK ? a.rng[1] : 0;
    auto put_mask = [&]() __attribute__((always_inline)) {
      if (next >= TM * TN / 8) return;
      const int row = next / (TN / 8), col = next % (TN / 8) * 8;
      const uint4 bits = dropout_words(seed, offset, ((uint64_t)(m0 + row) * N + n0 + col) >> 3);
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) m |= dropout_keeps(bits, j, a.drop) ? 1u << j : 0u;
      mask[next] = (uint8_t)m;
      next += 256;
    };
    // slabs past the last read zeros, so that the waits count the same throughout
    if constexpr (PH != JOIN) {
#pragma unroll
      for (int s = 0; s < NS; ++s) issue(s, kt0 + s);
      wait_vm<(NS - 1) * G::DPW < 63 ? (NS - 1) * G::DPW : 63>();
      lds_barrier();  // the first slab is in LDS
    }
    int stage = 0;
    for (int kt = kt0; kt < nkt; ++kt) {
      wait_vm<(NS - 2) * G::DPW>();
      lds_barrier();  // slab kt + 1 has landed, slab kt is in registers everywhere
      issue(stage, kt + NS);
      if constexpr (MASK) put_mask();
      stage = stage + 1 == NS ? 0 : stage + 1;
    }
    if constexpr (MASK)
      while (next < TM * TN / 8) put_mask();
    wait_vm<0>();
    Ahead up;
    if (ahead) load_ahead(up, tc);
    lds_barrier();  // every copy has landed, every wave is done with the ring
    finish([&] { ahead ? put_ahead(up, tc) : put_update(tc); }, [] {}, [] {});
  } else {
    // -------------------------------------------------------------- matrix waves
    f32x16_t acc[MT][NTL];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NTL; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    struct Frag {
      uint4 w[NTL][RD], x[MT][RD];
    };
    // Two sets, the next step's reads spread over this step's products; on the largest
    // sub-tile one, where a fragment is read again right after its last use (two sets
    // next to its accumulators spill), four products ahead of the next.
    constexpr bool ONE = NQ >= 8;
    Frag F[ONE ? 1 : 2];
    constexpr int NR = RD * (NTL + MT);
    // the r-th 16-byte read of step st (of this wave's) of a stage: W rows as the A
    // operand, x rows as the B operand
    auto read = [&](Frag& f, int stage, int st, int r) __attribute__((always_inline)) {
      const uint4* s = sm + stage * G::STAGE;
      const int q = r / RD, h = r % RD, ch = (2 * (kg * SPW + st) + lh) * RD + h;
      if (q < NTL)
        f.w[q][h] = s[lds_idx(TM + wc * WN + q * 32 + l32, ch)];
      else
        f.x[q - NTL][h] = s[lds_idx(wr * WM + (q - NTL) * 32 + l32, ch)];
    };
    auto read_row = [&](Frag& f, int stage, int st, int q) __attribute__((always_inline)) {
#pragma unroll
      for (int h = 0; h < RD; ++h) read(f, stage, st, q * RD + h);
    };
    // scales: four blocks of K at a time, the next four requested ahead
    const uint8_t* const xs = a.xs;
    const uint8_t* const ws = a.ws;
    int64_t xrow[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) xrow[i] = (int64_t)min(m0 + wr * WM + i * 32 + l32, M - 1) * kb_n;
    const int64_t wrow = (int64_t)(min(n0 + wc * WN, N - 1) / kFp8Block) * kb_n;
    uint32_t sx[MT], sxn[MT], sw, swn;
    auto load_four = [&](int kb) __attribute__((always_inline)) {
      kb = min(kb, kb_n - 1);
#pragma unroll
      for (int i = 0; i < MT; ++i) sxn[i] = load_scales(xs, xrow[i] + kb, g.xs_bytes);
      swn = load_scales(ws, wrow + kb, g.ws_bytes);
    };
    int four = -1;  // the four blocks that sx and sw are of
    auto next_four = [&](int f) __attribute__((always_inline)) {
      four = f;
#pragma unroll
      for (int i = 0; i < MT; ++i) sx[i] = sxn[i];
      sw = swn;
      load_four(4 * f + 4);
    };
    const int kb_first = (kt0 * (BK / G::STEP) + kg * SPW) / (kFp8Block / G::STEP);
    if constexpr (PH != JOIN) load_four(kb_first & ~3);
    auto kstep = [&](auto S, const Frag& fc, Frag& fn, int st, int kt) __attribute__((always_inline)) {
      constexpr int sp = decltype(S)::value;
      constexpr bool last = sp == SPW - 1;
      const int kb = (kt * (BK / G::STEP) + kg * SPW + sp) / (kFp8Block / G::STEP);
      if (kb >> 2 != four) next_four(kb >> 2);  // (each four in turn: a slab is no longer)
      const int shift = 8 * (kb & 3);
      // (the second half of a last slab may lie past the scales: zeros times any number)
      const bool past = BK > kFp8Block && kb >= kb_n;
      const int rst = last ? (st + 1 == NS ? 0 : st + 1) : st;
      constexpr int rsp = last ? 0 : sp + 1;
      if constexpr (last) lds_barrier();
      if constexpr (G::WIDE) {
        const int byte = past ? 127 : (sw >> shift) & 0xFF;
        uint4 xv[MT][2];
#pragma unroll
        for (int mi = 0; mi < MT; ++mi) {
          fp8_to_bf16(fc.x[mi][0], past ? 127 : (sx[mi] >> shift) & 0xFF, xv[mi]);
          if constexpr (ONE) read_row(fn, rst, rsp, NTL + mi);
        }
#pragma unroll
        for (int ni = 0; ni < NTL; ++ni) {
          uint4 v[2];
          fp8_to_bf16(fc.w[ni][0], byte, v);
#pragma unroll
          for (int mi = 0; mi < MT; ++mi)
#pragma unroll
            for (int h = 0; h < 2; ++h) acc[mi][ni] = mfma32(v[h], xv[mi][h], acc[mi][ni]);
          if constexpr (ONE) {
            read_row(fn, rst, rsp, ni);
          } else {
#pragma unroll
            for (int r = ni * NR / NTL; r < (ni + 1) * NR / NTL; ++r) read(fn, rst, rsp, r);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      } else {
#pragma unroll
        for (int m = 0; m < NQ; ++m) {
          const int mi = m / NTL, ni = m % NTL;
          acc[mi][ni] = mfma32_fp8(fc.w[ni][0], fc.w[ni][RD - 1], fc.x[mi][0], fc.x[mi][RD - 1], acc[mi][ni],
                                   past ? 127 : (int)(sw >> shift), past ? 127 : (int)(sx[mi] >> shift));
          if constexpr (ONE) {
            if (mi == MT - 1) read_row(fn, rst, rsp, ni);
            if (ni == NTL - 1) read_row(fn, rst, rsp, NTL + mi);
          } else {
#pragma unroll
            for (int r = m * NR / NQ; r < (m + 1) * NR / NQ; ++r) read(fn, rst, rsp, r);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    };
    if constexpr (PH != JOIN) {
      lds_barrier();  // the first slab is in LDS
#pragma unroll
      for (int r = 0; r < NR; ++r) read(F[0], 0, 0, r);
    }
    // Past the last slab the reads fill registers that are never used.
    constexpr int UN = SPW % 2 && !ONE ? 2 : 1;  // slabs until the two fragment sets are back in place
    int stage = 0;
    for (int kt = kt0; kt < nkt; kt += UN) {
#pragma unroll
      for (int u = 0; u < UN; ++u) {
        if (u > 0 && kt + u >= nkt) break;
        constexpr int one = SPW > 1 ? 1 : 0, two = SPW > 2 ? 2 : 0, three = SPW > 3 ? 3 : 0;
        constexpr int other = ONE ? 0 : 1;
        kstep(IC<0>{}, F[ONE ? 0 : u & 1], F[ONE ? 0 : (u & 1) ^ 1], stage, kt + u);
        if constexpr (SPW > 1) kstep(IC<one>{}, F[other], F[0], stage, kt + u);
        if constexpr (SPW > 2) {
          kstep(IC<two>{}, F[0], F[other], stage, kt + u);
          kstep(IC<three>{}, F[other], F[0], stage, kt + u);
        }
        stage = stage + 1 == NS ? 0 : stage + 1;
      }
    }
    lds_barrier();
    finish([] {}, [&] { put(acc); }, [&] { add_update(acc); });
  }
}

bool at_multiple(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

template <class G, bool MASK, Phase PH>
hipError_t launch_phase(GemmArgs& g, hipStream_t stream) {
  g.ntm = (g.a.M + G::TM - 1) / G::TM;
  g.ntn = (g.a.N + G::TN - 1) / G::TN;
  const int64_t total = (int64_t)g.ntm * g.ntn;
  if (total * G::NT >= (int64_t(1) << 32)) return hipErrorInvalidValue;
  g.total = (int)total;
  hipLaunchKernelGGL((fp8_gemm_kernel<G, MASK, PH>), dim3(g.total, PH == PART ? g.nsplit : 1), dim3(G::NT), 0, stream, g);
  return hipGetLastError();
}
template <class G, Phase PH>
hipError_t launch_masked(GemmArgs& g, hipStream_t stream) {
  return g.a.drop > 0 && g.a.y_on ? launch_phase<G, true, PH>(g, stream) : launch_phase<G, false, PH>(g, stream);
}
template <class G>
hipError_t launch_tile(GemmArgs& g, hipStream_t stream) {
  return launch_masked<G, WHOLE>(g, stream);
}
template <class G>
hipError_t launch_split(GemmArgs& g, const Fp8Plan& p, hipStream_t stream) {
  if (p.split_values(g.a.M, g.a.N) * 4 > g.a.split_bytes) return hipErrorInvalidValue;
  g.per = p.per;
  g.nsplit = p.nsplit;
  const hipError_t e = launch_phase<G, false, PART>(g, stream);
  if (e != hipSuccess) return e;
  return launch_masked<Tile<G::WIDE, 32, 64, 32, 64, 1, 128, 2, 2>, JOIN>(g, stream);
}
template <class G, int I>
hipError_t launch_planned(GemmArgs& g, const Fp8Plan& p, hipStream_t stream) {
  constexpr Fp8TileCost c = kFp8TileCosts[G::WIDE][I];
  static_assert(G::TM == c.tm && G::TN == c.tn && G::BK == c.bk, "the tile that the plan is of");
  if constexpr (c.parts) {
    if (p.nsplit > 1) return launch_split<G>(g, p, stream);
  }
  return launch_tile<G>(g, stream);
}

template <bool WIDE>
hipError_t launch_rows(GemmArgs& g, hipStream_t stream) {
  const Fp8Plan p = fp8_plan(WIDE, g.a.M, g.a.N, g.a.K);
  switch (p.tile) {
    case 0: return launch_planned<Tile<WIDE, 128, 256, 64, 128, 1, 128, 3>, 0>(g, p, stream);
    case 1: return launch_planned<Tile<WIDE, 128, 128, 64, 64, 2, 128, 4>, 1>(g, p, stream);
    case 2: return launch_planned<Tile<WIDE, 64, 128, 64, 64, 2, 128, 6>, 2>(g, p, stream);
    case 3: return launch_planned<Tile<WIDE, 64, 64, 32, 64, 2, 128, 4, 2>, 3>(g, p, stream);
    case 4: return launch_planned<Tile<WIDE, 32, 64, 32, 64, 4, 256, 6>, 4>(g, p, stream);
    default: return launch_planned<Tile<WIDE, 32, 32, 32, 32, 4, 256, 4, 2>, 5>(g, p, stream);
  }
}

template <int RP>
void launch_prep(const Fp8PrepArgs& a, hipStream_t stream) {
  const dim3 grid((a.M + 15) / 16, a.nch), block(P_WAVES * 64);
  if constexpr (RP == 0) {
    hipLaunchKernelGGL((fp8_prep_kernel<0, true, false>), grid, block, 0, stream, a);
  } else {
    if (!a.x)
      hipLaunchKernelGGL((fp8_prep_kernel<RP, false, false>), grid, block, 0, stream, a);
    else if (a.xa == a.x)
      hipLaunchKernelGGL((fp8_prep_kernel<RP, true, false>), grid, block, 0, stream, a);
    else
      hipLaunchKernelGGL((fp8_prep_kernel<RP, true, true>), grid, block, 0, stream, a);
  }
}

}  // namespace

hipError_t launch_fp8_prep(const Fp8PrepArgs& a, hipStream_t stream) {
  switch (a.A ? a.rp : 0) {
    case 0: launch_prep<0>(a, stream); break;
    case 16: launch_prep<16>(a, stream); break;
    case 32: launch_prep<32>(a, stream); break;
    case 64: launch_prep<64>(a, stream); break;
    case 128: launch_prep<128>(a, stream); break;
    default: return hipErrorInvalidValue;
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.ts) return e;
  const size_t blocks = ((size_t)a.M * a.rp / 4 + 255) / 256;
  const int lrp = 31 - __builtin_clz(a.rp);
  if (a.parts)
    hipLaunchKernelGGL((fp8_t_finish_kernel<true>), dim3((unsigned)blocks), dim3(256), 0, stream, a, lrp);
  else
    hipLaunchKernelGGL((fp8_t_finish_kernel<false>), dim3((unsigned)blocks), dim3(256), 0, stream, a, lrp);
  return hipGetLastError();
}

hipError_t launch_fp8_linear(const Fp8LinearArgs& a, hipStream_t stream) {
  if (a.M <= kFewRows && !a.ts) {
    launch_stream(a, stream);
    return hipGetLastError();
  }
  GemmArgs g{};
  g.a = a;
  const int64_t kb = (a.K + kFp8Block - 1) / kFp8Block;
  g.xs_bytes = a.M * kb;
  g.ws_bytes = (int64_t)((a.N + kFp8Block - 1) / kFp8Block) * kb;
  g.vec = a.N % (a.y_type == kF32 ? 4 : 8) == 0 && at_multiple(a.y_off, 16) && at_multiple(a.y_on, 16);
  g.bvec = a.r % 8 == 0 && a.ldb % 8 == 0 && at_multiple(a.B, 16);
  return a.y_type == kF32 ? launch_rows<true>(g, stream) : launch_rows<false>(g, stream);
}

}  // namespace hydra
