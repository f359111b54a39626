// Backward of the LoRA-switchable linear with the base weight frozen (the
// update stage of Hydra-PPO trains only the active adapter, Sec. 3 and
// App. A, Alg. 2).  With y = x W^T + s (x A^T) B^T, T = x A^T and U = dy B:
//   dx = dy W + s U A,   dA = s U^T x,   dB = s dy^T T.
// Steps, all on one stream:
//  1. B^T and A^T, zero padded to the padded rank RP (transpose_pad_kernel,
//     both in one launch);
//  2. the LoRA pre-pass of the forward GEMM (lora_tpre.hip) twice, in one
//     pair of launches: s U from dy against the rows of B^T, s T from x
//     against A, each as bf16 hi and lo parts (row-major for step 3,
//     transposed for step 4); over a weight in 8 bits as three parts for step
//     4, and s U in fp32 for step 3 into an fp32 dx;
//  3. dx by the forward's MFMA GEMM run on (dy, W^T), its LoRA slabs being
//     [hi | lo](s U) against rows of A^T: one pass over W^T, as in the forward
//     (over a weight in 8 bits: fp8_linear.hip);
//  4. dA and dB as sums of outer products over the rows m:
//     out[j][c] = sum_m P[m][j] Q[m][c] with (P, Q) = (s U, x) and (s T, dy),
//     on MFMAs (lora_outer_part_kernel: per row chunk partials, laid out like
//     the output), then the chunks added in chunk order
//     (lora_outer_finish_kernel, one thread per output element); dA and dB
//     share each of the two launches.  Every sum has a fixed order: the results
//     are the same from run to run.
#include <algorithm>

#include "hydra_device.h"
#include "hydra_fp8_plan.h"
#include "hydra_internal.h"

namespace hydra {
namespace {

// ------------------------------------------------------------ transpose_pad
constexpr int TP = 64;  // tile edge

struct TransposeJob {
  const uint16_t* src;  // [R x C]
  uint16_t* dst;        // [Cp x Rp]
  int R, C, Rp, Cp;
  int gx;               // tiles along Cp
};

// dst[c][q] = src[q][c] inside src's [R x C], zero outside, for the 64 x 64
// tile b of the job (tile b % gx along dst's rows, b / gx along its columns).
__device__ __forceinline__ void transpose_tile(const TransposeJob& j, int b) {
  __shared__ uint16_t tile[TP][TP + 2];
  const int c0 = (b % j.gx) * TP, q0 = (b / j.gx) * TP;
  const int lx = threadIdx.x & 63, ly = threadIdx.x >> 6;
  uint16_t v[TP / 4];
#pragma unroll
  for (int i = 0; i < TP / 4; ++i) {
    const int q = q0 + ly + 4 * i, c = c0 + lx;
    v[i] = (q < j.R && c < j.C) ? j.src[(size_t)q * j.C + c] : (uint16_t)0;
  }
#pragma unroll
  for (int i = 0; i < TP / 4; ++i) tile[ly + 4 * i][lx] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < TP / 4; ++i) {
    const int c = c0 + ly + 4 * i, q = q0 + lx;
    if (c < j.Cp && q < j.Rp) j.dst[(size_t)c * j.Rp + q] = tile[lx][ly + 4 * i];
  }
}

// Up to two transposes in one launch: workgroups [0, n0) take job j0's tiles,
// the rest j1's.
__global__ __launch_bounds__(256) void transpose_pad_kernel(TransposeJob j0, int n0, TransposeJob j1) {
  const int b = blockIdx.x;
  if (b < n0)
    transpose_tile(j0, b);
  else
    transpose_tile(j1, b - n0);
}

TransposeJob transpose_job(const uint16_t* src, int R, int C, uint16_t* dst, int Rp, int Cp, int& tiles) {
  TransposeJob j{src, dst, R, C, Rp, Cp, (Cp + TP - 1) / TP};
  tiles = j.gx * ((Rp + TP - 1) / TP);
  return j;
}

// ---------------------------------------------------------- outer products
constexpr int O_WAVES = 4;
constexpr int O_COLS = 256;        // columns per workgroup: 64 per wave, four 16-column MFMA tiles
constexpr int O_KS = 32;           // rows per k-step (the k of one 16x16x32 MFMA)
constexpr int O_LD = O_COLS + 4;   // LDS row stride in bf16 (130 dwords; see outer_part)
constexpr int O_TARGET_WG = 256;   // workgroups the chunking aims for (both products together: twice that)
constexpr int O_MIN_ROWS = 128;    // fewest rows per chunk
constexpr int O_MIN_ROWS_3 = 64;   // ... with three planes of P (which give each chunk more to do)

struct OuterArgs {
  const uint16_t* PT;  // [NP][RP][Mp] bf16: planes of P^T (P = s U or s T), hi and lo, or the next part too
  const uint16_t* Q;   // [M x C] bf16
  float* part;         // [nch x RP x C] (jc) or [nch x C x RP] fp32
  float* out;          // [r x C] (jc) or [C x r] fp32
  int M, Mp, C, RP, r;
  int mch, nch;        // rows per chunk (multiple of O_KS), chunks
  int jc;              // partials and output j-major
  int tiles;           // column tiles of O_COLS
  int vec;             // outer_whole: [C x r] outputs in 16-byte stores
};

// Partial out[j][c] = sum_m P[m][j] Q[m][c] over the rows of one chunk, for
// every j and the 256 columns of one tile (b = tile + tiles * chunk), on
// v_mfma_f32_16x16x32_bf16: A operand = 16 j x 32 m of P^T (its hi plane,
// then its lo plane: ~16 significant bits of P; NP = 3: 24), B operand = 32 m x 16
// columns of Q.  The MFMA wants eight consecutive m per lane, but m is Q's
// row index, so each 32-row slab of Q goes through LDS (row-major, double
// buffered, one barrier per slab) and every lane gathers its column's eight
// values with 16-bit reads.  With a row stride of 130 dwords the four row
// groups of one read land in disjoint bank windows.  Each wave owns 64
// columns and all RP j, so one slab in LDS serves every 16-wide j group.
template <int RP, int NP>
__device__ __forceinline__ void outer_part(const OuterArgs& a, int b) {
  constexpr int JG = RP / 16;
  __shared__ uint16_t qs[2][O_KS][O_LD];
  const int t = threadIdx.x;
  const int lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int l16 = lane & 15, lg = lane >> 4;
  const int tile = b % a.tiles;
  const int ch = b / a.tiles;
  const int c0 = tile * O_COLS;
  const int m_begin = ch * a.mch;
  const int m_end = min(a.M, m_begin + a.mch);
  const int nks = (m_end - m_begin + O_KS - 1) / O_KS;
  // slab copies: thread t moves 16 bytes (8 columns) of rows t / 32 + 8 u
  const int lr = t >> 5, lc = (t & 31) * 8;
  uint4 qv[4];
  auto load = [&](int ks) __attribute__((always_inline)) {
    const int m0 = m_begin + ks * O_KS;
    const int rows = min(O_KS, m_end - m0);
    const __amdgpu_buffer_rsrc_t qrs = make_rsrc(a.Q + (size_t)m0 * a.C, (uint32_t)rows * a.C * 2u);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int row = lr + 8 * u;
      qv[u] = buf_load16(qrs, (row < rows && c0 + lc < a.C) ? (row * a.C + c0 + lc) * 2 : kOutOfRange);
    }
  };
  auto store = [&](int st) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      uint2* d = reinterpret_cast<uint2*>(&qs[st][lr + 8 * u][lc]);
      d[0] = uint2{qv[u].x, qv[u].y};
      d[1] = uint2{qv[u].z, qv[u].w};
    }
  };
  f32x4_t acc[JG][4];
#pragma unroll
  for (int g = 0; g < JG; ++g)
#pragma unroll
    for (int s = 0; s < 4; ++s) acc[g][s] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  // A operands of slab ks (rows 16 g + l16 of the hi and lo planes, m0 + 8 lg .. + 7; Mp is a multiple of 32).
  // Up to padded rank 32 they are requested a slab ahead, so that their latency overlaps the previous slab's
  // MFMAs; at higher ranks the second set of registers would cost occupancy, and they are requested in the slab.
  constexpr bool PF = JG <= 2;
  uint4 ap[JG][NP], an[PF ? JG : 1][NP];
  auto load_p = [&](int ks, uint4 (&d)[JG][NP]) __attribute__((always_inline)) {
    const int m0 = m_begin + ks * O_KS;
#pragma unroll
    for (int g = 0; g < JG; ++g) {
      const uint16_t* p = a.PT + (size_t)(g * 16 + l16) * a.Mp + m0 + 8 * lg;
#pragma unroll
      for (int n = 0; n < NP; ++n) d[g][n] = *reinterpret_cast<const uint4*>(p + n * (size_t)a.RP * a.Mp);
    }
  };
  if constexpr (PF) load_p(0, ap);
  load(0);
  store(0);
  if (nks > 1) load(1);
  __syncthreads();
  for (int ks = 0; ks < nks; ++ks) {
    const int st = ks & 1;
    if constexpr (PF) {
      if (ks + 1 < nks) load_p(ks + 1, an);
    } else {
      load_p(ks, ap);
    }
    // B operands: column wave * 64 + 16 s + l16, rows 8 lg .. 8 lg + 7 of the slab
    uint4 bq[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const uint16_t* q = &qs[st][8 * lg][wave * 64 + s * 16 + l16];
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = (uint32_t)q[(2 * i) * O_LD] | ((uint32_t)q[(2 * i + 1) * O_LD] << 16);
      bq[s] = uint4{w[0], w[1], w[2], w[3]};
    }
#pragma unroll
    for (int g = 0; g < JG; ++g)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
#pragma unroll
        for (int n = 0; n < NP; ++n) acc[g][s] = mfma16(ap[g][n], bq[s], acc[g][s]);
      }
    if (ks + 1 < nks) {
      store(st ^ 1);  // stage st ^ 1 was last read before the previous barrier
      if (ks + 2 < nks) load(ks + 2);
      if constexpr (PF) {
#pragma unroll
        for (int g = 0; g < JG; ++g) {
#pragma unroll
          for (int n = 0; n < NP; ++n) ap[g][n] = an[g][n];
        }
      }
    }
    __syncthreads();
  }

  // acc[g][s] lane l holds out[16 g + 4 lg + e][c0 + 64 wave + 16 s + l16]; partials laid out like the output
  const size_t zc = (size_t)ch * a.RP * a.C;
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const int c = c0 + wave * 64 + s * 16 + l16;
    if (c >= a.C) continue;
#pragma unroll
    for (int g = 0; g < JG; ++g) {
      const int j = g * 16 + 4 * lg;
      if (a.jc) {
#pragma unroll
        for (int e = 0; e < 4; ++e) a.part[zc + (size_t)(j + e) * a.C + c] = acc[g][s][e];
      } else {
        *reinterpret_cast<f32x4_t*>(a.part + zc + (size_t)c * a.RP + j) = acc[g][s];
      }
    }
  }
}

// dA's and dB's partials in one launch: workgroups [0, n0) for o0, the rest o1.
template <int RP, int NP>
__global__ __launch_bounds__(O_WAVES * 64) void lora_outer_part_kernel(OuterArgs o0, int n0, OuterArgs o1) {
  const int b = blockIdx.x;
  if (b < n0)
    outer_part<RP, NP>(o0, b);
  else
    outer_part<RP, NP>(o1, b - n0);
}

constexpr int F_UNROLL = 8;

// out[e] = sum over chunks, in chunk order, of the partials of output element
// e; the loads of F_UNROLL chunks in flight before they are added.
__device__ __forceinline__ void outer_finish(const OuterArgs& a, size_t e) {
  if (e >= (size_t)a.r * a.C) return;
  const size_t src = a.jc ? e : e / a.r * a.RP + e % a.r;  // partial layout [RP x C] or [C x RP]
  const size_t stride = (size_t)a.RP * a.C;
  float v = 0.f;
  int ch = 0;
  for (; ch + F_UNROLL <= a.nch; ch += F_UNROLL) {
    float t[F_UNROLL];
#pragma unroll
    for (int u = 0; u < F_UNROLL; ++u) t[u] = a.part[src + (size_t)(ch + u) * stride];
#pragma unroll
    for (int u = 0; u < F_UNROLL; ++u) v += t[u];
  }
  for (; ch < a.nch; ++ch) v += a.part[src + (size_t)ch * stride];
  a.out[e] = v;
}

// One thread per output element; workgroups [0, n0) for o0, the rest o1.
__global__ __launch_bounds__(256) void lora_outer_finish_kernel(OuterArgs o0, int n0, OuterArgs o1) {
  const int b = blockIdx.x;
  if (b < n0)
    outer_finish(o0, (size_t)b * 256 + threadIdx.x);
  else
    outer_finish(o1, (size_t)(b - n0) * 256 + threadIdx.x);
}

// ... over all rows in one workgroup and 64 columns of the output, with no partial sums: for
// few rows.  Four waves share out the 16-wide j groups, and where those are fewer than
// four the 32-row slabs of a step, whose sums meet in LDS in wave order.
constexpr int W_COLS = 64, W_ROWS = 128, W_LD = W_COLS + 4;
template <int RP>
__device__ __forceinline__ void outer_whole(const OuterArgs& a, int b) {
  constexpr int NP = 3, JG = RP / 16, JW = JG < 4 ? JG : 4, JGW = JG / JW, SW = 4 / JW, SS = W_ROWS / O_KS / SW;
  __shared__ __attribute__((aligned(16))) uint16_t qs[2][W_ROWS][W_LD];
  const int t = threadIdx.x, lane = t & 63, l16 = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6), jw = wave % JW, sw = wave / JW;
  const int c0 = b * W_COLS, nks = a.Mp / O_KS, nst = (a.Mp + W_ROWS - 1) / W_ROWS;
  const int lr = t >> 3, lc = (t & 7) * 8;
  uint4 qv[4];
  auto load = [&](int st) __attribute__((always_inline)) {
    const int m0 = st * W_ROWS, rows = min(W_ROWS, a.M - m0);
    const __amdgpu_buffer_rsrc_t qrs = make_rsrc(a.Q + (size_t)m0 * a.C, (uint32_t)rows * a.C * 2u);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int row = lr + 32 * u;
      qv[u] = buf_load16(qrs, (row < rows && c0 + lc < a.C) ? (row * a.C + c0 + lc) * 2 : kOutOfRange);
    }
  };
  auto store = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      uint2* d = reinterpret_cast<uint2*>(&qs[buf][lr + 32 * u][lc]);
      d[0] = uint2{qv[u].x, qv[u].y};
      d[1] = uint2{qv[u].z, qv[u].w};
    }
  };
  f32x4_t acc[JGW][4];
#pragma unroll
  for (int g = 0; g < JGW; ++g)
#pragma unroll
    for (int s = 0; s < 4; ++s) acc[g][s] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  load(0);
  uint4 ap[SS][JGW][NP];
  auto load_p = [&](int st) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < SS; ++i) {
      const int ks = st * (W_ROWS / O_KS) + i * SW + sw;
#pragma unroll
      for (int g = 0; g < JGW; ++g) {
        const uint16_t* p = a.PT + (size_t)((jw * JGW + g) * 16 + l16) * a.Mp + ks * O_KS + 8 * lg;
#pragma unroll
        for (int n = 0; n < NP; ++n)
          ap[i][g][n] = ks < nks ? *reinterpret_cast<const uint4*>(p + n * (size_t)a.RP * a.Mp) : uint4{0, 0, 0, 0};
      }
    }
  };
  load_p(0);
  store(0);
  if (nst > 1) load(1);
  __syncthreads();
  for (int st = 0; st < nst; ++st) {
    if (st > 0) load_p(st);
#pragma unroll
    for (int i = 0; i < SS; ++i) {
      uint4 bq[4];  // column 16 s + l16, rows 8 lg ... + 7 of the slab
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const uint16_t* q = &qs[st & 1][(i * SW + sw) * O_KS + 8 * lg][s * 16 + l16];
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (uint32_t)q[2 * e * W_LD] | ((uint32_t)q[(2 * e + 1) * W_LD] << 16);
        bq[s] = uint4{w[0], w[1], w[2], w[3]};
      }
#pragma unroll
      for (int g = 0; g < JGW; ++g)
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int n = 0; n < NP; ++n) acc[g][s] = mfma16(ap[i][g][n], bq[s], acc[g][s]);
    }
    if (st + 1 < nst) {
      store((st + 1) & 1);
      if (st + 2 < nst) load(st + 2);
    }
    __syncthreads();
  }
  if constexpr (SW > 1) {
    f32x4_t* red = reinterpret_cast<f32x4_t*>(&qs[0][0][0]);  // [4][JGW][4][64]
    static_assert(4 * JGW * 4 * 64 * 16 <= (int)sizeof(qs), "the sums of the waves");
#pragma unroll
    for (int g = 0; g < JGW; ++g)
#pragma unroll
      for (int s = 0; s < 4; ++s) red[((wave * JGW + g) * 4 + s) * 64 + lane] = acc[g][s];
    __syncthreads();
    if (sw > 0) return;
#pragma unroll
    for (int g = 0; g < JGW; ++g)
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int w = 1; w < SW; ++w) acc[g][s] += red[(((w * JW + jw) * JGW + g) * 4 + s) * 64 + lane];
  }
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const int c = c0 + s * 16 + l16;
    if (c >= a.C) continue;
#pragma unroll
    for (int g = 0; g < JGW; ++g) {
      const int j = (jw * JGW + g) * 16 + 4 * lg;
      if (a.vec) {
        if (j < a.r) *reinterpret_cast<f32x4_t*>(a.out + (size_t)c * a.r + j) = acc[g][s];
        continue;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (j + e < a.r) a.out[a.jc ? (size_t)(j + e) * a.C + c : (size_t)c * a.r + j + e] = acc[g][s][e];
    }
  }
}

template <int RP>
__global__ __launch_bounds__(O_WAVES * 64) void lora_outer_whole_kernel(OuterArgs o0, int n0, OuterArgs o1) {
  const int b = blockIdx.x;
  if (b < n0)
    outer_whole<RP>(o0, b);
  else
    outer_whole<RP>(o1, b - n0);
}

// Whether the outer products take all rows in one workgroup.  The backward over an 8-bit
// weight, us in chunks and in one: 250 x 8192 x 2048 at rank 128 68.0 and 58.0, 128 x 4096 x
// 4096 at 128 52.4 and 42.6, 64 x 4096 x 4096 at 16 30.3 and 28.3, 300 x 11008 x 4096 at 64 85.5 and
// 76.1, 512 x 4096 x 4096 at 16, 64, 128 48.6, 59.6, 73.4 and 48.0, 58.9, 71.4, 1000 x 2048 x 2048 at
// 128 66.3 and 83.4.  (Two planes keep their chunks, and with them their bits.)
bool outer_in_one(int M, int planes) { return planes == 3 && M <= 512; }

// Rows per chunk and number of chunks of the outer products over M rows and
// C columns: enough chunks for about O_TARGET_WG workgroups, each chunk a
// multiple of O_KS rows and at least O_MIN_ROWS (by which chunk the sums are joined
// is part of the result: three planes have chunks of their own.  The backward over an
// 8-bit weight, us with chunks of at least 128, 64, 32 rows: 1000 x 2048 x 2048 at 128
// 70.1, 66.8, 75.3; with two planes and 128 rows 64.0).
void outer_chunks(int M, int C, int planes, int& mch, int& nch) {
  const int64_t tiles = (C + O_COLS - 1) / O_COLS;
  const int64_t want = std::max<int64_t>(1, (O_TARGET_WG + tiles - 1) / tiles);
  int64_t rows = (M + want - 1) / want;
  rows = std::max<int64_t>(planes == 3 ? O_MIN_ROWS_3 : O_MIN_ROWS, (rows + O_KS - 1) / O_KS * O_KS);
  mch = (int)rows;
  nch = (int)((M + rows - 1) / rows);
}

int padded_rows(int M) { return (M + O_KS - 1) / O_KS * O_KS; }

OuterArgs outer_job(const uint16_t* PT, const uint16_t* Q, int M, int C, int rp, int r, int planes, float* part,
                    float* out, bool jc, int& parts, int& finishes) {
  OuterArgs o{PT, Q, part, out, M, padded_rows(M), C, rp, r, 0, 0, jc ? 1 : 0, (C + O_COLS - 1) / O_COLS};
  o.vec = !jc && r % 4 == 0 && (reinterpret_cast<uintptr_t>(out) & 15) == 0;
  outer_chunks(M, C, planes, o.mch, o.nch);
  parts = outer_in_one(M, planes) ? (C + W_COLS - 1) / W_COLS : o.tiles * o.nch;
  finishes = (int)(((size_t)r * C + 255) / 256);
  return o;
}

template <int RP>
void launch_outer_rp(const OuterArgs& o0, int p0, const OuterArgs& o1, int p1, int M, int planes,
                     hipStream_t stream) {
  const dim3 grid(p0 + p1), block(O_WAVES * 64);
  if (outer_in_one(M, planes))
    hipLaunchKernelGGL((lora_outer_whole_kernel<RP>), grid, block, 0, stream, o0, p0, o1);
  else if (planes == 3)
    hipLaunchKernelGGL((lora_outer_part_kernel<RP, 3>), grid, block, 0, stream, o0, p0, o1);
  else
    hipLaunchKernelGGL((lora_outer_part_kernel<RP, 2>), grid, block, 0, stream, o0, p0, o1);
}

hipError_t launch_outer(const OuterArgs& o0, int p0, int f0, const OuterArgs& o1, int p1, int f1, int rp,
                        int M, int planes, hipStream_t stream) {
  switch (rp) {
    case 16: launch_outer_rp<16>(o0, p0, o1, p1, M, planes, stream); break;
    case 32: launch_outer_rp<32>(o0, p0, o1, p1, M, planes, stream); break;
    case 64: launch_outer_rp<64>(o0, p0, o1, p1, M, planes, stream); break;
    case 128: launch_outer_rp<128>(o0, p0, o1, p1, M, planes, stream); break;
    default: return hipErrorInvalidValue;
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || outer_in_one(M, planes)) return e;
  hipLaunchKernelGGL(lora_outer_finish_kernel, dim3(f0 + f1), dim3(256), 0, stream, o0, f0, o1);
  return hipGetLastError();
}

// ------------------------------------------------------- workspace layout
size_t up256(size_t v) { return (v + 255) / 256 * 256; }

struct BwdLayout {
  size_t bt, at, tsu, uT, tT, tpart, tpart2, split, opa, opb, total;
};

// (split: bytes for the partial sums of dx's product over an 8-bit weight)
BwdLayout layout(int M, int N, int K, int rp, int planes, size_t split) {
  BwdLayout l{};
  size_t o = 0;
  l.bt = o;    o += up256((size_t)rp * N * 2);                      // B^T [RP x N] bf16
  l.at = o;    o += up256((size_t)K * rp * 2);                      // A^T [K x RP] bf16
  l.tsu = o;   o += up256((size_t)M * 2 * rp * 2);                  // hi | lo of s U [M x 2 RP] bf16, or s U [M x RP] fp32
  const size_t Mp = (size_t)padded_rows(M);
  l.uT = o;    o += up256(planes * (size_t)rp * Mp * 2);            // planes of (s U)^T, [planes][RP][Mp] bf16
  l.tT = o;    o += up256(planes * (size_t)rp * Mp * 2);            // planes of (s T)^T, [planes][RP][Mp] bf16
  l.tpart = o; o += up256((size_t)kTpreMaxChunks * M * rp * 4);     // pre-pass partials (s U)
  l.tpart2 = o; o += up256((size_t)kTpreMaxChunks * M * rp * 4);    // pre-pass partials (s T)
  int mch, nch_a, nch_b;
  outer_chunks(M, K, planes, mch, nch_a);
  outer_chunks(M, N, planes, mch, nch_b);
  const bool one = outer_in_one(M, planes);  // (no partials)
  const size_t oa = one ? 0 : (size_t)nch_a * rp * K, ob = one ? 0 : (size_t)nch_b * rp * N;
  l.opa = o;                                                        // dA's outer-product partials
  l.opb = o + up256(oa * 4);                                        // dB's outer-product partials
  l.split = o;                                                      // dx's, which is there before them
  l.total = o + std::max(up256(oa * 4) + up256(ob * 4), up256(split));
  return l;
}

}  // namespace

hipError_t launch_transpose_pad(const uint16_t* src, int R, int C, uint16_t* dst, int Rp, int Cp,
                                hipStream_t stream) {
  int n;
  const TransposeJob j = transpose_job(src, R, C, dst, Rp, Cp, n);
  hipLaunchKernelGGL(transpose_pad_kernel, dim3(n), dim3(256), 0, stream, j, n, j);
  return hipGetLastError();
}

size_t backward_ws_bytes(int M, int N, int K, int rp, int planes, size_t split) {
  return rp == 0 ? up256(split) : layout(M, N, K, rp, planes, split).total;
}

hipError_t launch_lora_backward(const BackwardArgs& a, void* ws, hipStream_t stream) {
  const int rp = padded_rank(a.r);
  hipError_t e;
  uint8_t* const w = static_cast<uint8_t*>(ws);
  const size_t split = a.base8 ? a.base8->split_bytes : 0;
  // dx over a weight in 8 bits: dy's bytes, then the product with its update
  auto dx_over_8 = [&](const void* ts, const uint16_t* at, size_t split_at) {
    Fp8LinearArgs g = *a.base8;
    g.split = reinterpret_cast<float*>(w + split_at);
    Fp8PrepArgs q{};
    q.x = q.xa = a.dy;
    q.M = a.M;
    q.K = a.N;
    q.xq = const_cast<uint8_t*>(g.xq);
    q.xs = const_cast<uint8_t*>(g.xs);
    fp8_prep_chunks(q.M, q.K, 0, q.nch, q.kch);
    const hipError_t err = launch_fp8_prep(q, stream);
    if (err != hipSuccess) return err;
    g.ts = ts;
    g.B = at;
    g.r = g.rp = g.ldb = rp;
    return launch_fp8_linear(g, stream);
  };
  if (rp == 0 && a.base8) return dx_over_8(nullptr, nullptr, 0);
  if (rp == 0) {  // no adapter: dx = dy W only
    if (!a.dx) return hipSuccess;
    LinearArgs g{};
    g.x = a.dy;
    g.W = a.Wt;
    g.M = a.M;
    g.N = a.K;
    g.K = a.N;
    g.y_off = a.dx;
    return launch_lora_gemm(g, stream);
  }
  const BwdLayout l = layout(a.M, a.N, a.K, rp, a.planes, split);
  uint16_t* bt = reinterpret_cast<uint16_t*>(w + l.bt);
  uint16_t* at = reinterpret_cast<uint16_t*>(w + l.at);
  const bool want_dx = a.dx || a.base8;
  const bool want_u = want_dx || a.dA;  // s U = s dy B
  const bool want_t = a.dB != nullptr;  // s T = s x A^T

  // 1. B^T [RP x N] (for s U) and A^T [K x RP] (the dx GEMM's LoRA rows), one launch
  {
    int n0 = 0, n1 = 0;
    TransposeJob j0{}, j1{};
    if (want_u) j0 = transpose_job(a.B, a.N, a.r, bt, a.N, rp, n0);
    if (want_dx) j1 = transpose_job(a.A, a.r, a.K, at, rp, a.K, n1);
    if (n0 + n1 > 0) {
      hipLaunchKernelGGL(transpose_pad_kernel, dim3(n0 + n1), dim3(256), 0, stream, j0, n0, j1);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  // 2. the pre-passes: s U from dy against the rows of B^T (hi | lo for dx, fp32 for dA), s T from x (fp32)
  TpreArgs u{}, tt{};
  u.x = a.dy;
  u.A = bt;
  u.s = a.s;
  u.M = a.M;
  u.K = a.N;
  u.r = a.r;
  u.Kform = tt.Kform = std::max(a.N, a.K);
  u.Kall = tt.Kall = a.N + a.K;
  const bool whole = a.base8 && a.base8->y_type == kF32;  // (s U in fp32, else as two parts)
  u.ts = want_dx && !whole ? reinterpret_cast<uint16_t*>(w + l.tsu) : nullptr;
  u.tv = whole ? reinterpret_cast<float*>(w + l.tsu) : nullptr;
  u.part = reinterpret_cast<float*>(w + l.tpart);
  u.tT = a.dA ? reinterpret_cast<uint16_t*>(w + l.uT) : nullptr;
  u.Mp = padded_rows(a.M);
  u.planes = tt.planes = a.planes;
  tt.x = a.x;
  tt.A = a.A;
  tt.s = a.s;
  tt.M = a.M;
  tt.K = a.K;
  tt.r = a.r;
  tt.part = reinterpret_cast<float*>(w + l.tpart2);
  tt.tT = reinterpret_cast<uint16_t*>(w + l.tT);
  tt.Mp = padded_rows(a.M);
  if (want_u && want_t)
    e = launch_lora_tpre2(u, tt, rp, stream);
  else
    e = launch_lora_tpre(want_u ? u : tt, rp, nullptr, stream);
  if (e != hipSuccess) return e;
  // 3. dx = dy W + s U A: the GEMM over W^T with slabs ([hi | lo](s U), A^T)
  if (a.base8) {
    if ((e = dx_over_8(w + l.tsu, at, l.split)) != hipSuccess) return e;
  } else if (a.dx) {
    LinearArgs g{};
    g.x = a.dy;
    g.W = a.Wt;
    g.s = a.s;
    g.M = a.M;
    g.N = a.K;
    g.K = a.N;
    g.r = a.r;
    g.y_on = a.dx;
    if ((e = launch_lora_gemm_slabs(g, u.ts, at, rp, stream)) != hipSuccess) return e;
  }
  // 4. dA[j][k] = sum_m sU[m][j] x[m][k] and dB[n][j] = sum_m dy[m][n] sT[m][j]: partials, then the finish
  int p0 = 0, f0 = 0, p1 = 0, f1 = 0;
  OuterArgs o0{}, o1{};
  if (a.dA)
    o0 = outer_job(u.tT, a.x, a.M, a.K, rp, a.r, a.planes, reinterpret_cast<float*>(w + l.opa), a.dA, true, p0, f0);
  if (a.dB)
    o1 = outer_job(tt.tT, a.dy, a.M, a.N, rp, a.r, a.planes, reinterpret_cast<float*>(w + l.opb), a.dB, false, p1, f1);
  if (p0 + p1 > 0)
    if ((e = launch_outer(o0, p0, f0, o1, p1, f1, rp, a.M, a.planes, stream)) != hipSuccess) return e;
  return hipSuccess;
}

}  // namespace hydra
