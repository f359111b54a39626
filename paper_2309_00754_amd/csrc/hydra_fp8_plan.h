// Sizes and plans of the linear over an 8-bit weight (fp8_linear.hip), host code
// alone: what its workspace holds and what its launches write there follow from
// the same numbers.
#pragma once

#include <cstddef>
#include <cstdint>

namespace hydra {

// ------------------------------------------------------------------ before the product

constexpr int kFewRows = 16;
constexpr int kStagedChunks = 8;  // most partial sums of T at padded rank 16 above kFewRows rows

// Whether the product takes s T as ts, else the partial sums.  A tile's partial sums of T
// at a high rank are many, and another launch pays that adds
// them up once.  us without and with it: 2048 x 11008 x 4096 at rank 128 into bf16 198.6 and
// 161.6, 1024 x 4096 x 4096 64.7 and 53.4, 250 x 2048 x 8192 46.8 and 37.4, 40 x 1024 x 1024 17.8 and
// 19.2; 2048 x 4096 x 4096 at 64 64.0 and 60.9, 512 38.9 and 38.3, 64 21.9 and 22.8; 2048 at 32
// 54.3 and 53.8, 512 33.9 and 35.1.
inline bool fp8_finishes_t(int M, int rp) { return rp > 16 && M > kFewRows && (int64_t)M * rp >= 24576; }
// Chunks of K: about 512 workgroups, each at least a block a wave (few rows at a rank
// above 16: fewer, as A's rows take the time; 1 x 4096 x 4096 at rank 128 18.1 -> 13.6 us, 8 x
// 8192 x 4096 at 64 19.7 -> 17.9), and no more partial sums of T than the product can
// add up on the side.  2048 x 4096 at rank 16 takes 8.5 to 9.1 us with 256, 512, 768 or
// 1024 workgroups and with 4, 8 or 16 waves.
inline void fp8_prep_chunks(int M, int K, int rp, int& nch, int& kch) {
  const int kb = (K + 127) / 128, mb = (M + 15) / 16;
  int want = (512 + mb - 1) / mb;
  const int most = rp == 0 ? 64 : M <= kFewRows ? 32 : rp <= 32 || fp8_finishes_t(M, rp) ? kStagedChunks : 4;
  want = want < most ? want : most;
  kch = (kb + want - 1) / want;
  const int least = M <= kFewRows && rp > 16 ? 256 / rp : 8;
  kch = kch < least ? least : kch;
  nch = (kb + kch - 1) / kch;
}
// Bytes of room for those partial sums that any call with up to M rows can do with.
inline size_t fp8_prep_most(int M, int rp) {
  if (rp == 0) return 0;
  const size_t few = (size_t)32 * (M < kFewRows ? M : kFewRows);
  const size_t by_rows = (size_t)kStagedChunks * M, by_grid = (size_t)(512 + 1) * 16 + M;
  const size_t many = M <= kFewRows ? 0 : by_rows < by_grid ? by_rows : by_grid;
  return (few > many ? few : many) * rp * 4;
}

// ------------------------------------------------------------------ tiles

// The tile by a model of its time: base + fixed w + K / 128 (step w + pair r), us, for w
// workgroups a CU one after the other (pair: in r rounds of two together).  The
// numbers are fits to 15 row counts from 17 to 4096 and eight (N, K) from 1000 x 688
// to 11008 x 4096 and 4096 x 11008 (rms error 5 to 11%).  They choose the best of the six
// tiles or one 0.4% slower on average, 9% at most.  What they say: a small tile's
// slab costs its copies (32 to 50 GB/s into a CU), the largest one's its products.
// us, M x N x K into bf16 and fp32: 64 x 4096 x 4096 10.0 and 11.5, 333 x 4096 x
// 11008 37 and 48, 1000 x 4096 x 4096 24 and 37, 2048 x 4096 x 4096 38 and 60.
struct Fp8TileCost {
  int tm, tn, bk;  // rows, columns, values of K in a slab
  bool parts;      // may take K in parts
  float base, fixed, step, pair;
};
constexpr int kFp8Tiles = 6;
constexpr Fp8TileCost kFp8TileCosts[2][kFp8Tiles] = {{{128, 256, 128, true, 0.f, 5.8f, 0.767f, 0.f},
                                                      {128, 128, 128, true, 0.f, 4.99f, 0.516f, 0.f},
                                                      {64, 128, 128, true, 0.1f, 4.19f, 0.376f, 0.f},
                                                      {64, 64, 128, false, 2.47f, 1.23f, 0.136f, 0.143f},
                                                      {32, 64, 256, true, 1.98f, 1.93f, 0.219f, 0.f},
                                                      {32, 32, 256, false, 3.36f, 0.5f, 0.084f, 0.095f}},
                                                     {{128, 256, 128, true, 0.f, 6.42f, 1.318f, 0.f},
                                                      {128, 128, 128, true, 0.f, 5.24f, 0.775f, 0.f},
                                                      {64, 128, 128, true, 0.f, 4.56f, 0.542f, 0.f},
                                                      {64, 64, 128, false, 2.16f, 1.58f, 0.182f, 0.195f},
                                                      {32, 64, 256, true, 1.57f, 2.23f, 0.272f, 0.f},
                                                      {32, 32, 256, false, 2.9f, 0.72f, 0.067f, 0.165f}}};

// K in parts: few rows and a long K leave CUs without a tile.  The
// parts' sums go through memory, and a second launch joins them, for 3.9 us and the
// sums written and read at 6.75 TB/s (a fit to 330 cases, rms error 9%).  us, whole ->
// in parts, fp32: 17 x 2048 x 8192 17.9 -> 11.4, 64 x 4096 x 11008 25.3 -> 21.8, 200 x 4096 x
// 11008 38.6 -> 32.7; with tile 0 among them 333 x 4096 x 11008 59.3 -> 57.1 (bf16 51.2 ->
// 47.8), rank 16 and x quantized in the call; 54 to 56 (42) with the joining launch that asks
// for the parts' sums first.  Below K = 4096 never faster.
constexpr int kFp8MaxSplit = 8, kFp8MaxParts = 512;

struct Fp8Plan {
  int tile;
  int nsplit, per;  // parts of K, of `per` slabs
  // fp32 values of the parts' sums, [nsplit][M][N]
  size_t split_values(int M, int N) const { return nsplit > 1 ? (size_t)nsplit * M * N : 0; }
};
inline Fp8Plan fp8_plan(bool wide, int M, int N, int K) {
  int tile = 0, split = 1;
  float least = 0.f;
  for (int i = 0; i < kFp8Tiles; ++i) {
    const Fp8TileCost& c = kFp8TileCosts[wide][i];
    const int64_t tiles = (int64_t)((M + c.tm - 1) / c.tm) * ((N + c.tn - 1) / c.tn);
    const int slabs = (K + 127) / 128;
    const bool may = c.parts && tiles < 256;
    for (int s = 1; s <= (may ? kFp8MaxSplit : 1) && s * 4 <= (s == 1 ? 4 : slabs); ++s) {
      const int64_t n = tiles * s;
      if (s > 1 && n > kFp8MaxParts) break;
      const float w = (float)((n + 255) / 256), r = (float)((n + 511) / 512), sl = (float)((slabs + s - 1) / s);
      float us = c.base + c.fixed * w + sl * (c.step * w + c.pair * r);
      if (s > 1) us += 3.9f + (float)s * 8.f * (float)M * (float)N / 6.75e6f;
      if ((i == 0 && s == 1) || us < least) {
        least = us;
        tile = i;
        split = s;
      }
    }
  }
  const int bk = kFp8TileCosts[wide][tile].bk, slabs = (K + bk - 1) / bk, per = (slabs + split - 1) / split;
  return Fp8Plan{tile, (slabs + per - 1) / per, per};
}

// Most values of one part of a tile.
constexpr size_t fp8_largest_part() {
  size_t v = 0;
  for (const auto& type : kFp8TileCosts)
    for (const Fp8TileCost& c : type) v = c.parts && (size_t)c.tm * c.tn > v ? (size_t)c.tm * c.tn : v;
  return v;
}
// Bytes of room for the parts' sums that any call with up to M rows can do with (0
// where K is never split): a plan has at most kFp8MaxSplit sums of every output, and at
// most kFp8MaxParts parts of the largest tile.
inline size_t fp8_split_most(int M, int N, int K) {
  if (K <= 128 * 7) return 0;
  const size_t all = (size_t)kFp8MaxSplit * M * N, parts = kFp8MaxParts * fp8_largest_part();
  return (all < parts ? all : parts) * 4;
}

}  // namespace hydra
