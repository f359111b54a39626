"""What a linear over an 8-bit base writes into its workspace against the room that it is promised there, over types, rows,
outputs and lengths, without a GPU: the plans are host code (csrc/hydra_fp8_plan.h), compiled here with the host's compiler
and walked through whole."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2309_00754_amd", "csrc")

PROGRAM = r"""
#include <cmath>
#include <cstdio>
#include <random>

#include "hydra_fp8_plan.h"

using namespace hydra;

long split = 0, rounds = 0, wrong = 0;

void fail(const char* what, int M, int N, int K, int x, size_t need, size_t room) {
  if (wrong++ < 20) std::printf("%s: %d x %d x %d, %d: %zu bytes for %zu\n", what, M, N, K, x, room, need);
}

void product(int M, int N, int K) {
  const size_t room = fp8_split_most(M, N, K);
  for (int wide = 0; wide < 2; ++wide) {
    const Fp8Plan p = fp8_plan(wide, M, N, K);
    const Fp8TileCost& c = kFp8TileCosts[wide][p.tile];
    const int slabs = (K + c.bk - 1) / c.bk;
    const size_t need = p.split_values(M, N) * 4;
    if (need > room) fail("parts of K", M, N, K, p.nsplit, need, room);
    if (p.nsplit < 1 || (p.nsplit > 1 && !c.parts) || (long)p.nsplit * p.per < slabs || (long)(p.nsplit - 1) * p.per >= slabs)
      fail("a part without a slab, or a slab without a part", M, N, K, p.nsplit, need, room);
    const long parts = (long)((M + c.tm - 1) / c.tm) * ((N + c.tn - 1) / c.tn) * p.nsplit;
    split += p.nsplit > 1;
    rounds += p.nsplit > 1 && c.tm * c.tn > 128 * 128 && parts > 256;
  }
}

void before(int M, int K) {
  for (int rp = 16; rp <= 128; rp *= 2) {
    int nch = 0, kch = 0;
    fp8_prep_chunks(M, K, rp, nch, kch);
    const size_t need = (size_t)nch * M * rp * 4, room = fp8_prep_most(M, rp);
    if (need > room) fail("sums of T", M, 0, K, rp, need, room);
    if ((long)nch * kch * 128 < K) fail("a chunk short", M, 0, K, rp, nch, kch);
  }
}

int main() {
  const int cols[] = {16, 100, 688, 1000, 1030, 1040, 2048, 2600, 4096, 4352, 5120, 6000, 8192, 8200, 11008, 13824, 16384,
                      32000, 32768, 50272};
  const int lengths[] = {16, 880, 896, 912, 1024, 2048, 4096, 4112, 5120, 6000, 8192, 11008, 13824, 16000, 32768, 50272};
  for (int N : cols)
    for (int K : lengths) {
      size_t last = 0;
      for (int M = 1; M <= 4200; ++M) {
        product(M, N, K);
        const size_t room = fp8_split_most(M, N, K);
        if (room < last) fail("less room for more rows", M, N, K, 0, last, room);
        last = room;
      }
    }
  for (int K : lengths)
    for (int rp = 0; rp <= 128; rp = rp ? 2 * rp : 16) {
      size_t last = 0;
      for (int M = 1; M <= 20000; ++M) {
        if (rp == 16) before(M, K);
        const size_t room = fp8_prep_most(M, rp);
        if (room < last) fail("less room for more rows", M, 0, K, rp, last, room);
        last = room;
      }
    }
  // sizes at large: logarithms spread evenly over all that the calls take
  std::mt19937 g(1);
  const auto draw = [&](double most) { return (int)std::exp2(std::uniform_real_distribution<double>(0, most)(g)); };
  for (int i = 0; i < 1000000; ++i) {
    const int M = draw(20), N = draw(21), K = 16 * draw(17);
    if ((int64_t)((M + 127) / 128) * ((N + 255) / 256) >= (1 << 23)) continue;
    product(M, N, K);
    before(M, K);
  }
  std::printf("%ld in parts, %ld of them over more than 256 parts of the largest tile, %ld wrong\n", split, rounds, wrong);
  return wrong ? 1 : split > 0 && rounds > 0 ? 0 : 2;
}
"""


def test_every_plan_fits_the_room_it_is_promised(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "plans.cpp", tmp_path / "plans"
    src.write_text(PROGRAM)
    r = subprocess.run([cxx, "-O2", "-std=c++17", "-Wall", "-I", CSRC, str(src), "-o", str(exe)], capture_output=True,
                       text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout
