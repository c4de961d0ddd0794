"""What the plan of the 8-bit integer products (csrc/int8/int8_plan.h) has chosen is what it returns: no tile that the cost found best is
given up because the ring has taken the shared memory that the tile's reads behind it need."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2311_15806_b200", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <initializer_list>
#include "int8_plan.h"
using namespace pipe::i8;

int main() {
  const int Os[] = {1, 40, 128, 200, 384, 768, 1024, 1411, 2048, 2560, 3584, 4096, 6144, 8192, 11008, 20000};
  const int Is[] = {512, 1024, 1408, 2048, 4096, 5120, 8192, 11008, 14336, 18944, 28672, 65536, 131071};
  const int Ns[] = {1, 2, 8, 13, 16, 17, 32, 33, 48, 64, 65, 130, 200, 700};
  long shapes = 0, splits = 0, failed = 0;
  for (int E : {1, 2, 8, 64, 1024})
    for (int O : Os)
      for (int I : Is)
        for (int N : Ns)
          for (int ragged = E > 1; ragged < 2; ++ragged) {
            const TcShape c{E, O, I, ragged != 0, N};
            TcPlan p{};
            bool good = plan_tc(c, &p);
            ++shapes;
            splits += p.split > 1;
            // of this tile no other split costs less
            const int64_t experts = ragged ? (N < E ? N : E) : 1, mean = div_up(N, experts), blocks = div_up(I, kBlock);
            const int64_t units = ragged ? (2 * mean > p.TN ? div_up(2 * mean + p.TN, 2 * p.TN) : 1) * experts : div_up(N, p.TN);
            const int64_t tiles = units * div_up(O, p.TM * p.cg), own = tile_cost(tiles, blocks, p.TN, p.TM, p.cg, p.split);
            for (int split = 1; split <= 8; ++split)
              if (split == 1 || may_split(tiles, blocks, p.TN, p.cg, split)) good = good && tile_cost(tiles, blocks, p.TN, p.TM, p.cg, split) >= own;
            // and it lies in shared memory: the table, and 128 rows of weights of the last stage's last block
            const int stage = p.KS * (p.TM + p.TN / p.cg) * kBlock;
            good = good && p.smem <= kMaxSmem && p.smem >= 1024 + static_cast<int>(p.off_table) + 4 * unit_ints(E) &&
                   p.smem >= 1024 + (p.ring - 1) * stage + (p.KS - 1) * p.TM * kBlock + 128 * kBlock && p.smem >= 1024 + p.ring * stage + (128 - p.TM) * kBlock;
            if (!good && failed++ < 5) std::printf("E %d O %d I %d N %d ragged %d: TN %d TM %d cg %d split %d ring %d smem %d\n", E, O, I, N, ragged, p.TN, p.TM, p.cg, p.split, p.ring, p.smem);
          }
  std::printf("%ld shapes, %ld split, %ld failed\n", shapes, splits, failed);
  return failed != 0 || splits < 100;
}
"""


def test_the_split_that_costs_least_is_the_one_returned(tmp_path):
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(CSRC, "int8"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
