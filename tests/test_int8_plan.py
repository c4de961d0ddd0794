"""The plan of the tensor-core products of the 8-bit layers (csrc/int8/int8_plan.h): host arithmetic, compiled on its own and gone over for
many shapes.  What its numbers have to keep, the kernel takes for granted."""
import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2311_15806_b200", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <random>
#include "int8_plan.h"
using namespace pipe::i8;
static int failed = 0;
static TcShape now;
#define CHECK(x) do { if (!(x) && failed++ < 5) std::printf("E %d O %d I %d N %lld ragged %d: %s\n", now.E, now.O, now.I, (long long)now.N, now.ragged, #x); } while (0)

static void look(const TcShape& c) {
  now = c;
  TcPlan p{};
  if (!plan_tc(c, &p)) {   // refused only where a number does not fit
    CHECK(p.tiles * p.split * p.cg >= (int64_t{1} << 31));
    return;
  }
  const int own = p.TN / p.cg, wide = (p.TN + 31) / 32 * 32;
  // tiles: whole MMA widths, boxes and atoms of the swizzle
  CHECK(p.cg == 1 || p.cg == 2);
  CHECK(p.TN >= 16 && p.TN <= 256 && p.TN % (p.cg == 2 ? 32 : 16) == 0 && (p.cg == 2 || p.TN <= 128));
  CHECK(p.TM % 8 == 0 && p.TM >= 32 && p.TM <= 128 && own % 8 == 0);
  CHECK(p.KS == 1 || p.KS == 2 || p.KS == 4);
  CHECK(accumulator_columns(p.TN) == wide);
  // accumulators: two, of a split one, what the drain reads at once inside of them
  CHECK(p.columns >= 32 && p.columns <= 512 && (p.columns & (p.columns - 1)) == 0);
  CHECK((p.split > 1 ? 1 : 2) * wide <= p.columns);
  // ring and shared memory
  const int stage = p.KS * (p.TM + own) * 128;
  CHECK(p.ring >= 2 && p.ring <= kMaxRing);
  CHECK(static_cast<int>(p.off_turn) == p.ring * stage && p.off_turn % 1024 == 0);
  CHECK(p.off_sx - p.off_turn == (p.split > 1 ? 0u : p.drain * kTurnBytes) && p.off_sx % 16 == 0);
  CHECK(p.off_table - p.off_sx == (p.split > 1 ? 0u : 4u * 4u * wide) && p.off_table % 4 == 0);
  CHECK(p.smem >= 1024 + static_cast<int>(p.off_table) + 4 * unit_ints(c.E) && p.smem <= kMaxSmem);
  // the last block's weights, read as 128 rows
  CHECK(p.smem >= 1024 + (p.ring - 1) * stage + (p.KS - 1) * p.TM * 128 + 128 * 128);
  CHECK(p.split == 1 || p.ring * stage >= p.TN * 512);               // a split's sums
  CHECK(p.cg == 1 || 2 * (p.smem + 1024) > 228 * 1024);              // no two pairs' CTAs on an SM
  // launch
  CHECK(p.stages == div_up(c.I, 128 * p.KS) && p.mtiles == div_up(c.O, p.TM * p.cg));
  CHECK(p.split >= 1 && p.split <= 8 && (p.split == 1 || (p.cg == 1 && p.stages >= p.split)));
  CHECK(p.teams >= 1 && p.teams <= p.tiles && (p.split > 1 ? p.teams == p.tiles : p.teams * p.cg <= kChipSMs));
  CHECK(p.teams * p.cg * p.split < (int64_t{1} << 31) && p.tiles < (int64_t{1} << 31));
  CHECK(int64_t{p.stages} * p.split < (int64_t{1} << 31) && p.ahead >= 0);
}

int main() {
  const int Os[] = {1, 7, 31, 64, 65, 127, 128, 129, 200, 256, 257, 384, 768, 1411, 2048, 4096, 5003, 11008, 50000, 1 << 20, 1 << 29};
  const int Is[] = {1, 16, 100, 128, 129, 256, 384, 512, 1024, 1408, 2048, 4096, 4160, 11008, 65536, 131071};
  const int64_t Ns[] = {1, 2, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 96, 97, 127, 128, 129, 150, 160, 192, 200, 255, 256, 257, 300, 511, 512, 513, 700, 1000, 1024,
                        2049, 4096, 18944, 20001, 100000, 1 << 20, (1 << 30) - 1, 1 << 30};
  const int Es[] = {1, 2, 3, 8, 24, 64, 100, 512, 1023, 1024};
  long n = 0;
  for (int O : Os)
    for (int I : Is)
      for (int64_t N : Ns) {
        look({1, O, I, false, N});
        for (int E : Es)
          if (int64_t{E} * O <= (int64_t{1} << 30)) look({E, O, I, true, N}), ++n;
        ++n;
      }
  std::mt19937_64 g(7);
  for (int i = 0; i < 200000; ++i) {
    auto draw = [&](double most) { return static_cast<int64_t>(std::exp(std::uniform_real_distribution<double>(0, std::log(most))(g))); };
    const int E = static_cast<int>(draw(1024));
    const bool ragged = E > 1 || (g() & 1);
    look({E, static_cast<int>(1 + draw((1 << 29) / E)), static_cast<int>(1 + draw(131070)), ragged, 1 + draw(1 << 30)});
    ++n;
  }
  std::printf("%ld shapes, %d failed\n", n, failed);
  return failed != 0;
}
"""


def test_the_plan_keeps_what_the_kernel_takes_for_granted(tmp_path):
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text("#include <cmath>\n" + PROGRAM)
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(CSRC, "int8"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout


def test_waits_that_give_up_leave_together():
    """Behind a wait of the drain come operations of whole warps: its verdict is voted on.  Copies and products are one elected thread's, which
    meets its warp again before the block's barriers.  A split's CTA gives tensor memory back before it waits for the others."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "int8", "int8_tc.cu")).read())
    kernel = text[text.index("int8_tc_kernel(const __grid_constant__"):text.index("static auto tc_kernel(int cg)")]
    copies = kernel[kernel.index("if (warp == 0) {"):kernel.index("} else if (warp == 1) {")]
    products = kernel[kernel.index("} else if (warp == 1) {"):kernel.index("} else if (p.split == 1) {")]
    rest = kernel[kernel.index("} else if (p.split == 1) {"):]
    for one in (copies, products):
        assert re.search(r"elect_one\(\)\) \{", one) and one.rstrip().endswith("}\n    __syncwarp();")
        assert one.count("__syncwarp") == 1 and "__all_sync" not in one and "__shfl" not in one
    assert rest.count("mbar_wait<") == rest.count("__all_sync(0xffffffffu, mbar_wait<") == 2 and "bar.sync" not in rest
    assert kernel.index("tcgen05.dealloc.cta_group::1") < kernel.index("if (CG == 1 && p.split > 1) {") < kernel.rindex("cluster_sync();")
    assert products.index("if (!ok) drain_ring(done") > products.index("commit<CG>(d_full") and "drain_ring(full" in copies
