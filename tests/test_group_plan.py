"""The plan of the tensor-core products of the 4-bit layers (csrc/group/group_plan.h): host arithmetic, compiled on its own and gone over
for many shapes.  What its numbers have to keep, the kernel takes for granted."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2311_15806_b200", "csrc", "group")

PROGRAM = r"""
#include <cstdio>
#include <random>
#include "group_plan.h"
using namespace pipe::grp;
static int failed = 0;
static TcShape now;
#define CHECK(x) do { if (!(x) && failed++ < 5) std::printf("E %d O %d I %d N %lld ragged %d: %s\n", now.E, now.O, now.I, (long long)now.N, now.ragged, #x); } while (0)

static void look(const TcShape& c) {
  now = c;
  TcPlan p{};
  if (!plan_tc(c, &p)) {   // refused only where a number does not fit
    CHECK(static_cast<int64_t>(c.E) * (c.I / 32) >= (int64_t{1} << 31) || p.tiles >= (int64_t{1} << 31));
    return;
  }
  const int own = p.TN / p.cg;
  // tiles: whole MMA widths, pairs only with two halves to share and always beyond 128 rows, tensor memory's 512 columns
  CHECK(p.TN % 32 == 0 && p.TN >= 32 && p.TN <= 256 && (p.cg == 1 || p.cg == 2));
  CHECK(p.cg == 1 || c.O > 128);
  CHECK(p.TN <= 128 || p.cg == 2);
  CHECK(p.ta == (p.TN <= 128));
  CHECK(2 * p.TN + (p.ta ? 64 * widener_groups(true) : 0) <= 512 && (!p.ta || 2 * p.TN <= 256));
  CHECK(own <= 256 && own * 128 % 1024 == 0);                        // a box, whole atoms of the swizzle
  // rings
  CHECK(p.ring >= widener_groups(p.ta) && p.ring <= kTMaxRing);
  CHECK(p.code_depth >= widener_groups(p.ta) && p.code_depth <= kTMaxCodes);
  // shared memory: activations, widened weights, codes, turn, table, behind at most 1023 bytes up to a multiple of 1024
  CHECK(static_cast<int>(p.off_a) == p.ring * own * 256 && p.off_a % 1024 == 0);
  CHECK(p.off_codes - p.off_a == (p.ta ? 0u : 2u * kTSlotBytes) && p.off_codes % 1024 == 0);
  CHECK(p.off_turn - p.off_codes == static_cast<uint32_t>(p.code_depth) * kTCodeBytes && p.off_turn % 16 == 0);
  CHECK(p.off_table - p.off_turn == (p.split > 1 ? 0u : 2u * kTTurnBytes) && p.off_table % 4 == 0);
  CHECK(p.smem == 1024 + static_cast<int>(p.off_table) + 4 * unit_ints(c.E) && p.smem <= kTMaxSmem);
  CHECK(p.split == 1 || p.off_table >= static_cast<uint32_t>(p.TN) * 512);   // the sums of a split leave the table alone
  CHECK(2 * (p.smem + 1024) > 228 * 1024);                           // no two of these on an SM: each takes all of tensor memory
  // launch
  CHECK(p.stages == div_up(c.I, 128) && p.mtiles == div_up(c.O, 128 * p.cg));
  CHECK(p.split >= 1 && p.split <= 8 && (p.split == 1 || (p.cg == 1 && p.stages >= 4 * p.split)));
  CHECK(p.teams >= 1 && p.teams <= p.tiles && (p.split > 1 ? p.teams == p.tiles : p.teams * p.cg <= kChipSMs));
  CHECK(p.teams * p.cg * p.split < (int64_t{1} << 31));
}

int main() {
  const int Os[] = {1, 7, 64, 127, 128, 129, 200, 256, 257, 384, 768, 1411, 2048, 4096, 5003, 11008, 50000, 1 << 20, 1 << 29};
  const int Is[] = {32, 96, 128, 160, 256, 384, 512, 1024, 1408, 2048, 4096, 4160, 11008, 65536, 1 << 20, 1 << 29};
  const int64_t Ns[] = {1, 2, 16, 17, 31, 32, 33, 48, 63, 64, 65, 96, 97, 127, 128, 129, 150, 160, 192, 200, 255, 256, 257, 300, 511, 512, 513, 700, 1000, 1024,
                        2049, 4096, 18944, 20001, 100000, 1 << 20, (1 << 30) - 1, 1 << 30};
  const int Es[] = {1, 2, 3, 8, 24, 64, 100, 512, 1023, 1024};
  long n = 0;
  for (int O : Os)
    for (int I : Is)
      for (int64_t N : Ns) {
        look({1, O, I, false, N});
        ++n;
        for (int E : Es) look({E, O, I, true, N}), ++n;
      }
  std::mt19937_64 rng(7);
  auto draw = [&](double lo, double hi) { return lo * __builtin_exp(std::uniform_real_distribution<double>(0, __builtin_log(hi / lo))(rng)); };
  for (int i = 0; i < 300000; ++i) {
    const bool ragged = rng() & 1;
    look({ragged ? static_cast<int>(draw(1, 1025)) : 1, static_cast<int>(draw(1, 60000)), 32 * static_cast<int>(draw(1, 2000)), ragged, static_cast<int64_t>(draw(1, 300000))});
    ++n;
  }
  // no deal of the rows makes more units than the bound
  for (int i = 0; i < 20000; ++i) {
    const int E = static_cast<int>(draw(1, 200)), per = 8 << (rng() % 6);
    const int64_t N = static_cast<int64_t>(draw(1, 5000));
    int64_t left = N, units = 0;
    for (int e = 0; e < E && left > 0; ++e) {
      int64_t rows = e == E - 1 || rng() % 4 == 0 ? left : static_cast<int64_t>(rng() % (2 * N / E + 2));
      if (rng() % 3 == 0) rows = rows / per * per + 1;
      rows = rows < left ? rows : left;
      left -= rows;
      units += div_up(rows, per);
    }
    now = {E, per, 0, true, N};
    CHECK(units <= most_units(true, N, E, per));
  }
  std::printf("%ld shapes, %d failures\n", n, failed);
  return failed != 0;
}
"""


def _run(tmp_path, header):
    (tmp_path / "group_plan.h").write_text(header)
    (tmp_path / "plan.cpp").write_text(PROGRAM)
    exe = tmp_path / "plan"
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", str(tmp_path), str(tmp_path / "plan.cpp"), "-o", str(exe)], check=True)
    return subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)


def _header():
    return open(os.path.join(CSRC, "group_plan.h")).read()


def test_every_plan_keeps_what_the_kernel_takes_for_granted(tmp_path):
    r = _run(tmp_path, _header())
    assert r.returncode == 0, r.stdout


def test_tiles_of_256_rows_on_one_sm_would_be_seen(tmp_path):
    """The plan that once put the rings beyond shared memory."""
    header = _header()
    for line in ("|| (pair == 1 && cap > 128)", "if (p->code_depth < widener_groups(p->ta)) return false;"):
        assert line in header
        header = header.replace(line, "")
    r = _run(tmp_path, header)
    assert r.returncode == 1 and "p.TN <= 128 || p.cg == 2" in r.stdout and "p.code_depth >= widener_groups(p.ta)" in r.stdout, r.stdout
