// The plan of a tensor-core product of the 4-bit layers: tile, split, rings and shared memory.  Plain host arithmetic, compiled on its own
// by the tests, which go over the shapes.
#pragma once

#include <stdint.h>

namespace pipe {
namespace grp {

constexpr int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr int kChipSMs = 148;
constexpr int kTStage = 128;         // reduction length of a stage
constexpr int kTMaxRing = 6;         // most stages of activations
constexpr int kTMaxCodes = 12;       // most stages of codes
constexpr int kTMaxSmem = 226 * 1024;   // dynamic shared memory (the rest of 227 KiB: barriers)
constexpr int kTCodeBytes = 128 * kTStage / 2;            // of a stage
constexpr int kTSlotBytes = 128 * kTStage * 2;            // widened weights of a stage
constexpr int kTTurnBytes = 32 * 128 * 2;   // 32 rows of y by 128 channels
constexpr int widener_groups(bool ta) { return ta ? 4 : 2; }   // of four warps; ta: widened weights in tensor memory

// The integers of the table of units.
constexpr int unit_ints(int E) { return 3 * E + 1; }
// The most units of `per` rows that N rows on E experts can make: every expert with rows has at most one tile that is not full.
inline int64_t most_units(bool ragged, int64_t N, int E, int per) {
  if (!ragged) return div_up(N, per);
  return (N < E ? N : static_cast<int64_t>(E)) + N / per;
}

struct TcShape {
  int E, O, I;
  bool ragged;     // rows are dealt to the experts by offsets (otherwise one expert owns all N)
  int64_t N;
};
struct TcPlan {
  int TN;          // rows of a tile
  int cg;          // CTAs of a tile: 1, or a pair
  bool ta;         // widened weights in tensor memory
  int mtiles;      // ceil(O / (128 cg))
  int stages;      // ceil(I / 128)
  int split;       // CTAs (pairs have none) that share a tile's reduction axis
  int code_depth;
  int ring;        // stages of activations, at least the groups of wideners
  uint32_t off_a, off_codes, off_turn, off_table;   // shared memory behind the activations
  int smem;        // dynamic shared memory
  int64_t tiles;   // the most there can be
  int64_t teams;   // clusters of the launch
};

// The tile's rows (p->TN), the CTAs of a tile (p->cg) and those that share its axis (p->split): the least of
//     rounds of tiles on the SMs * (stages of a CTA * time of a stage + half a microsecond) + the sum over the CTAs of a split,
// in nanoseconds, with the times of a stage that were measured (11008 <-> 4096 and 2048 x 2048, 17 to 1024 rows):
//     one CTA 0.31 + TN / 1000 us, a pair with its weights in tensor memory 0.31 + 0.8 TN / 1000, in shared memory 0.36 + 1.2 TN / 1000,
//     and 0.6 at least (its two groups of wideners),
//     the split's sums 0.5 us + 3 ns a row and CTA.
// Either side of its choices there (us, when the rule was made; 17 to 512 rows have since become some 3 % faster): 2048 x 2048, 128 rows: units of 32 rows 10.3, of 128 12.4, those split four ways 11.4, eight ways 28;
// 4096 -> 11008: 300 rows as 3 units of pairs 33.5, as 2 43.6, 512 rows 46.4 and 49.4, 1024 rows 74.3 and 70.4; 11008 -> 4096, 17 rows: split
// four ways 15.6, not split 34.7.  kClusters: the clusters of 1, 2, .. CTAs, a whole SM each, that stand on the chip at once (as the runtime
// counts them, less one or two where they leave SMs of a processing cluster free: those differ from chip to chip).
constexpr int kClusters[9] = {0, 148, 74, 44, 32, 24, 20, 14, 14};
inline void choose_tile(const TcShape& c, TcPlan* p) {
  const int64_t experts = c.ragged ? (c.N < c.E ? c.N : c.E) : 1;
  const int64_t mean = div_up(c.N, experts);   // rows of an expert
  int64_t best = -1;
  for (int cap = 32; cap <= 256; cap *= 2) {
    // rows fill units evenly where there is one expert; otherwise an expert's last unit is half full, on average
    const int64_t units2 = c.ragged ? (2 * mean > cap ? 2 * mean + cap : 2 * cap) * experts / cap : 2 * div_up(c.N, cap);
    const int rows = c.ragged ? static_cast<int>(mean < cap ? div_up(mean, 32) * 32 : cap)
                               : static_cast<int>(div_up(div_up(2 * c.N, units2), 32) * 32);
    for (int pair = 1; pair <= 2; ++pair) {
      if ((pair == 2 && c.O <= 128) || (pair == 1 && cap > 128)) continue;
      const int64_t tiles = div_up(units2, 2) * div_up(c.O, 128 * pair);
      const int64_t stage = pair == 1 ? 310 + rows : (cap <= 128 ? 310 + rows * 4 / 5 : (rows < 200 ? 600 : 360 + rows * 6 / 5));
      for (int split = 1; split <= 8; ++split) {
        if (split > 1 && (pair == 2 || tiles > kClusters[split] || p->stages < 4 * split)) break;
        const int64_t rounds = div_up(tiles, pair == 2 ? kClusters[2] : kClusters[split]);
        const int64_t cost = rounds * (div_up(p->stages, split) * stage + 500) + (split > 1 ? 500 + 3 * split * rows : 0);
        if (best < 0 || cost < best) {
          best = cost;
          p->TN = c.ragged ? cap : rows;
          p->split = split;
          p->cg = pair;
        }
      }
    }
  }
  // (the bound on an expert call's units may be more than the clusters of one round can take: those tiles are one each)
  if (p->split > 1 && most_units(c.ragged, c.N, c.E, p->TN) * div_up(c.O, 128) * p->split >= (int64_t{1} << 31)) p->split = 1;
}


// False: not for the tensor-core kernel (coordinates or tiles beyond 31 bits, or no room for the rings).
inline bool plan_tc(const TcShape& c, TcPlan* p) {
  if (static_cast<int64_t>(c.E) * (c.I / 32) >= (int64_t{1} << 31)) return false;   // (rows of the code array: a copy's coordinate)
  p->stages = static_cast<int>(div_up(c.I, kTStage));
  choose_tile(c, p);
  p->ta = p->TN <= 128;
  p->mtiles = static_cast<int>(div_up(c.O, 128 * p->cg));
  p->tiles = most_units(c.ragged, c.N, c.E, p->TN) * p->mtiles;
  if (p->tiles >= (int64_t{1} << 31)) return false;
  p->teams = p->split > 1 ? p->tiles : kChipSMs / p->cg;
  if (p->teams > p->tiles) p->teams = p->tiles;
  p->ring = p->ta ? 4 : 3;
  const int x_bytes = p->ring * (p->TN / p->cg) * 256, a_bytes = p->ta ? 0 : widener_groups(false) * kTSlotBytes;
  const int turn = p->split > 1 ? 0 : 2 * kTTurnBytes, table = unit_ints(c.E) * 4;
  const int room = kTMaxSmem - 1024 - x_bytes - a_bytes - turn - table;
  p->code_depth = room / kTCodeBytes < kTMaxCodes ? room / kTCodeBytes : kTMaxCodes;
  if (p->code_depth < widener_groups(p->ta)) return false;
  p->off_a = x_bytes;
  p->off_codes = p->off_a + a_bytes;
  p->off_turn = p->off_codes + p->code_depth * kTCodeBytes;
  p->off_table = p->off_turn + turn;
  p->smem = 1024 + static_cast<int>(p->off_table) + table;
  return true;
}

}  // namespace grp
}  // namespace pipe
