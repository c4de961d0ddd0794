// The plan of a tensor-core product of the 8-bit integer layers: tile, split, ring and shared memory.  Plain host arithmetic, compiled on
// its own by the tests, which go over the shapes.
#pragma once

#include <stdint.h>

#include "../group/group_plan.h"

namespace pipe {
namespace i8 {

using grp::div_up;
using grp::kChipSMs;
using grp::kClusters;
using grp::most_units;
using grp::unit_ints;

constexpr int kBlock = 128;                 // codes of a block of the reduction axis: bytes, a row of the 128-byte swizzle
constexpr int kMaxRing = 16;
constexpr int kMaxSmem = 226 * 1024;        // dynamic shared memory (the rest of 227 KiB: barriers)
constexpr int kDrainWarps = 8, kMoreDrainWarps = 16;
constexpr int kShort = 1408;
constexpr int kTurnBytes = 32 * 32 * 2;     // a warp's 32 rows of y by 32 channels, 16-bit

struct TcShape {
  int E, O, I;
  bool ragged;     // rows are dealt to the experts by offsets (otherwise one expert owns all N)
  int64_t N;
};
struct TcPlan {
  int TN;          // most rows of a tile
  int TM;          // channels of a CTA's tile, a multiple of 16 from 32 (a pair: 64) to 128
  int KS;          // blocks of the reduction axis in a stage
  int cg;          // CTAs of a tile: 1, or a pair of SMs
  int mtiles;      // ceil(O / (TM cg))
  int stages;      // ceil(I / (128 KS))
  int split;       // CTAs (pairs have none) that share a tile's reduction axis
  int ring;        // stages in flight
  int columns;     // of tensor memory that a CTA takes
  uint32_t off_turn, off_sx, off_table;   // shared memory behind the ring
  int drain;       // warps that drain
  int smem;        // dynamic shared memory
  int ahead;       // blocks of the first tile's weights that are asked into L2 early
  int64_t tiles;   // the most there can be
  int64_t teams;   // CTAs, pairs or clusters of the launch
};

constexpr int accumulator_columns(int TN) { return (TN + 31) & ~31; }

// Shared memory, tensor memory and launch of a chosen tile.  False: it does not fit.
inline bool lay_out(const TcShape& c, TcPlan* p) {
  p->stages = static_cast<int>(div_up(c.I, kBlock * p->KS));
  p->mtiles = static_cast<int>(div_up(c.O, p->TM * p->cg));
  p->tiles = most_units(c.ragged, c.N, c.E, p->TN) * p->mtiles;
  if (p->tiles * p->split * p->cg >= (int64_t{1} << 31)) return false;
  // Accumulators: two of TN columns, rounded up to what a drain reads at once; of a split one.  CTAs that wait for one another while they
  // hold tensor memory, the pairs, take so much shared memory that no two of them meet on an SM.
  const int wide = accumulator_columns(p->TN);
  p->columns = 32;
  while (p->columns < (p->split > 1 ? 1 : 2) * wide) p->columns *= 2;
  // Short sums on more than a round of tiles wait for the drain: 16 warps of it; longer ones want the ring.  By 8 and by 16 warps, us:
  //   4096 rows to 11008 channels, 16-bit, identity     I = 256 39, 35; 1024 46, 43; 1408 52, 52; 2048 66, 69; 4096 119, 126
  //                                SiLU                 60, 50; 65, 55; 67, 60; 78, 74; 122, 125
  //                                32-bit, identity     46, 38; 53, 52; 63, 64; 80, 82
  //                                SiLU                 68, 54; 72, 62; 77, 69; 88, 85
  //   4096 channels, 16-bit, identity and SiLU          1024 21, 20 and 30, 26; 1408 22.7, 23.1 and 31, 27; 2048 28, 29 and 33, 31
  //   1024 rows to 32000                                1024 35, 34 and 48, 42; 1408 42, 42 and 52, 47; 2048 55, 58 and 62, 61
  // and in one round 300 rows of I = 1024 9.1, 11.0.  (With an activation 16 still win at 2048, which the rule, blind to it, gives away: 1 to 8 %.)
  p->drain = p->split == 1 && c.I <= kShort && p->tiles > kChipSMs / p->cg ? kMoreDrainWarps : kDrainWarps;
  const int turn = p->split > 1 ? 0 : p->drain * kTurnBytes, sx = p->split > 1 ? 0 : 4 * wide * 4, table = unit_ints(c.E) * 4;
  const int stage = p->KS * (p->TM + p->TN / p->cg) * kBlock;
  // (the MMA reads 128 rows of weights, also behind the last stage's, where the others lie)
  const int read = (128 - p->TM) * kBlock, others = turn + sx + table;
  const int room = kMaxSmem - 1024 - (read > others ? read : others);
  p->ring = room / stage < kMaxRing ? room / stage : kMaxRing;
  p->ahead = 16;   // (4096 -> 11008 on one row: 10.2 us, with none 10.9, with 128 10.4)
  if (p->ring < 2 || p->columns > 512) return false;
  p->off_turn = static_cast<uint32_t>(p->ring * stage);
  p->off_sx = p->off_turn + turn;
  p->off_table = p->off_sx + sx;
  p->smem = 1024 + p->ring * stage + (read > others ? read : others);
  p->teams = p->split > 1 ? p->tiles : kChipSMs / p->cg;
  if (p->teams > p->tiles) p->teams = p->tiles;
  return true;
}

// The blocks of a stage: as many as about 48 KB hold, 4 at most (a stage's barriers cost what 128 columns of MMA do; larger stages leave too
// few in the ring).  4096 -> 11008 on one row: 4 blocks 10.1 us, 2 10.4, 1 11.9; on 64 rows: 4 13.0, 2 12.0.
inline int stage_blocks(int TM, int TN, int cg) {
  const int block = (TM + TN / cg) * kBlock;
  return 4 * block <= 50000 ? 4 : (2 * block <= 50000 ? 2 : 1);
}

// Tile (rows TN, channels TM, CTAs cg) and split: the least of, in nanoseconds,
//   rounds of tiles on the SMs * max(blocks of a CTA * max(160, 2.3 (TM + TN / cg)), 7000 + 5 TN)
//   + 47 TN + 30 a CTA (the next launch's start is overlapped on SMs that are left free) + 450 for a pair + 5000 for a split,
// a form (the copies' bytes, the drain, the launch's latency) whose numbers are fitted to 6000 timings of 75 shapes; the choice takes 2 %
// longer than the best that was timed, on average.  Either side (us): 11008 x 4096, one row: TM 80 10.1, TM 128 11.2; 128 rows: pairs of TM
// 80 14.0, single CTAs of TM 80 14.9; 512 rows: pairs of 192 rows 24.0, of 256 27.4; 4096 x 11008, one row: TM 128 split four ways 12.0,
// TM 32 not split 15.1; 3584 x 18944, one row: TM 112 split four ways 15.5, not split 26.8; 200 x 11008, 32 rows: four ways 8.6, not split 16.7;
// 4096 rows, 4096 -> 11008: pairs of 256 rows 123, single CTAs 150.  It is furthest off on small layers and few rows, whose tiles all stay
// below the floor: one row, weights from HBM, 4096 x 4096 TM 80 8.3, TM 32 8.0, TM 128 split three ways 8.0; 2048 x 2048 TM 128 5.8, TM 64 5.3; 1024
// x 4096 TM 80 7.3, TM 32 7.2, TM 64 split four ways 6.0.
inline int64_t tile_cost(int64_t tiles, int64_t blocks, int TN, int TM, int cg, int split) {
  const int64_t rounds = split > 1 ? 1 : div_up(tiles, kChipSMs / cg), load = (TM + TN / cg) * 23 / 10;
  const int64_t work = div_up(blocks, split) * (load > 160 ? load : 160), floor = 7000 + 5 * TN;
  const int64_t ctas = tiles * cg * split;
  return rounds * (work > floor ? work : floor) + 47 * TN + 30 * (ctas < kChipSMs ? ctas : kChipSMs) + (cg == 2 ? 450 : 0) + (split > 1 ? 5000 : 0);
}
// Whether that many CTAs may share a tile's axis: their clusters stand on the chip at once, each has four blocks.
inline bool may_split(int64_t tiles, int64_t blocks, int TN, int cg, int split) {
  return cg == 1 && TN <= 64 && blocks >= 4 * split && tiles <= kClusters[split];
}
inline bool plan_tc(const TcShape& c, TcPlan* p) {
  const int64_t experts = c.ragged ? (c.N < c.E ? c.N : c.E) : 1;
  const int64_t mean = div_up(c.N, experts);   // rows of an expert
  const int64_t blocks = div_up(c.I, kBlock);
  const int64_t least = div_up(mean, 256);
  int64_t best = -1;
  int last = 0;
  for (int64_t n = least; n < least + 8; ++n) {   // units of an expert with as many rows as that
    int rows = static_cast<int>(div_up(mean, n));
    if (c.ragged) rows = rows > 128 ? 256 : 2 * rows;   // (experts have unequal numbers of rows)
    const int small = (rows + 15) & ~15, wide = (rows + 31) & ~31;
    if (small == last) continue;
    last = small;
    for (int cg = 1; cg <= 2; ++cg) {
      if (cg == 2 && c.O <= 64) continue;
      const int TN = cg == 2 ? wide : (small < 128 ? small : 128);
      // rows fill units evenly where there is one expert; otherwise an expert's last unit is half full, on average
      const int64_t units = c.ragged ? (2 * mean > TN ? div_up(2 * mean + TN, 2 * TN) : 1) * experts : div_up(c.N, TN);
      for (int TM = cg == 1 ? 32 : 64; TM <= 128; TM += 16) {
        const int64_t tiles = units * div_up(c.O, TM * cg);
        for (int split = 1; split <= 8; ++split) {
          if (split > 1 && !may_split(tiles, blocks, TN, cg, split)) break;
          const int64_t cost = tile_cost(tiles, blocks, TN, TM, cg, split);
          if (best < 0 || cost < best) {
            best = cost;
            p->TN = TN; p->TM = TM; p->cg = cg; p->split = split;
          }
        }
      }
    }
  }
  p->KS = stage_blocks(p->TM, p->TN, p->cg);
  return lay_out(c, p);
}

}  // namespace i8
}  // namespace pipe
