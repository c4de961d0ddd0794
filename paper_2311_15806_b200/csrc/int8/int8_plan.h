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
constexpr int kDrainWarps = 8;
constexpr int kTurnBytes = 32 * 32 * 2;     // a warp's 32 rows of y by 32 channels, 16-bit

struct TcShape {
  int E, O, I;
  bool ragged;     // rows are dealt to the experts by offsets (otherwise one expert owns all N)
  int64_t N;
};
struct TcPlan {
  int TN;          // most rows of a tile
  int TM;          // channels of a CTA's tile, a multiple of 8: 128 for a pair
  int KS;          // blocks of the reduction axis in a stage
  int cg;          // CTAs of a tile: 1, or a pair of SMs
  int mtiles;      // ceil(O / (TM cg))
  int stages;      // ceil(I / (128 KS))
  int split;       // CTAs (pairs have none) that share a tile's reduction axis
  int ring;        // stages in flight
  int resident;    // CTAs of an SM
  int columns;     // of tensor memory that a CTA takes
  uint32_t off_turn, off_sx, off_table;   // shared memory behind the ring
  int smem;        // dynamic shared memory
  int ahead;       // blocks of the first tile's weights that are asked into L2 early
  int64_t tiles;   // the most there can be
  int64_t teams;   // CTAs, pairs or clusters of the launch
};

// Shared memory, tensor memory and launch of a chosen tile.  False: it does not fit.
inline bool lay_out(const TcShape& c, TcPlan* p) {
  p->stages = static_cast<int>(div_up(c.I, kBlock * p->KS));
  p->mtiles = static_cast<int>(div_up(c.O, p->TM * p->cg));
  p->tiles = most_units(c.ragged, c.N, c.E, p->TN) * p->mtiles;
  if (p->tiles * p->split * p->cg >= (int64_t{1} << 31)) return false;
  // Accumulators: two of TN columns, 32 at least (what a drain reads at once); of a split one.  CTAs that wait for one another while they
  // hold tensor memory, the pairs, take so much shared memory that no two of them meet on an SM.
  const int wide = p->TN < 32 ? 32 : p->TN;
  p->columns = 32;
  while (p->columns < (p->split > 1 ? 1 : 2) * wide) p->columns *= 2;
  const int turn = p->split > 1 ? 0 : kDrainWarps * kTurnBytes, sx = p->split > 1 ? 0 : kDrainWarps * wide * 4, table = unit_ints(c.E) * 4;
  const int stage = p->KS * (p->TM + p->TN / p->cg) * kBlock;
  const int room = kMaxSmem / p->resident - (p->resident > 1 ? 1024 : 0) - 1024 - turn - sx - table;
  p->ring = room / stage < kMaxRing ? room / stage : kMaxRing;
  p->ahead = 16;
  if (p->ring < 2 || p->resident * p->columns > 512) return false;
  p->off_turn = static_cast<uint32_t>(p->ring * stage);
  p->off_sx = p->off_turn + turn;
  p->off_table = p->off_sx + sx;
  // the MMA reads 128 rows of weights, also behind the last stage's
  const int read = p->ring * stage + (128 - p->TM) * kBlock, all = static_cast<int>(p->off_table) + table;
  p->smem = 1024 + (read > all ? read : all);
  if (p->smem > kMaxSmem / p->resident) return false;
  p->teams = p->split > 1 ? p->tiles : kChipSMs * p->resident / p->cg;
  if (p->teams > p->tiles) p->teams = p->tiles;
  return true;
}

inline bool plan_tc(const TcShape& c, TcPlan* p) {
  const int64_t experts = c.ragged ? (c.N < c.E ? c.N : c.E) : 1;
  const int64_t mean = div_up(c.N, experts);   // rows of an expert
  int64_t best = -1;
  TcPlan t{};
  for (int cap = 16; cap <= 256; cap *= 2) {
    const int64_t units = c.ragged ? div_up(2 * mean > cap ? 2 * mean + cap : 2 * cap, 2 * cap) * experts : div_up(c.N, cap);
    for (int pair = 1; pair <= 2; ++pair) {
      if ((pair == 2 && (c.O <= 128 || cap < 64)) || (pair == 1 && cap > 128)) continue;
      for (int TM = pair == 2 ? 128 : 32; TM <= 128; TM += 16) {
        const int64_t tiles = units * div_up(c.O, TM * pair);
        const int64_t rounds = div_up(tiles, kChipSMs / pair);
        const int64_t block = pair == 1 ? 100 + (cap + TM) : 200 + cap * 6 / 10;
        const int64_t cost = rounds * (div_up(c.I, kBlock) * block + 500);
        t = TcPlan{};
        t.TN = cap; t.TM = TM; t.KS = pair == 2 ? 1 : 2; t.cg = pair; t.split = 1; t.resident = 1;
        if ((best < 0 || cost < best) && lay_out(c, &t)) {
          best = cost;
          *p = t;
        }
      }
    }
  }
  return best >= 0;
}

}  // namespace i8
}  // namespace pipe
