// Which workgroup has which group of 128 own rows, and which part of the streamed axis.
#ifndef DSATTN_ATTN_SPLIT_H
#define DSATTN_ATTN_SPLIT_H

#include <hip/hip_runtime.h>

#include <algorithm>

namespace dsattn {

// A launch over `units` (heads times groups of own rows): workgroups 0 .. full - 1 have a unit
// each, the others share the remaining units, `parts` workgroups to each.  Their sums are joined
// from partial results, slot x - full of workgroup x.
//
// Two workgroups run on each of the 256 CUs at a time, 512 in all, so what is left over after
// whole rounds of 512 units (all of a small problem) is cut into parts.
__host__ __device__ constexpr int lesser(int a, int b) { return a < b ? a : b; }

enum UnitOrder { kGroupByGroup, kHeadByHead, kHeadsToXcds };
struct WorkSplit {
  int units, full, parts;
  UnitOrder order;
  __host__ __device__ int shared() const { return units - full; }
  __host__ __device__ int grid() const { return full + shared() * parts; }
  __host__ __device__ int slots() const { return shared() * parts; }
  // Workgroups go to the 8 XCDs in turn.  kHeadsToXcds: each gets a contiguous share of the units.
  __host__ __device__ int unit(int x) const {
    if (x >= full) return full + (x - full) % shared();
    if (order != kHeadsToXcds) return x;
    const int xcd = x & 7;
    return xcd * (full >> 3) + lesser(xcd, full & 7) + (x >> 3);
  }
  // The workgroup that has a unit, or its first part.
  __host__ __device__ int workgroup(int unit) const {
    if (unit >= full || order != kHeadsToXcds) return unit;
    const int most = full >> 3, more = full & 7, longer = more * (most + 1);
    const int xcd = unit < longer ? unit / (most + 1) : more + (unit - longer) / most;
    return 8 * (unit - xcd * most - lesser(xcd, more)) + xcd;
  }
  __host__ __device__ int part(int x) const { return x < full ? 0 : (x - full) / shared(); }
  // This workgroup's share [first, last) of `count` visits.
  __host__ __device__ void share(int x, int count, int& first, int& last) const {
    first = 0;
    last = count;
    if (x < full) return;
    const int n = (count + parts - 1) / parts;
    first = lesser(count, part(x) * n);
    last = lesser(count, first + n);
  }
};

// Head and 128-row group of a unit: head after head, or group after group of all heads.  A bias that
// closes later keys leaves the first key group and the last query group the most to do, so these
// come first (queries: the own rows are queries, taken from behind).
struct Place {
  int bh, group;
};
__host__ __device__ inline Place place_of(const WorkSplit& split, bool bias, int unit, int bh, int groups,
                                 bool queries) {
  const bool by_group = split.order == kGroupByGroup;
  const int group = by_group ? unit / bh : unit % groups;
  return Place{by_group ? unit % bh : unit / groups, bias && queries ? groups - 1 - group : group};
}

// Workgroups that run on an XCD at a time stream the same head through its L2 where each XCD has a
// share of heads (24 heads of 27280 rows forward with a bias 8.69 ms instead of 8.98 group by group;
// without one, backward, 256 of 1024 0.556 ms instead of 0.583 head by head, 40 of 7800 4.29 instead
// of 4.32, and from 16 of 32760 to 128 of 4096 the same within 0.3 %), which needs equal shares: not
// under a mask, whose heads keep more or less, nor where a causal bias leaves a part of a head more
// than another (5 heads of 32760 backward 6.86 ms instead of 5.37, group by group).  Few rounds want
// the groups in order, too.
inline UnitOrder unit_order(bool bias, bool mask, int bh, long long units) {
  if (mask) return kHeadByHead;
  return !bias || (bh % 8 == 0 && units >= 4 * 512) ? kHeadsToXcds : kGroupByGroup;
}

// Rows of a slot of partial sums: up to 32, or those of the waves that have any.
__host__ __device__ inline int part_rows(int n) {
  return n <= 32 ? n : n < 128 ? (n + 31) / 32 * 32 : 128;
}

// tiles: what a unit streams, at most.  join: what a part adds to the join, in times of a tile.
// Measured, in parts of the keys or queries: one head of 2048 rows backward 139 us alone, 60 in 4, 50 in
// the 8 taken here, 53 in 16; one token over 32760 keys of one head 636 us alone, 51 in 16, 29 in 64,
// 30 in the 86 taken, 47 in 256.
inline WorkSplit make_split(long long units, int tiles, double join, UnitOrder order) {
  const int rest = (int)(units % 512);
  // Up to 256 workgroups have a CU each and take 0.6 of the time of two on one; a part begins
  // with about two tiles' time without products.  The join is a launch, and adds up part by part.
  const auto cost = [&](int s) {
    const int all = rest * s, last = all % 512;
    const double rounds = (double)(all / 512) + (last == 0 ? 0.0 : last <= 256 ? 0.6 : 1.0);
    return rounds * ((tiles + s - 1) / s + 2) + (s == 1 ? 0.0 : 1.5 + 0.04 * s + (double)all * join);
  };
  int parts = 1;
  if (rest > 0)
    for (int s = 2; s <= std::min(tiles, 1024 / rest); ++s)
      if (cost(s) < cost(parts)) parts = s;
  return WorkSplit{(int)units, parts == 1 ? (int)units : (int)units - rest, parts, order};
}

}  // namespace dsattn

#endif
