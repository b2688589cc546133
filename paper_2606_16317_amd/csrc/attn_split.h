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
struct WorkSplit {
  int units, full, parts;
  __host__ __device__ int shared() const { return units - full; }
  __host__ __device__ int grid() const { return full + shared() * parts; }
  __host__ __device__ int slots() const { return shared() * parts; }
  __device__ int unit(int x) const { return x < full ? x : full + (x - full) % shared(); }
  __device__ int part(int x) const { return x < full ? 0 : (x - full) / shared(); }
  // This workgroup's share [first, last) of `count` visits.
  __device__ void share(int x, int count, int& first, int& last) const {
    first = 0;
    last = count;
    if (x < full) return;
    const int n = (count + parts - 1) / parts;
    first = min(count, part(x) * n);
    last = min(count, first + n);
  }
};

// Head and 128-row group of a unit.  A bias that closes later keys leaves the first key group
// and the last query group the most to do: with a bias these come first for all heads, so that no
// long one starts late.  (Otherwise a head's groups stand together, whose tiles L2 then shares.)
struct Place {
  int bh, group;
};
__device__ inline Place place_of(bool bias, int unit, int bh, int groups, bool queries) {
  if (!bias) return Place{unit / groups, unit % groups};
  const int group = unit / bh;
  return Place{unit % bh, queries ? groups - 1 - group : group};
}

// Rows of a unit's partial sums.
__host__ __device__ inline int part_rows(int n) { return n < 128 ? n : 128; }

// tiles: what a unit streams, at most.  join: what a part adds to the join, in times of a tile.
inline WorkSplit make_split(long long units, int tiles, double join) {
  const int rest = (int)(units % 512);
  // Up to 256 workgroups have a CU each and take 0.6 of the time of two on one; a part begins
  // with about two tiles' time without products, and the join is a launch.
  const auto cost = [&](int s) {
    const int all = rest * s, last = all % 512;
    const double rounds = (double)(all / 512) + (last == 0 ? 0.0 : last <= 256 ? 0.6 : 1.0);
    return rounds * ((tiles + s - 1) / s + 2) + (s == 1 ? 0.0 : 2.0 + (double)all * join);
  };
  int parts = 1;
  if (rest > 0)
    for (int s = 2; s <= std::min(tiles / 2, 1024 / rest); ++s)
      if (cost(s) < cost(parts)) parts = s;
  return WorkSplit{(int)units, parts == 1 ? (int)units : (int)units - rest, parts};
}

}  // namespace dsattn

#endif
