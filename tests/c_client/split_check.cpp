// Host check of the division of work (attn_split.h): every unit's every visit belongs to exactly one
// workgroup, whatever the order, and the way back from a unit to its workgroups is the same.

#include <stdio.h>

#include <vector>

#include "attn_bwd_launch.h"

using namespace dsattn;

#define CHECK(ok)                                                                              \
  do {                                                                                         \
    if (!(ok)) {                                                                               \
      printf("line %d: %s (units %d full %d parts %d order %d)\n", __LINE__, #ok, s.units,      \
             s.full, s.parts, (int)s.order);                                                   \
      return false;                                                                            \
    }                                                                                          \
  } while (0)

static bool check_split(const WorkSplit& s, int tiles) {
  CHECK(s.full >= 0 && s.full <= s.units && s.parts >= 1);
  CHECK(s.parts > 1 || s.full == s.units);
  CHECK(s.grid() == s.full + s.slots());
  std::vector<int> seen(s.units, 0), next(s.units, 0);
  for (int x = 0; x < s.grid(); ++x) {
    const int unit = s.unit(x);
    CHECK(unit >= 0 && unit < s.units && (unit < s.full) == (x < s.full));
    CHECK(s.part(x) == seen[unit]);   // a unit's parts in order
    CHECK(x == s.workgroup(unit) + (x < s.full ? 0 : seen[unit] * s.shared()));
    ++seen[unit];
    for (const int count : {0, 1, s.parts - 1, tiles}) {
      int first, last;
      s.share(x, count, first, last);
      CHECK(0 <= first && first <= last && last <= count);
      if (x < s.full) CHECK(first == 0 && last == count);
    }
    int first, last;
    s.share(x, tiles, first, last);
    CHECK(first == next[unit]);
    next[unit] = last;
  }
  for (int unit = 0; unit < s.units; ++unit) {
    CHECK(seen[unit] == (unit < s.full ? 1 : s.parts));
    CHECK(next[unit] == tiles);
  }
  return true;
}

// Units to heads and groups, and what the table's gradient takes for the unit of a head's key group.
static bool check_places(const WorkSplit& s, int bh, int groups) {
  for (const bool bias : {false, true})
    for (const bool queries : {false, true}) {
      std::vector<int> seen((size_t)bh * groups, 0);
      for (int unit = 0; unit < s.units; ++unit) {
        const Place at = place_of(s, bias, unit, bh, groups, queries);
        CHECK(at.bh >= 0 && at.bh < bh && at.group >= 0 && at.group < groups);
        CHECK(seen[(size_t)at.bh * groups + at.group]++ == 0);
        if (bias && !queries)
          CHECK(unit == (s.order == kGroupByGroup ? at.group * bh + at.bh : at.bh * groups + at.group));
      }
    }
  return true;
}

int main() {
  bool ok = true;
  const UnitOrder orders[] = {kGroupByGroup, kHeadByHead, kHeadsToXcds};
  // every split of a few thousand units, whether the cost rule takes it or not
  for (const UnitOrder order : orders)
    for (int full = 0; full < 2100; full += full < 40 ? 1 : 37)
      for (int shared = 0; shared < 512; shared += shared < 10 ? 1 : 71)
        for (int parts = 2; parts < 9; parts += 3)
          ok = ok && check_split(shared > 0 ? WorkSplit{full + shared, full, parts, order}
                                            : WorkSplit{full, full, 1, order}, 23);
  // what the rule makes of heads, groups and tiles
  int xcds = 0, cut = 0, both = 0;
  for (int bh = 1; bh <= 1100; bh += bh < 20 ? 1 : 12)
    for (int groups = 1; groups <= 40; groups += groups < 6 ? 1 : 7)
      for (int tiles = 0; tiles <= 130; tiles += 13)
        for (const bool bias : {false, true}) {
          const long long units = (long long)bh * groups;
          const WorkSplit s = make_split(units, tiles, 0.012, unit_order(bias, false, bh, units));
          ok = ok && s.parts <= (tiles > 1 ? tiles : 1) && s.slots() <= 1024;
          ok = ok && check_split(s, tiles) && check_places(s, bh, groups);
          xcds += bias && s.order == kHeadsToXcds;
          cut += s.parts > 1;
          both += bias && s.order == kHeadsToXcds && s.parts > 1 && s.full > 0;
        }
  ok = ok && xcds > 0 && cut > 0 && both > 0;
  // no batch, no query or no key: no distances, and the rest of the call has nothing to divide
  ok = ok && bias_distances(0, 5, 7) == 0 && bias_distances(2, 0, 7) == 0 &&
       bias_distances(2, 5, 0) == 0 && bias_distances(2, 5, 7) == 11;
  ok = ok && make_split(0, 9, 0.012, kGroupByGroup).grid() == 0;
  // the sizes that the GPU tests take for XCD order: whole rounds, some left over, some shared
  const auto xcd_split = [](int bh, int n) {
    const long long units = (long long)bh * ((n + 127) / 128);
    return make_split(units, (n + 63) / 64, 0.012, unit_order(true, false, bh, units));
  };
  ok = ok && xcd_split(1024, 200).order == kHeadsToXcds && xcd_split(1024, 200).full == 2048;
  ok = ok && xcd_split(1032, 200).order == kHeadsToXcds && xcd_split(1032, 200).full == 2064;
  ok = ok && xcd_split(416, 520).order == kHeadsToXcds && xcd_split(416, 520).full == 2048 &&
       xcd_split(416, 520).parts > 1;
  printf("%s\n", ok ? "ok" : "failed");
  return ok ? 0 : 1;
}
