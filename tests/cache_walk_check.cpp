// Host check of csrc/cache_walk.h: every slot that some row sees lies in exactly one tile of the walk, no tile
// starts behind the length, max_tiles' bound holds, and the workers' shares cut the list of all segments into
// pieces whose slots are distinct.
#include <cstdio>
#include <set>
#include <vector>

#include "cache_walk.h"

using namespace minf;

static int fails = 0;
#define CHECK(c)                                                 \
  if (!(c)) {                                                    \
    if (fails++ < 10) printf("FAIL line %d: %s\n", __LINE__, #c); \
  }

static int walks() {
  int cases = 0;
  const int caps[] = {1, 31, 32, 33, 64, 100, 257, 500};
  const int news[] = {1, 2, 5, 33, 64};
  const int inits[] = {0, 1, 31, 32, 40, 200, 500};
  const int locals[] = {1, 2, 31, 32, 33, 64, 100, 500};
  for (int cap : caps)
    for (int T : news)
      for (int ni : inits)
        for (int nl : locals) {
          if (ni > cap || nl > cap) continue;
          const int bound_keys = ni + nl + T + 2 * CACHE_TILE;
          const int bound = ((bound_keys < cap ? bound_keys : cap) + CACHE_TILE - 1) / CACHE_TILE;
          for (int len = -1; len <= cap + 1; len += (cap > 100 ? 7 : 1)) {
            const SeqWalk w = seq_walk(len, cap, T, ni, nl);
            ++cases;
            CHECK(w.len == (len < 0 ? 0 : len > cap ? cap : len));
            CHECK(w.tiles >= 0 && w.tiles <= bound);
            std::vector<int> times(cap + CACHE_TILE, 0);
            for (int t = 0; t < w.tiles; ++t) {
              CHECK(w.base(t) >= 0 && w.base(t) < w.len && w.base(t) % CACHE_TILE == 0);
              for (int i = 0; i < CACHE_TILE; ++i) {
                ++times[w.base(t) + i];
                if (w.base(t) + i < w.len) CHECK(w.tile_of(w.base(t) + i) == t);
              }
            }
            for (int j = 0; j < w.len; ++j) {
              bool seen = false;
              for (int t = 0; t < T; ++t) seen = seen || (w.i0 + t >= 0 && cache_visible(j, w.i0 + t, ni, nl));
              CHECK(times[j] <= 1);
              CHECK(!seen || times[j] == 1);
              CHECK(!seen || j < w.e1 || j >= w.lo);
              CHECK(T > 1 || seen == (j < w.e1 || j >= w.lo));
              CHECK((w.tile_of(j) >= 0) == (times[j] == 1));
            }
          }
        }
  return cases;
}

// Row tiles: the walk of some rows of a sequence holds every slot that one of them sees once, and parts hold
// every tile once.
static int rows() {
  int cases = 0;
  for (int cap : {1, 64, 65, 200, 700})
    for (int T : {1, 2, 40, 64})
      for (int group : {1, 3, 8})
        for (int tile_rows : {64, 128, 256})
          for (int ni : {0, 5, 100})
            for (int nl : {1, 50, 700}) {
              if (ni > cap || nl > cap) continue;
              for (int len = 0; len <= cap; len += (cap > 100 ? 37 : 1))
                for (int r0 = 0; r0 < T * group; r0 += tile_rows) {
                  ++cases;
                  const int r1 = (r0 + tile_rows < T * group ? r0 + tile_rows : T * group) - 1;
                  const auto w = rows_walk(r0, r1, group, len, cap, T, ni, nl);
                  const int i0 = len - T;
                  std::vector<int> times(cap + SHARED_TILE, 0);
                  for (int t = 0; t < w.tiles; ++t) {
                    CHECK(w.base(t) >= 0 && w.base(t) < len && w.base(t) % SHARED_TILE == 0);
                    for (int i = 0; i < SHARED_TILE; ++i) ++times[w.base(t) + i];
                  }
                  for (int j = 0; j < cap; ++j) {
                    bool seen = false;
                    for (int t = r0 / group; t <= r1 / group; ++t) seen = seen || (i0 + t >= 0 && cache_visible(j, i0 + t, ni, nl));
                    CHECK(times[j] <= 1 && (!seen || times[j] == 1));
                    CHECK(!seen || (j < w.len && (j < w.e1 || j >= w.lo)));
                  }
                  // the position of the first row's token where it is one
                  CHECK(i0 + r1 / group < 0 || w.i0 == i0 + r0 / group);
                  CHECK(i0 + r1 / group >= 0 || w.tiles == 0);
                  for (int splits : {1, 2, 7, 64}) {
                    const int per = part_tiles(w.tiles, splits), parts = part_count(w.tiles, splits);
                    CHECK(parts <= splits && parts * per >= w.tiles && (w.tiles == 0 ? parts == 0 : (parts - 1) * per < w.tiles));
                  }
                }
            }
  return cases;
}

static int shares() {
  int cases = 0;
  const std::vector<std::vector<int>> lists = {{1}, {5, 0, 3}, {40, 1, 1, 1, 300, 2}, {0, 0}, {7, 7, 7, 7, 7, 7, 7}, {5000}};
  for (const auto &tiles : lists)
    for (int workers : {1, 4, 64, 1024}) {
        ++cases;
        int total = 0;
        for (int t : tiles) total += t > 0 ? t + SEGMENT_COST : 0;
        const int share = worker_share(total, workers);
        CHECK((int64_t)share * workers >= total);
        std::set<int> used;
        int t0 = 0;
        for (int t : tiles) {
          if (t == 0) continue;
          t0 += SEGMENT_COST;
          const SegmentPieces p = segment_pieces(t0, t0 + t, share);
          CHECK(p.first >= 0 && p.last < workers && p.first <= p.last && p.count() >= 1);
          if (p.first != p.last) {
            // every worker of the segment is covered by one piece, its own or its group's, in ascending order
            std::set<int> seen;
            int before = -1;
            for (int i = 0; i < p.count(); ++i) {
              const int w = p.worker(i);
              CHECK(w > before && w >= p.first && w <= p.last);
              before = w;
              const bool whole = group_inside(w / WORKER_GROUP, t0, t0 + t, share);
              CHECK(!whole || w % WORKER_GROUP == 0);
              for (int k = 0; k < (whole ? WORKER_GROUP : 1); ++k) CHECK(seen.insert(w + k).second);
              const int a = t0 > w * share ? t0 : w * share;
              const int slot = piece_slot(w, t0, share);
              CHECK(slot == 2 * w + (a > w * share));      // as the worker numbers it
              CHECK(used.insert(slot).second);
            }
            CHECK((int)seen.size() == p.last - p.first + 1 && *seen.begin() == p.first && *seen.rbegin() == p.last);
          }
          t0 += t;
        }
      }
  return cases;
}

int main() {
  for (int len = 0; len <= 300; ++len) {                         // the rest of a prefix behind its whole tiles
    const SeqWalk w = rest_walk(len, 300);
    CHECK(w.s2 == len / 64 * 64 && w.tiles == (len % 64 + 31) / 32 && w.T1 == 0 && w.e1 == 0 && w.lo == w.s2 && w.len == len);
    CHECK(w.tiles == 0 || (w.base(0) == w.s2 && w.base(w.tiles - 1) < len && w.i0 == len - 1));
  }
  const int a = walks(), b = shares(), c = rows();
  if (fails == 0) printf("ok walks %d shares %d rows %d\n", a, b, c);
  return fails != 0;
}
