// How the cache calls cut their work (plain C++: the kernels use it, and a test enumerates it on the host).
//
// A sequence's keys are walked in tiles of 32: of the slots 0 .. len-1 those that some of its n_new rows
// can see, the first n_init ones and the window that ends at the last token.  The tiles of all sequences and
// K/V heads form one list, and every worker (a wave) takes an equal, consecutive share of it: a batch of
// unequal lengths fills the chip as evenly as one of equal ones, and the lengths stay on the device.
#ifndef MINF_CACHE_WALK_H_
#define MINF_CACHE_WALK_H_

#include <stdint.h>

#ifdef __HIPCC__
#define MINF_HD __host__ __device__ inline
#else
#define MINF_HD inline
#endif

namespace minf {

constexpr int CACHE_TILE = 32, SHARED_TILE = 64;
// A segment (below) costs a worker its tiles and, for its rows and its result, as much as two more: it takes up so
// many places more in the list, in front of its tiles.
constexpr int SEGMENT_COST = 2;

// Tiles of one sequence: T1 tiles of the sink from slot 0 on, then the window's from slot s2 (a multiple of
// the tile) on.  Sink and window that touch in a tile are walked as one (T1 = 0, s2 = 0).
template <int TILE>
struct TileWalk {
  int32_t len, i0, T1, s2, tiles;       // i0: position of the first of the n_new rows (negative: no token)
  int32_t e1, lo;                       // some row sees the slots 0 .. e1 - 1 and lo .. len - 1, no row another one
  MINF_HD int32_t places() const { return tiles > 0 ? tiles + SEGMENT_COST : 0; }
  MINF_HD int32_t base(int32_t t) const { return t < T1 ? t * TILE : s2 + (t - T1) * TILE; }
  // tile that holds a slot, or -1
  MINF_HD int32_t tile_of(int32_t slot) const {
    if (slot < T1 * TILE) return slot / TILE;
    return slot >= s2 && slot < len ? T1 + (slot - s2) / TILE : -1;
  }
};
typedef TileWalk<CACHE_TILE> SeqWalk;

// n_init, n_local: at most the capacity, so that no sum here leaves 32 bits.
template <int TILE>
MINF_HD TileWalk<TILE> tile_walk(int32_t len, int32_t capacity, int32_t n_new, int32_t n_init, int32_t n_local) {
  TileWalk<TILE> w;
  w.len = len < 0 ? 0 : (len > capacity ? capacity : len);
  w.i0 = w.len - n_new;
  w.e1 = n_init < w.len ? n_init : w.len;
  w.lo = w.i0 - n_local + 1;
  if (w.lo < 0) w.lo = 0;
  w.s2 = w.lo / TILE * TILE;
  w.T1 = (w.e1 + TILE - 1) / TILE;
  if (w.s2 <= w.T1 * TILE) w.s2 = w.T1 = 0;
  w.tiles = w.T1 + (w.len - w.s2 + TILE - 1) / TILE;
  return w;
}
MINF_HD SeqWalk seq_walk(int32_t len, int32_t capacity, int32_t n_new, int32_t n_init, int32_t n_local) {
  return tile_walk<CACHE_TILE>(len, capacity, n_new, n_init, n_local);
}

// What is left of a prefix of len slots behind its whole tiles of 64.
MINF_HD SeqWalk rest_walk(int32_t len, int32_t capacity) {
  SeqWalk w = seq_walk(len, capacity, 1, 0, capacity);
  w.lo = w.s2 = w.len / SHARED_TILE * SHARED_TILE;
  w.e1 = w.T1 = 0;
  w.tiles = (w.len - w.s2 + CACHE_TILE - 1) / CACHE_TILE;
  return w;
}

// The rows first .. last of a sequence (row r is token r / group of its n_new): what they see.
MINF_HD TileWalk<SHARED_TILE> rows_walk(int32_t first, int32_t last, int32_t group, int32_t len, int32_t capacity, int32_t n_new,
                                        int32_t n_init, int32_t n_local) {
  len = len < 0 ? 0 : (len > capacity ? capacity : len);
  const int32_t t0 = first / group, t1 = last / group;
  int32_t end = len - n_new + t1 + 1;
  if (end < 0) end = 0;
  TileWalk<SHARED_TILE> w = tile_walk<SHARED_TILE>(end, capacity, t1 - t0 + 1, n_init, n_local);
  return w;
}

MINF_HD bool cache_visible(int32_t key, int32_t pos, int32_t n_init, int32_t n_local) {
  return key <= pos && (key < n_init || pos - key < n_local);
}

// Places per worker: equal shares.
MINF_HD int32_t worker_share(int32_t total, int32_t workers) {
  const int32_t c = (total + workers - 1) / workers;
  return c < 1 ? 1 : c;
}

// Workers come in groups (workgroups) of WORKER_GROUP.  The segment (one row tile of one sequence and K/V head)
// whose tiles lie at the places [t0, t1) of the list is taken by the workers first .. last, and leaves a piece per
// worker, except that a group whose places all lie in it joins its workers' pieces to one.
// Slots of the pieces: a part that begins at a worker's own first place takes the worker's slot 0 (so does a
// group's piece: of its first worker), another one slot 1; no worker has more than two parts of segments that
// it does not hold whole.
constexpr int WORKER_GROUP = 4;
MINF_HD bool group_inside(int32_t group, int32_t t0, int32_t t1, int32_t share) {
  const int32_t g0 = group * WORKER_GROUP * share;
  return g0 >= t0 && g0 + WORKER_GROUP * share <= t1;
}
struct SegmentPieces {
  int32_t first, last;              // workers
  int32_t g0, g1;                   // groups that lie inside (g0 >= g1: none)
  MINF_HD int32_t count() const { return g0 < g1 ? last - first + 1 - (g1 - g0) * (WORKER_GROUP - 1) : last - first + 1; }
  // worker whose slot holds piece i
  MINF_HD int32_t worker(int32_t i) const {
    const int32_t head = g0 * WORKER_GROUP - first;
    if (g0 >= g1 || i < head) return first + i;
    return i < head + g1 - g0 ? (g0 + i - head) * WORKER_GROUP : g1 * WORKER_GROUP + i - head - (g1 - g0);
  }
};
MINF_HD SegmentPieces segment_pieces(int32_t t0, int32_t t1, int32_t share) {
  SegmentPieces p;
  p.first = t0 / share;
  p.last = (t1 - 1) / share;
  const int32_t group_places = WORKER_GROUP * share;
  p.g0 = (t0 + group_places - 1) / group_places;
  p.g1 = t1 / group_places;
  return p;
}
MINF_HD int32_t piece_slot(int32_t worker, int32_t t0, int32_t share) {
  return 2 * worker + (t0 > worker * share ? 1 : 0);
}

// Tiles that the waves of a workgroup take together are cut into at most `splits` parts of equally many: tiles per part.
MINF_HD int32_t part_tiles(int32_t tiles, int32_t splits) { return (tiles + splits - 1) / splits; }
MINF_HD int32_t part_count(int32_t tiles, int32_t splits) {
  const int32_t per = part_tiles(tiles, splits);
  return per > 0 ? (tiles + per - 1) / per : 0;
}

}  // namespace minf
#endif
