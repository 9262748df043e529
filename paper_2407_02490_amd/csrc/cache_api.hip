// C ABI of the cache calls: argument validation, workspace layout and launches.  As in the prefill calls
// everything is checked on the host before anything is enqueued; no allocation, no synchronisation.
#include <math.h>
#include <string.h>

#include "batch_rule.h"
#include "cache_walk.h"
#include "minf_internal.h"

using namespace minf;

namespace {

constexpr int CUS = 256;
constexpr int32_t MAX_CAPACITY = 1 << 29;              // positions, and sums of a few of them, in 32 bits
constexpr int64_t MAX_BLOCKS = (1 << 24) - 1;          // of 256 threads, in one grid dimension

bool stride_ok(const int64_t (&s)[3], int head_dim) {
  for (int i = 0; i < 3; ++i)
    if (s[i] < 0 || s[i] % 8 != 0) return false;
  return s[2] >= head_dim && s[2] <= (int64_t)1 << 24;  // rows of a tile must fit 32-bit byte offsets
}
bool aligned16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

BatchLayout rows_of(const void *p, const int64_t (&s)[3], int batch, int heads, int tokens) {
  return BatchLayout{reinterpret_cast<uintptr_t>(p) / 2, s[0], s[1], s[2], batch, heads, tokens};
}

struct Range {
  uintptr_t from, to;
  bool meets(const Range &r) const { return from < r.to && r.from < to; }
};
Range range_of(const BatchLayout &x) { return Range{(uintptr_t)x.base * 2, (uintptr_t)(x.base + (uint64_t)x.end()) * 2}; }
Range weight_range(const minf_kv_cache *c) {
  const uintptr_t p = reinterpret_cast<uintptr_t>(c->weight);
  return Range{p, p + 4 * (uintptr_t)((c->batch - 1) * c->weight_stride[0] + (c->n_kv_heads - 1) * c->weight_stride[1] + c->capacity)};
}
Range lens_range(const int32_t *p, int n) {
  return Range{reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + 4 * (uintptr_t)n};
}
Range k_range(const minf_kv_cache *c) { return range_of(rows_of(c->k, c->k_stride, c->batch, c->n_kv_heads, c->capacity)); }
Range v_range(const minf_kv_cache *c) { return range_of(rows_of(c->v, c->v_stride, c->batch, c->n_kv_heads, c->capacity)); }

minf_status check_cache(const minf_kv_cache *c, bool need_weight, bool written) {
  if (!c || !c->k || !c->v || !c->lens || (need_weight && !c->weight)) return MINF_ERR_NULL;
  if (c->head_dim != 128) return MINF_ERR_SHAPE;
  if (c->batch < 1 || c->n_kv_heads < 1 || c->capacity < 1 || c->capacity > MAX_CAPACITY) return MINF_ERR_SHAPE;
  if ((int64_t)c->batch * c->n_kv_heads > 65535) return MINF_ERR_SHAPE;
  if (!stride_ok(c->k_stride, 128) || !stride_ok(c->v_stride, 128) || !aligned16(c->k) || !aligned16(c->v)) return MINF_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(c->lens) % 4 != 0) return MINF_ERR_SHAPE;
  if (need_weight) {
    if (reinterpret_cast<uintptr_t>(c->weight) % 4 != 0 || c->weight_stride[0] < 0 || c->weight_stride[1] < 0) return MINF_ERR_SHAPE;
    if (written) {                                                     // no two slots in one place
      const int64_t a = c->batch > 1 ? c->weight_stride[0] : INT64_MAX, b = c->n_kv_heads > 1 ? c->weight_stride[1] : INT64_MAX;
      const int64_t lo = a < b ? a : b, hi = a < b ? b : a;
      const int64_t n = a < b ? c->batch : c->n_kv_heads;
      if (lo < c->capacity) return MINF_ERR_SHAPE;
      if (hi != INT64_MAX && hi < (n - 1) * lo + c->capacity) return MINF_ERR_SHAPE;
    }
  }
  return MINF_OK;
}

minf_status check_queries(const minf_queries *x, const minf_kv_cache *c, bool need_o) {
  if (!x || !x->q || (need_o && !x->o)) return MINF_ERR_NULL;
  if (x->n_q_heads < 1 || x->n_q_heads % c->n_kv_heads != 0) return MINF_ERR_SHAPE;
  if (x->n_new < 1 || x->n_new > MINF_MAX_NEW) return MINF_ERR_BUDGET;
  if (!(x->softmax_scale >= 0.f) || isinf(x->softmax_scale)) return MINF_ERR_SHAPE;
  if (!stride_ok(x->q_stride, 128) || !aligned16(x->q)) return MINF_ERR_SHAPE;
  if ((int64_t)c->batch * x->n_q_heads * x->n_new > MAX_BLOCKS) return MINF_ERR_SHAPE;
  if (need_o) {
    if (!stride_ok(x->o_stride, 128) || !aligned16(x->o)) return MINF_ERR_SHAPE;
    if (!places_differ(rows_of(x->o, x->o_stride, c->batch, x->n_q_heads, x->n_new))) return MINF_ERR_SHAPE;
  }
  return MINF_OK;
}

// Everything but the workspace's addresses; need: its bytes.
struct Plan {
  CacheCall x;
  size_t need, at_ml, at_shared[2], at_shared_ml[2], at_stat, at_logits;     // [0] own, [1] prefix
};

// Segments of so few tiles that one workgroup each, all at a time, ends sooner than parts and their join.  (32 heads of
// 128, 256 and 512 keys, 24 rows: 14.2, 14.5, 15.1 us in parts, 8.4, 10.1, 13.4 whole; 80 rows: 16.6, 17.8, 18.8 and 11.2,
// 13.0, 17.9; 240 rows of 256 and 512 keys: 26.7, 29.1 and 14.8, 19.6.)
bool brief(int64_t segments, int64_t tiles) { return segments <= CUS && tiles <= 8; }

// How the rows of `heads` K/V heads (of a sequence) are taken, whole: 256 at a time: row tiles, and parts such that the
// workgroups, one per CU, come in rounds of least time.  A workgroup's start and end cost as much as six tiles.
// ragged: the tiles are those of a full cache, of several sequences whose lengths the host does not know.  Then the time
// counts as well that parts of any length, half of a full one on average, take when a CU that is done takes the next.
void plan_shared(SharedPart &p, int64_t heads, int64_t rows, int64_t tiles, bool whole, bool ragged) {
  p.on = 1;
  p.rows = (int32_t)rows;
  p.tile_rows = rows <= 64 ? 64 : rows <= 128 || !whole ? 128 : 256;
  p.row_tiles = (int32_t)((rows + p.tile_rows - 1) / p.tile_rows);
  p.splits = 1;
  const int64_t segments = heads * p.row_tiles, cost = 6;
  int64_t least = INT64_MAX;
  for (int s = 1; s <= 64 && s <= tiles; ++s) {
    const int64_t part = part_tiles((int32_t)tiles, s) + cost;
    int64_t time = (segments * s + CUS - 1) / CUS * part;
    if (ragged) time += segments * (tiles / 2 + cost * s) / CUS + part;
    if (time < least) { least = time; p.splits = s; }
  }
}

minf_status make_plan(const minf_queries *q, const minf_kv_cache *c, const minf_kv_cache *prefix, int32_t n_init,
                      int32_t n_local, int32_t weights, bool need_o, Plan &p) {
  minf_status s = check_cache(c, weights != MINF_WEIGHTS_NONE, true);
  if (s != MINF_OK) return s;
  if (prefix) {
    if ((s = check_cache(prefix, false, false)) != MINF_OK) return s;
    if (prefix->batch != 1 || prefix->n_kv_heads != c->n_kv_heads) return MINF_ERR_SHAPE;
  }
  if ((s = check_queries(q, c, need_o)) != MINF_OK) return s;
  if (weights < MINF_WEIGHTS_NONE || weights > MINF_WEIGHTS_ADD) return MINF_ERR_UNSUPPORTED;
  if (n_init < 0 || n_local < 1) return MINF_ERR_BUDGET;
  CacheCall &x = p.x;
  memset(&x, 0, sizeof(x));
  x.q = static_cast<const bf16_t *>(q->q); x.o = static_cast<bf16_t *>(q->o);
  x.k = static_cast<const bf16_t *>(c->k); x.v = static_cast<const bf16_t *>(c->v);
  x.lens = c->lens;
  x.q_sb = q->q_stride[0]; x.q_sh = q->q_stride[1]; x.q_st = q->q_stride[2];
  x.o_sb = q->o_stride[0]; x.o_sh = q->o_stride[1]; x.o_st = q->o_stride[2];
  x.k_sb = c->k_stride[0]; x.k_sh = c->k_stride[1]; x.k_st = c->k_stride[2];
  x.v_sb = c->v_stride[0]; x.v_sh = c->v_stride[1]; x.v_st = c->v_stride[2];
  x.batch = c->batch; x.n_kv = c->n_kv_heads; x.group = q->n_q_heads / c->n_kv_heads; x.n_new = q->n_new;
  x.capacity = c->capacity;
  x.n_init = n_init < c->capacity ? n_init : c->capacity;
  x.n_local = n_local < c->capacity ? n_local : c->capacity;
  const float scale = q->softmax_scale > 0.f ? q->softmax_scale : 1.0f / sqrtf((float)c->head_dim);
  x.c_log2 = scale * 1.4426950408889634f;
  x.rows = x.group * x.n_new;
  const int64_t p_rows = prefix ? (int64_t)x.batch * x.rows : 0;
  // the longest walk: sink and window, each with a tile that it fills in part
  const int64_t visible = (int64_t)x.n_init + x.n_local + x.n_new + 2 * SHARED_TILE, seen = visible < x.capacity ? visible : x.capacity;
  const bool ragged = x.batch > 1 && seen == x.capacity;               // walks of lengths that the host does not know
  // Rows that the workers take: up to 32, in one block of 16 or two.  With two a wave has its SIMD to itself, and where
  // the walks are alike in length waves that share tiles are faster: 20 rows, 4 heads of 40K, 30 -> 26 us, 32 sequences
  // with windows of 5K, 69 -> 61 (8 heads of 128K the same); 32 sequences of up to 32K, 198 -> 229.
  // So they are, of up to 64 rows, where a workgroup per K/V head and sequence takes it whole in no more time than the
  // launch of the join does (brief(); with weights that launch gives them as well): 8 heads of 64, 256 and 512 keys,
  // 4 rows each, 12.0, 12.4, 12.3 us by workers, 7.0, 8.9, 12.4 by one workgroup; 256 heads 13.7, 18.4, 24.1 and 7.6, 12.4, 16.9.
  const int64_t own_tiles = (seen + SHARED_TILE - 1) / SHARED_TILE, own_heads = (int64_t)x.batch * x.n_kv;
  const bool own_sh = x.rows > 32 || (x.rows > 16 && !prefix && !ragged) ||
                      (x.rows <= 64 && !prefix && weights == MINF_WEIGHTS_NONE && brief(own_heads, own_tiles));
  const bool p_sh = p_rows > 32;
  // (of a prefix of more than 128 rows only a rest of less than 64 slots)
  const int64_t most = own_sh ? (p_sh ? 0 : p_rows) : p_sh || p_rows < x.rows ? x.rows : p_rows;
  x.row_blocks = most <= 16 ? 1 : 2;
  const int tile_rows = 16 * x.row_blocks;
  x.row_tiles = own_sh ? 0 : (x.rows + tile_rows - 1) / tile_rows;
  x.p_row_tiles = p_sh && p_rows <= 128 ? 0 : (int32_t)((p_rows + tile_rows - 1) / tile_rows);
  x.slot_rows = prefix || x.rows > tile_rows ? tile_rows : x.rows;
  x.direct = !prefix;
  x.max_tiles = (int32_t)((seen + CACHE_TILE - 1) / CACHE_TILE);
  int64_t segments = (int64_t)x.batch * x.n_kv * x.row_tiles;
  int64_t places = segments * (x.max_tiles + SEGMENT_COST);
  if (own_sh) plan_shared(x.own_sh, own_heads, x.rows, own_tiles, false, ragged);
  if (own_sh && !prefix && brief(own_heads * x.own_sh.row_tiles, own_tiles)) x.own_sh.splits = 1;
  if (prefix) {
    x.pk = static_cast<const bf16_t *>(prefix->k); x.pv = static_cast<const bf16_t *>(prefix->v);
    x.p_lens = prefix->lens;
    x.pk_sh = prefix->k_stride[1]; x.pk_st = prefix->k_stride[2];
    x.pv_sh = prefix->v_stride[1]; x.pv_st = prefix->v_stride[2];
    x.p_cap = prefix->capacity;
    segments += (int64_t)x.n_kv * x.p_row_tiles;
    places += (int64_t)x.n_kv * x.p_row_tiles * ((prefix->capacity + CACHE_TILE - 1) / CACHE_TILE + SEGMENT_COST);
    if (p_sh) plan_shared(x.p_sh, x.n_kv, p_rows, (prefix->capacity + SHARED_TILE - 1) / SHARED_TILE, true, false);
  }
  if (places >= (int64_t)1 << 30) return MINF_ERR_SHAPE;               // the list of tiles is counted in 32 bits
  x.workers = CUS * 4;
  // workspace: O of the pieces, their references and sums, the same of the rows that waves take together, statistics
  // of the rows, logits (for the weights of up to 16 rows)
  const size_t slots = segments > 0 ? ((size_t)2 * x.workers + (size_t)segments) * x.slot_rows : 0;
  const size_t heads = (size_t)x.batch * x.n_kv;
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  p.at_ml = up(slots * 128 * sizeof(float));
  p.at_stat = p.at_ml + up(slots * sizeof(float2));
  for (int i = 0; i < 2; ++i) {
    const SharedPart &sh = i ? x.p_sh : x.own_sh;
    p.at_shared[i] = p.at_shared_ml[i] = p.at_stat;
    if (!sh.on) continue;
    const int64_t items = (int64_t)(i ? x.n_kv : heads) * sh.row_tiles * sh.splits;
    if (items + 8 * sh.row_tiles > MAX_BLOCKS / 2) return MINF_ERR_SHAPE;
    if (!i && sh.splits == 1 && x.direct) continue;                    // O is final
    p.at_shared_ml[i] = p.at_shared[i] + up((size_t)items * sh.tile_rows * 128 * sizeof(float));
    p.at_stat = p.at_shared_ml[i] + up((size_t)items * sh.tile_rows * sizeof(float2));
  }
  p.at_logits = p.need = p.at_stat;
  if (weights != MINF_WEIGHTS_NONE) {
    if ((int64_t)heads * (x.rows + (x.capacity + 1023) / 1024) > MAX_BLOCKS) return MINF_ERR_SHAPE;
    x.weight = c->weight;
    x.w_sb = c->weight_stride[0]; x.w_sh = c->weight_stride[1];
    x.add_weights = weights == MINF_WEIGHTS_ADD;
    p.at_logits = p.at_stat + up(heads * x.rows * sizeof(float2));
    p.need = p.at_logits;
    if (x.rows <= 16) p.need += up(heads * x.max_tiles * x.rows * CACHE_TILE * sizeof(float));
  }
  if (p.need == 0) p.need = 256;                                       // 0 is the answer to invalid arguments
  return MINF_OK;
}

// o over something that other workgroups still read, or weights over an input.  (o in the place of q: a workgroup reads
// its rows before it writes them; but the weights of more than 16 rows per K/V head are computed from q afterwards.)
bool outputs_meet_inputs(const minf_queries *q, const minf_kv_cache *c, const minf_kv_cache *prefix, bool weight) {
  const BatchLayout lo = rows_of(q->o, q->o_stride, c->batch, q->n_q_heads, q->n_new);
  const BatchLayout lq = rows_of(q->q, q->q_stride, c->batch, q->n_q_heads, q->n_new);
  const Range o = range_of(lo);
  const bool again = weight && q->n_q_heads / c->n_kv_heads * q->n_new > 16;
  const bool in_place = !again && lo.base == lq.base && lo.sb == lq.sb && lo.sh == lq.sh && lo.st == lq.st;
  if (weight) {
    const Range w = weight_range(c);
    if (w.meets(k_range(c)) || w.meets(v_range(c)) || w.meets(range_of(lq)) || w.meets(lens_range(c->lens, c->batch))) return true;
  }
  auto apart = [&](const void *p, const int64_t (&s)[3], int batch, int heads, int tokens) {
    return input_apart(lo, rows_of(p, s, batch, heads, tokens));
  };
  if (!in_place && !apart(q->q, q->q_stride, c->batch, q->n_q_heads, q->n_new)) return true;
  if (!apart(c->k, c->k_stride, c->batch, c->n_kv_heads, c->capacity) ||
      !apart(c->v, c->v_stride, c->batch, c->n_kv_heads, c->capacity)) return true;
  if (prefix && (!apart(prefix->k, prefix->k_stride, 1, prefix->n_kv_heads, prefix->capacity) ||
                 !apart(prefix->v, prefix->v_stride, 1, prefix->n_kv_heads, prefix->capacity))) return true;
  return o.meets(lens_range(c->lens, c->batch)) || (prefix && o.meets(lens_range(prefix->lens, 1))) ||
         (weight && o.meets(weight_range(c)));
}

minf_status run_plan(const minf_queries *q, const minf_kv_cache *c, const minf_kv_cache *prefix, int32_t n_init,
                     int32_t n_local, int32_t weights, void *ws, size_t ws_bytes, void *hip_stream) {
  Plan p;
  const minf_status s = make_plan(q, c, prefix, n_init, n_local, weights, true, p);
  if (s != MINF_OK) return s;
  if (outputs_meet_inputs(q, c, prefix, weights != MINF_WEIGHTS_NONE)) return MINF_ERR_SHAPE;
  if (!ws || ws_bytes < p.need || reinterpret_cast<uintptr_t>(ws) % 256 != 0) return MINF_ERR_WORKSPACE;
  char *w = static_cast<char *>(ws);
  p.x.piece_o = reinterpret_cast<float *>(w);
  p.x.piece_ml = reinterpret_cast<float2 *>(w + p.at_ml);
  for (int i = 0; i < 2; ++i) {
    SharedPart &sh = i ? p.x.p_sh : p.x.own_sh;
    sh.o = reinterpret_cast<float *>(w + p.at_shared[i]);
    sh.ml = reinterpret_cast<float2 *>(w + p.at_shared_ml[i]);
  }
  if (weights != MINF_WEIGHTS_NONE) {
    p.x.stat = reinterpret_cast<float2 *>(w + p.at_stat);
    if (p.x.rows <= 16) p.x.logits = reinterpret_cast<float *>(w + p.at_logits);
  }
  return launch_cache_attn(p.x, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? MINF_OK : MINF_ERR_HIP;
}

// The selection's cut and workspace.  Rows of up to 32K slots, what a workgroup holds in registers: one workgroup per
// row, one launch instead of four (calls, 8 rows of 8K / 16K / 32K: 15, 19, 30 us, in chunks 27, 28, 31; 256 rows: 65, 129,
// 244 and 78, 147, 268).  Longer ones in chunks of 4096 to 32768 slots (a chunk's counts are 16-bit numbers), small
// enough for one workgroup per CU.
struct EvictPlan {
  int32_t chunks, chunk_slots;
  size_t at_hist, at_state, need;
};
EvictPlan evict_plan(int64_t rows, int64_t capacity) {
  EvictPlan p;
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  p.chunks = 0;
  p.chunk_slots = 0;
  p.at_hist = p.at_state = p.need = up(rows * sizeof(int32_t));
  if (capacity <= 32768) return p;
  int64_t slots = (rows * capacity / CUS + 1023) / 1024 * 1024;
  slots = slots < 4096 ? 4096 : slots > 32768 ? 32768 : slots;
  p.chunk_slots = (int32_t)slots;
  p.chunks = (int32_t)((capacity + slots - 1) / slots);
  p.at_state = p.at_hist + up((size_t)3 * rows * p.chunks * 2048 * 2);
  p.need = p.at_state + up((size_t)rows * p.chunks * sizeof(SelectState));
  return p;
}

bool same_strides(const int64_t *a, const int64_t *b, int n) { return memcmp(a, b, n * sizeof(int64_t)) == 0; }

}  // namespace

extern "C" {

size_t minf_cache_attn_workspace_bytes(const minf_queries *x, const minf_kv_cache *cache, int32_t n_init,
                                       int32_t n_local, int32_t weights) {
  Plan p;
  return make_plan(x, cache, nullptr, n_init, n_local, weights, false, p) == MINF_OK ? p.need : 0;
}

size_t minf_prefix_attn_workspace_bytes(const minf_queries *x, const minf_kv_cache *prefix, const minf_kv_cache *cache) {
  Plan p;
  if (!prefix || !cache) return 0;
  return make_plan(x, cache, prefix, 0, cache->capacity, MINF_WEIGHTS_NONE, false, p) == MINF_OK ? p.need : 0;
}

size_t minf_cache_evict_workspace_bytes(const minf_kv_cache *cache, int32_t keep) {
  if (check_cache(cache, true, false) != MINF_OK || keep < 1) return 0;
  return evict_plan((int64_t)cache->batch * cache->n_kv_heads, cache->capacity).need;
}

minf_status minf_cache_attn(const minf_queries *x, const minf_kv_cache *cache, int32_t n_init, int32_t n_local,
                            int32_t weights, void *ws, size_t ws_bytes, void *hip_stream) {
  return run_plan(x, cache, nullptr, n_init, n_local, weights, ws, ws_bytes, hip_stream);
}

minf_status minf_prefix_attn(const minf_queries *x, const minf_kv_cache *prefix, const minf_kv_cache *cache,
                             void *ws, size_t ws_bytes, void *hip_stream) {
  if (!prefix || !cache) return MINF_ERR_NULL;
  return run_plan(x, cache, prefix, 0, cache->capacity > 0 ? cache->capacity : 1, MINF_WEIGHTS_NONE, ws, ws_bytes, hip_stream);
}

minf_status minf_cache_evict(const minf_kv_cache *cache, int32_t n_init, int32_t n_recent, int32_t keep,
                             const minf_kv_cache *to, int32_t *kept, void *ws, size_t ws_bytes, void *hip_stream) {
  if (!to || !kept) return MINF_ERR_NULL;
  minf_status s = check_cache(cache, true, false);
  if (s != MINF_OK) return s;
  if ((s = check_cache(to, true, true)) != MINF_OK) return s;
  if (to->batch != cache->batch || to->n_kv_heads != cache->n_kv_heads) return MINF_ERR_SHAPE;
  if (!places_differ(rows_of(to->k, to->k_stride, to->batch, to->n_kv_heads, to->capacity)) ||
      !places_differ(rows_of(to->v, to->v_stride, to->batch, to->n_kv_heads, to->capacity))) return MINF_ERR_SHAPE;
  // K, V and weights of `to` in places of their own: they move at the same time
  if (!input_apart(rows_of(to->k, to->k_stride, to->batch, to->n_kv_heads, to->capacity),
                   rows_of(to->v, to->v_stride, to->batch, to->n_kv_heads, to->capacity)) ||
      weight_range(to).meets(k_range(to)) || weight_range(to).meets(v_range(to))) return MINF_ERR_SHAPE;
  if (n_init < 0 || n_recent < 0 || keep < 1 || (int64_t)n_init + n_recent > keep) return MINF_ERR_BUDGET;
  const bool in_place = to->k == cache->k;
  if (in_place) {
    if (to->v != cache->v || to->weight != cache->weight || !same_strides(to->k_stride, cache->k_stride, 3) ||
        !same_strides(to->v_stride, cache->v_stride, 3) || !same_strides(to->weight_stride, cache->weight_stride, 2) ||
        to->capacity != cache->capacity)
      return MINF_ERR_SHAPE;
  } else {
    if (to->capacity < keep) return MINF_ERR_BUDGET;
    const Range from[3] = {k_range(cache), v_range(cache), weight_range(cache)};
    const Range into[3] = {k_range(to), v_range(to), weight_range(to)};
    for (const Range &a : into)
      for (const Range &b : from)
        if (a.meets(b)) return MINF_ERR_SHAPE;
  }
  // the slots of an in-place eviction end at the capacity: a larger keep keeps everything
  if (keep > cache->capacity && in_place) return MINF_ERR_BUDGET;
  const Range lists[2] = {Range{reinterpret_cast<uintptr_t>(kept), reinterpret_cast<uintptr_t>(kept) + 4 * (uintptr_t)keep * cache->batch * cache->n_kv_heads},
                          lens_range(to->lens, to->batch)};
  if (lists[0].from % 4 != 0) return MINF_ERR_SHAPE;
  for (int i = 0; i < 2; ++i) {
    const Range others[7] = {k_range(cache), v_range(cache), weight_range(cache), k_range(to), v_range(to), weight_range(to),
                             lists[1 - i]};
    for (const Range &r : others)
      if (lists[i].meets(r)) return MINF_ERR_SHAPE;
    if ((i == 0 || to->lens != cache->lens) && lists[i].meets(lens_range(cache->lens, cache->batch))) return MINF_ERR_SHAPE;
  }
  const EvictPlan p = evict_plan((int64_t)cache->batch * cache->n_kv_heads, cache->capacity);
  if (!ws || ws_bytes < p.need || reinterpret_cast<uintptr_t>(ws) % 256 != 0) return MINF_ERR_WORKSPACE;
  EvictCall x;
  x.k = static_cast<const bf16_t *>(cache->k); x.v = static_cast<const bf16_t *>(cache->v);
  x.to_k = static_cast<bf16_t *>(to->k); x.to_v = static_cast<bf16_t *>(to->v);
  x.weight = cache->weight; x.to_weight = to->weight;
  x.lens = cache->lens; x.to_lens = to->lens; x.kept = kept; x.counts = static_cast<int32_t *>(ws);
  x.k_sb = cache->k_stride[0]; x.k_sh = cache->k_stride[1]; x.k_st = cache->k_stride[2];
  x.v_sb = cache->v_stride[0]; x.v_sh = cache->v_stride[1]; x.v_st = cache->v_stride[2];
  x.w_sb = cache->weight_stride[0]; x.w_sh = cache->weight_stride[1];
  x.tk_sb = to->k_stride[0]; x.tk_sh = to->k_stride[1]; x.tk_st = to->k_stride[2];
  x.tv_sb = to->v_stride[0]; x.tv_sh = to->v_stride[1]; x.tv_st = to->v_stride[2];
  x.tw_sb = to->weight_stride[0]; x.tw_sh = to->weight_stride[1];
  x.batch = cache->batch; x.n_kv = cache->n_kv_heads; x.capacity = cache->capacity; x.to_capacity = to->capacity;
  x.n_init = n_init; x.n_recent = n_recent; x.keep = keep;
  x.chunks = p.chunks; x.chunk_slots = p.chunk_slots;
  x.hist = reinterpret_cast<uint32_t *>(static_cast<char *>(ws) + p.at_hist);
  x.state = reinterpret_cast<SelectState *>(static_cast<char *>(ws) + p.at_state);
  return launch_cache_evict(x, in_place, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? MINF_OK : MINF_ERR_HIP;
}

}  // extern "C"
