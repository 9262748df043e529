// Attention of new tokens against a KV cache, and eviction from it, for gfx950 (MI355X).
//
//   o_i = sum_j p_ij v_j,  p_ij = exp(c q_i k_j - m_i) / sum_j' exp(c q_i k_j' - m_i),  j over the visible slots
//   w_j (+)= sum over the rows i of a K/V head's group of p_ij
//
// Every key costs 512 bytes and, with R rows per K/V head, 512 R flops: up to some hundred rows the memory bounds
// it, so the kernels are built to keep loads in flight.
// Up to 16 rows, or 32 (cache_attn_kernel): a wave is a worker of its own.  It takes a consecutive share of the tiles of
// all sequences (cache_walk.h), fetches tile t+1 into its half of an LDS ring (global -> LDS, no registers) while it
// computes tile t, and meets no barrier.  Rows are the columns of 16x16x32 MFMAs (S^T = K Q^T, O^T += V^T P^T): the
// accumulator layout of S^T is the operand layout that the second product needs, so P never leaves registers.
// (8 heads of 4 rows, 128K keys: 537 MB of K and V, the call 103 us, 5.2 TB/s.)
// More rows (cache_shared_kernel, and cache_prefix_kernel for a prefix of more than 128): the waves of a workgroup
// share the tiles.
// A segment (row tile of a sequence and K/V head) that several workers or workgroups share leaves pieces
// (reference, sum, unnormalised O) in the workspace, which cache_join_kernel joins.
#include <type_traits>

#include "cache_walk.h"
#include "mfma_tile.h"

namespace minf {

constexpr int CACHE_WAVES = WORKER_GROUP;                       // per workgroup
constexpr int CACHE_RING = 2 * 2 * HALF_BYTES;                  // per wave: two slots of a K and a V tile
constexpr int CACHE_LOGITS = 8192;                              // per wave: logits on their way out
static_assert(CACHE_TILE * ROW_BYTES == HALF_BYTES, "a tile of the walk is half a 64-key tile");

__device__ inline int uni(int v) { return __builtin_amdgcn_readfirstlane(v); }

// ---- where a worker is in the list of tiles (wave-uniform) --------------------------------------------
// The kernel's arguments where they lie.  What a worker needs once per segment is read there, from an address
// the compiler knows nothing about: taken from `x` it would hold all of it in scalar registers, more than there
// are, through the tile loop.
typedef const __attribute__((address_space(4))) CacheCall CacheArgs;
__device__ inline CacheArgs &args_again(CacheArgs *p) {
  asm volatile("" : "+s"(p));
  return *p;
}

// Part of a segment (row tile of a sequence and K/V head) that a worker takes: its tiles t0 .. t1 - 1.
struct CachePart {
  int prefix;            // 1: the shared prefix
  int b, kvh, rt;        // sequence, K/V head, row tile
  int t0, t1;
  SeqWalk w;             // of the sequence (or of the prefix)
};

// Lengths: `mine` holds those of the first 64 sequences, one a lane, loaded once.
template <class X>
__device__ inline SeqWalk walk_of_len(X &x, int len) {
  return seq_walk(len, x.capacity, x.n_new, x.n_init, x.n_local);
}
template <class X>
__device__ inline int first_lens(X &x, int lane) { return lane < x.batch ? x.lens[lane] : 0; }
template <class X>
__device__ inline int places_of(X &x, int b, int mine) {       // b: 64 i + lane
  return b < x.batch ? walk_of_len(x, b < 64 ? mine : x.lens[b]).places() : 0;
}
template <class X>
__device__ inline SeqWalk walk_of(X &x, int b, int mine) {     // wave-uniform
  return walk_of_len(x, b < 64 ? __builtin_amdgcn_readlane(mine, b) : uni(x.lens[uni(b)]));
}
// What the workers take of the prefix, which every row sees: all of it, or what cache_prefix_kernel leaves.  (Nothing
// where there are no row tiles of theirs.)
template <class X>
__device__ inline SeqWalk prefix_walk(X &x) {
  const int len = x.p_cap > 0 ? uni(x.p_lens[0]) : 0;
  return x.p_sh.on ? rest_walk(len, x.p_cap) : seq_walk(len, x.p_cap, 1, 0, x.p_cap);
}

__device__ inline int wave_scan(int v, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int u = __shfl_up(v, d);
    if (lane >= d) v += u;
  }
  return v;
}

// Places of all sequences in the list, and of those in front of sequence b, per K/V head and row tile.
template <class X>
__device__ inline void count_places(X &x, int b, int mine, int lane, int &all, int &before) {
  all = before = 0;
  for (int b0 = 0; b0 < x.batch; b0 += 64) {
    const int t = places_of(x, b0 + lane, mine);
    all += t;
    before += b0 + lane < b ? t : 0;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    all += __shfl_xor(all, d);
    before += __shfl_xor(before, d);
  }
  all = uni(all);
  before = uni(before);
}

// The part that begins at place g of the list, of those before place g1 (none: t0 >= t1); pre: places of the prefix.
template <class X>
__device__ inline CachePart seek(X &x, int &g, int g1, int pre, int mine, int lane) {
  CachePart c;
  int s, at = g;
  if (g < pre) {
    c.prefix = 1;
    c.w = prefix_walk(x);
    s = uni(at / c.w.places());
    at -= s * c.w.places();
    c.b = 0; c.kvh = uni(s / x.p_row_tiles); c.rt = s - c.kvh * x.p_row_tiles;
  } else {
    at -= pre;
    const int heads = x.n_kv * x.row_tiles;
    int before = 0;
    c.prefix = 0;
    c.b = 0;
    for (int b0 = 0; b0 < x.batch; b0 += 64) {
      const int t = places_of(x, b0 + lane, mine);
      const int incl = wave_scan(t, lane);
      const unsigned long long beyond = __builtin_amdgcn_ballot_w64((before + incl) * heads > at);
      if (beyond != 0) {
        const int first = __builtin_ctzll(beyond);
        c.b = uni(b0 + first);
        before += uni(__shfl(incl, first)) - uni(__shfl(t, first));
        break;
      }
      before += uni(__shfl(incl, 63));
    }
    c.w = walk_of(x, c.b, mine);
    at -= before * heads;
    s = uni(at / c.w.places());
    at -= s * c.w.places();
    c.kvh = uni(s / x.row_tiles);
    c.rt = s - c.kvh * x.row_tiles;
  }
  const int head = max(SEGMENT_COST - at, 0);          // places in front of the first tile
  g += head;
  c.t0 = at + head - SEGMENT_COST;
  c.t1 = min(c.w.tiles, c.t0 + g1 - g);
  return c;
}

// The part behind c, of at most `most` tiles.
template <class X>
__device__ inline CachePart next_part(X &x, CachePart c, int most, int mine) {
  c.t0 = 0;
  if (++c.rt >= (c.prefix ? x.p_row_tiles : x.row_tiles)) {
    c.rt = 0;
    if (++c.kvh >= x.n_kv) {
      c.kvh = 0;
      if (c.prefix) { c.prefix = 0; c.b = -1; }
      do c.w = walk_of(x, ++c.b, mine);
      while (c.w.tiles == 0);                  // there is one: the list goes on
    }
  }
  c.t1 = min(c.w.tiles, most);
  return c;
}

template <class X>
__device__ inline int segment_of(X &x, const CachePart &c) {
  return c.prefix ? c.kvh * x.p_row_tiles + c.rt
                  : x.n_kv * x.p_row_tiles + (c.b * x.n_kv + c.kvh) * x.row_tiles + c.rt;
}

// ---- tile arithmetic ------------------------------------------------------------------------------------
// Rows of a segment: 16 NB per row tile.  Row r of a sequence is token r / group of the n_new, query head
// r % group of the K/V head's group; rows of the prefix are those of all sequences, one after the other.
// Lane l = 16 g + n holds, of row n of each block of 16: the query's d = 32 ks + 8 g + (0..7), the logits of the
// keys 4 g + (0..3) and 16 + 4 g + (0..3) of a tile, O at d = 16 db + 4 g + (0..3).
typedef float f32x4 __attribute__((ext_vector_type(4)));
template <int NB>
struct CacheQ {
  bf16x8 q[NB][4];
};
template <int NB>
struct CacheRows {
  CacheQ<NB> q;
  f32x4 o[NB][8];         // [row block][d block]
  float m[NB], l[NB];     // exponent reference of the row (base 2), this lane's share of the running sum
  int pos[NB];            // position of this lane's row: it sees the slots up to there
  int tok[NB];            // its token, 0 .. n_new - 1
};

struct LaneRow {
  int b, t, g;
};
template <class X>
__device__ inline LaneRow lane_row(X &x, const CachePart &c, int row) {
  LaneRow a;
  a.b = c.b;
  int r = row;
  if (c.prefix) { a.b = r / x.rows; r -= a.b * x.rows; }
  a.t = r / x.group;
  a.g = r - a.t * x.group;
  return a;
}
// This lane's row of block nb; rows behind the last one repeat it, nobody stores them.
template <int NB, class X>
__device__ inline LaneRow block_row(X &x, const CachePart &c, int nb, int lane) {
  const int last = (c.prefix ? x.batch * x.rows : x.rows) - 1;
  return lane_row(x, c, min((c.rt * NB + nb) * 16 + (lane & 15), last));
}

template <int NB, class X>
__device__ inline void load_queries(X &x, const CachePart &c, CacheQ<NB> &q, int lane) {
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const LaneRow a = block_row<NB>(x, c, nb, lane);
    const bf16_t *row = x.q + a.b * x.q_sb + (int64_t)(c.kvh * x.group + a.g) * x.q_sh + a.t * x.q_st + 8 * (lane >> 4);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) q.q[nb][ks] = *reinterpret_cast<const bf16x8 *>(row + 32 * ks);
  }
}

template <int NB, class X>
__device__ inline void begin_part(X &x, const CachePart &c, CacheRows<NB> &st, int lane) {
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const LaneRow a = block_row<NB>(x, c, nb, lane);
    st.tok[nb] = c.prefix ? 0 : a.t;
    st.pos[nb] = c.prefix ? c.w.len - 1 : c.w.i0 + a.t;
    st.m[nb] = -INFINITY;
    st.l[nb] = 0.f;
#pragma unroll
    for (int db = 0; db < 8; ++db) st.o[nb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
}

// Per-lane byte offsets of the MFMA operands in a tile (layout: mfma_tile.h).
struct CacheLane {
  int k[4];        // k step ks of key lane % 16; the second 16 keys lie 16 rows further, at the same swizzle
  int v[8];        // d block db of the keys 4 g .. 4 g + 3, transposed on reading
  __device__ inline void init(int lane) {
    const int n = lane & 15, g = lane >> 4, j = n >> 2, c = n & 3;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) k[ks] = swz_byte(n, 4 * ks + g);
#pragma unroll
    for (int db = 0; db < 8; ++db) v[db] = swz_byte(4 * g + j, 2 * db + (c >> 1)) + (c & 1) * 8;
  }
};
constexpr int HALF_TILE_ROWS = 16 * ROW_BYTES;
__device__ inline int lane_key(int lane, int e) { return 4 * (lane >> 4) + (e & 3) + 16 * (e >> 2); }

// Some value of the V tile is an infinity or NaN: the largest magnitude of its 16-bit numbers.
template <int BYTES>
__device__ inline bool tile_not_finite(const char *tV, int lane) {
  typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
  u16x8 most = 0;
#pragma unroll
  for (int i = 0; i < BYTES / 1024; ++i)
    most = __builtin_elementwise_max(most, *reinterpret_cast<const u16x8 *>(tV + i * 1024 + lane * 16) & (unsigned short)0x7fff);
  bool bad = false;
#pragma unroll
  for (int j = 0; j < 8; ++j) bad = bad || most[j] >= 0x7f80;
  return __builtin_amdgcn_ballot_w64(bad) != 0;
}

// Logits on their way to memory (for the weights).  They are collected in LDS, as they lie in memory, [tile][row][32],
// and go out in one burst of up to 8 KiB: memory that is read at full rate pays for writes in between by more than
// their bytes, and for small ones most.  (8 heads of 4 rows, 1M tokens, 4.3 GB read and 134 MB written: tiles stored
// one by one 963 us, in bursts 910, without the stores 717.  A loop that only reads and stores as much: 702 without
// stores, 960 with 1 KiB a tile, 855 with 8 KiB every 16 tiles, 813 with 32 KiB, for which LDS has no room.)
struct CacheLogits {
  char *room;            // CACHE_LOGITS bytes of LDS
  char *to;              // of the part's next tile in memory
  int tile_bytes, used;  // rows x 128; bytes waiting
  __device__ inline void flush(int lane) {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    for (int i = lane * 16; i < used; i += 1024) *reinterpret_cast<uint4 *>(to + i) = *reinterpret_cast<const uint4 *>(room + i);
    to += used;
    used = 0;
  }
};

// What the tiles of a part have in common.
struct CacheMask {
  int n_init, n_local, first_pos, last_pos, n_tok;
  // every row sees every key of the tile
  template <int TILE>
  __device__ inline bool whole(int kb) const {
    return kb + TILE - 1 <= first_pos && (kb + TILE - 1 < n_init || last_pos - kb < n_local);
  }
};

// O^T += V^T P^T for the tokens one by one, with the V rows that a token does not see as zeros: 0 * inf and
// 0 * NaN of a slot that a row's mask excludes would otherwise reach the row.  Only tiles with a mask and
// with such values take it, and only where there are several tokens: slots that no row sees are zeros.  O goes
// through 4 KiB of LDS (`room`), half of its d at a time, so that this rare path costs the others no registers.
// tV: 32 keys from kb on; P in PARTS parts.
template <int NB, int PARTS>
__device__ inline void update_by_token(CacheRows<NB> &st, const bf16x8 (&p)[NB][PARTS], const char *tV, char *room, int kb,
                                       const CacheMask &mask, int lane) {
  f32x4 *mine = reinterpret_cast<f32x4 *>(room) + lane;
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int db = 0; db < 4; ++db) mine[64 * db] = st.o[nb][4 * half + db];
#pragma unroll 1
      for (int i = 0; i < 4 * mask.n_tok; ++i) {
        const int db = i & 3, t = i >> 2;
        const int at = swz_byte(4 * (lane >> 4) + ((lane & 15) >> 2), 2 * (4 * half + db) + ((lane & 3) >> 1)) + (lane & 1) * 8;
        s16x8 w = __builtin_bit_cast(s16x8, lds_read_vt(tV, at, at + HALF_TILE_ROWS));
#pragma unroll
        for (int e = 0; e < 8; ++e)
          w[e] = cache_visible(kb + lane_key(lane, e), mask.first_pos + t, mask.n_init, mask.n_local) ? w[e] : (short)0;
        const bf16x8 a = __builtin_bit_cast(bf16x8, w);
        f32x4 add = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int part = 0; part < PARTS; ++part) add = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p[nb][part], add, 0, 0, 0);
        if (st.tok[nb] == t) mine[64 * db] += add;
      }
#pragma unroll
      for (int db = 0; db < 4; ++db) st.o[nb][4 * half + db] = mine[64 * db];
    }
}

// P of two logits as PARTS bf16.  One: rounded, off by half a step, 2^-8 of P.  Two: the high part is the largest bf16
// below P, what is left of it, at most a step (2^-7 of P's power of two), is the low part, rounded: off by 2^-16 of P.
// Both parts of P > 0 are greater than 0, so an infinity of V stays one: with a rounded high part the rest would be 0 or
// negative about every second time, and inf + 0 * inf or inf - inf is NaN.  (Down to P of 2^-102: a rest below 2^-126 is none.)
// P = 0 gives two zeros.
template <int PARTS>
__device__ inline void split_p(f32x2 v, bf16x2 (&part)[PARTS]) {
  if (PARTS == 1) {
    part[0] = __builtin_convertvector(v, bf16x2);
    return;
  }
  const float x = v[0], y = v[1];                              // (a bit cast of a vector's element takes the first one)
  const unsigned a = __builtin_elementwise_sub_sat(__builtin_bit_cast(unsigned, x), 1u);
  const unsigned b = __builtin_elementwise_sub_sat(__builtin_bit_cast(unsigned, y), 1u);
  part[0] = __builtin_bit_cast(bf16x2, __builtin_amdgcn_perm(b, a, 0x07060302u));
  const f32x2 rest = {x - __builtin_bit_cast(float, a & 0xffff0000u), y - __builtin_bit_cast(float, b & 0xffff0000u)};
  part[PARTS - 1] = __builtin_convertvector(rest, bf16x2);
}

// A row's exponent reference is its maximum when it was last taken, and REF_ROOM more: logits may outgrow that maximum by
// so much before it is taken anew, and nearly every tile needs no maximum across lanes and no rescaling.  P is at
// most 1 whenever (2^-16 for the maximum itself, which costs a sum in fp32 nothing): no product with V leaves fp32.
constexpr float REF_ROOM = 16.f;

// One tile of 32 keys from slot kb on.  EDGE: some row may not see some key.  keep: the logits are wanted (one
// block of rows).  wait_v awaits the V tile (the K tile is there); of an EDGE tile it clears the slots that no row sees.
template <int NB, bool EDGE, class WaitV>
__device__ inline void cache_tile(const CacheMask &mask, CacheRows<NB> &st, const CacheLane &lo, float c_log2, int kb,
                                  char *tK, const char *tV, bool keep, CacheLogits &out, int lane, WaitV wait_v) {
  f32x4 s[NB][2];
#pragma unroll
  for (int ks = 0; ks < 4; ++ks)
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const bf16x8 a = lds_read_k(tK, lo.k[ks] + kt * HALF_TILE_ROWS);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
        s[nb][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, st.q.q[nb][ks], ks == 0 ? zero : s[nb][kt], 0, 0, 0);
      }
    }
  if (EDGE) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        s[nb][e >> 2][e & 3] = cache_visible(kb + lane_key(lane, e), st.pos[nb], mask.n_init, mask.n_local) ? s[nb][e >> 2][e & 3] : -INFINITY;
  }
  bool outgrown = false;
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    float mx = s[nb][0][0];
#pragma unroll
    for (int e = 1; e < 8; ++e) mx = fmaxf(mx, s[nb][e >> 2][e & 3]);
    outgrown = outgrown || mx * c_log2 > st.m[nb];
  }
  if (__builtin_amdgcn_ballot_w64(outgrown) != 0) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float mx = s[nb][0][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) mx = fmaxf(mx, s[nb][e >> 2][e & 3]);
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32)) * c_log2;
      const float m_new = fmaxf(st.m[nb], mx + REF_ROOM);
      const float f = m_new == -INFINITY ? 1.f : fast_exp2(st.m[nb] - m_new);
      st.m[nb] = m_new;
      st.l[nb] *= f;
#pragma unroll
      for (int db = 0; db < 8; ++db) st.o[nb][db] *= f;
    }
  }
  // P as the sum of two bf16 (16 bits of mantissa): the matrix cores idle here, and the output is then as
  // good as from fp32 weights
  bf16x8 p[NB][2];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const float m = st.m[nb] == -INFINITY ? 0.f : st.m[nb];
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const f32x2 v = {fast_exp2(fmaf(s[nb][e >> 2][e & 3], c_log2, -m)), fast_exp2(fmaf(s[nb][e >> 2][(e & 3) + 1], c_log2, -m))};
      sum += v[0] + v[1];
      bf16x2 two[2];
      split_p<2>(v, two);
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        p[nb][part][e] = two[part][0];
        p[nb][part][e + 1] = two[part][1];
      }
    }
    st.l[nb] += sum;
  }
  wait_v(EDGE);
  if (EDGE && mask.n_tok > 1 && tile_not_finite<HALF_BYTES>(tV, lane)) {
    update_by_token<NB, 2>(st, p, tV, tK, kb, mask, lane);
  } else {
#pragma unroll
    for (int db = 0; db < 8; ++db) {
      const bf16x8 a = lds_read_vt(tV, lo.v[db], lo.v[db] + HALF_TILE_ROWS);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int part = 0; part < 2; ++part)
          st.o[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p[nb][part], st.o[nb][db], 0, 0, 0);
    }
  }
  if (NB == 1 && keep) {
    char *row = out.room + out.used + (lane & 15) * 128 + 16 * (lane >> 4);
    if (128 * (lane & 15) < out.tile_bytes) {
      *reinterpret_cast<f32x4 *>(row) = s[0][0] * c_log2;
      *reinterpret_cast<f32x4 *>(row + 64) = s[0][1] * c_log2;
    }
    out.used += out.tile_bytes;
    if (out.used + out.tile_bytes > CACHE_LOGITS) out.flush(lane);
  }
}

// A lane's row of O that is final.
template <int NB, class X>
__device__ inline void store_row(X &x, const CachePart &c, const CacheRows<NB> &st, int nb, int row, float l, int lane) {
  const LaneRow a = lane_row(x, c, row);
  const float inv = l > 0.f || l != l ? 1.0f / l : 0.f;
  bf16_t *to = x.o + a.b * x.o_sb + (int64_t)(c.kvh * x.group + a.g) * x.o_sh + a.t * x.o_st + 4 * (lane >> 4);
#pragma unroll
  for (int db = 0; db < 8; ++db) {
    const f32x4 r = st.o[nb][db] * inv;
    const f32x2 u = {r[0], r[1]}, w = {r[2], r[3]};
    uint2 two;
    two.x = __builtin_bit_cast(unsigned, __builtin_convertvector(u, bf16x2));
    two.y = __builtin_bit_cast(unsigned, __builtin_convertvector(w, bf16x2));
    *reinterpret_cast<uint2 *>(to + 16 * db) = two;
  }
  if (x.stat && lane < 16) x.stat[((int64_t)c.b * x.n_kv + c.kvh) * x.rows + row] = float2{st.m[nb], l};
}

// End of a worker's part of a segment: rows of O that are final go out, others into the workspace.
template <int NB, class X>
__device__ inline void end_part(X &x, const CachePart &c, const CacheRows<NB> &st, bool whole, int slot, int lane) {
  const int n = lane & 15, g = lane >> 4, rows = c.prefix ? x.batch * x.rows : x.rows;
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int row = (c.rt * NB + nb) * 16 + n;
    float l = st.l[nb] + __shfl_xor(st.l[nb], 16);
    l += __shfl_xor(l, 32);
    if (row >= rows) continue;
    if (whole && x.direct) {
      store_row<NB>(x, c, st, nb, row, l, lane);
      continue;
    }
    const int64_t at = (int64_t)slot * x.slot_rows + nb * 16 + n;
    if (g == 0) x.piece_ml[at] = float2{st.m[nb], l};
    float *to = x.piece_o + at * D + 4 * g;
#pragma unroll
    for (int db = 0; db < 8; ++db) *reinterpret_cast<f32x4 *>(to + 16 * db) = st.o[nb][db];
  }
}

// The same for the four waves of a workgroup whose parts are one segment's: their pieces become one.  lds: the rings.
template <int NB, class X>
__device__ inline void end_group(X &x, const CachePart &c, const CacheRows<NB> &st, char *lds, int lane) {
  constexpr int ROW = D * 4 + 16;                                      // 16 bytes between rows: banks
  constexpr int AT_ML = 16 * NB * ROW;
  const int n = lane & 15, g = lane >> 4, wave = uni(threadIdx.x >> 6);
  char *room = lds + wave * CACHE_RING;
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    float l = st.l[nb] + __shfl_xor(st.l[nb], 16);
    l += __shfl_xor(l, 32);
    if (g == 0) *reinterpret_cast<float2 *>(room + AT_ML + (16 * nb + n) * 8) = float2{st.m[nb], l};
#pragma unroll
    for (int db = 0; db < 8; ++db)
      *reinterpret_cast<f32x4 *>(room + (16 * nb + n) * ROW + (16 * db + 4 * g) * 4) = st.o[nb][db];
  }
  __syncthreads();
  const int first = c.rt * NB * 16, rows = min((c.prefix ? x.batch * x.rows : x.rows) - first, 16 * NB);
  const int64_t slot = 2 * WORKER_GROUP * (int64_t)blockIdx.x;
  for (int i = threadIdx.x; i < rows * 32; i += 64 * CACHE_WAVES) {
    const int row = i >> 5, d = 4 * (i & 31);
    float2 ml[CACHE_WAVES];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int w = 0; w < CACHE_WAVES; ++w) {
      ml[w] = *reinterpret_cast<const float2 *>(lds + w * CACHE_RING + AT_ML + row * 8);
      m = fmaxf(m, ml[w].x);
    }
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < CACHE_WAVES; ++w) {
      if (ml[w].x == -INFINITY && ml[w].y == 0.f) continue;            // no visible key
      const float f = fast_exp2(ml[w].x - m);
      l += ml[w].y * f;
      o += *reinterpret_cast<const f32x4 *>(lds + w * CACHE_RING + row * ROW + d * 4) * f;
    }
    const int64_t at = slot * x.slot_rows + row;
    if (d == 0) x.piece_ml[at] = float2{m, l};
    *reinterpret_cast<f32x4 *>(x.piece_o + at * D + d) = o;
  }
}

// Where a worker's tile loads come from: bases of the segment's K/V head, and the lanes' offsets inside 16 rows.
struct CacheSource {
  const char *kh, *vh;
  unsigned k_rb, v_rb;                 // bytes between rows
  unsigned kofs[4], vofs[4];
  __device__ static inline void lanes(unsigned (&ofs)[4], unsigned rb, int lane) {
    // the four 1 KiB blocks of 16 rows share a base and differ by the loads' immediate offset, which shifts the
    // global and the LDS address alike: block j has its row distance less 1024 j here
    const unsigned rl = lane >> 4, cpos = lane & 15;
#pragma unroll
    for (unsigned j = 0; j < 4; ++j) ofs[j] = (4 * j + rl) * rb + (((cpos ^ (rl << 2)) ^ j) << 4) - 1024 * j;
  }
  template <class X>
  __device__ inline void strides(X &x, int prefix, int lane) {
    k_rb = (unsigned)(prefix ? x.pk_st : x.k_st) * 2u;
    v_rb = (unsigned)(prefix ? x.pv_st : x.v_st) * 2u;
    lanes(kofs, k_rb, lane);
    lanes(vofs, v_rb, lane);
  }
  template <class X>
  __device__ inline void heads(X &x, const CachePart &c) {
    kh = reinterpret_cast<const char *>(c.prefix ? x.pk + c.kvh * x.pk_sh : x.k + c.b * x.k_sb + c.kvh * x.k_sh);
    vh = reinterpret_cast<const char *>(c.prefix ? x.pv + c.kvh * x.pv_sh : x.v + c.b * x.v_sb + c.kvh * x.v_sh);
  }
  // 16 rows from row0 on to the LDS address lds
  __device__ static inline void rows16(const char *row0, const unsigned (&ofs)[4], unsigned lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\t"
                 "global_load_lds_dwordx4 %0, %1\n\t"
                 "global_load_lds_dwordx4 %3, %1 offset:1024\n\t"
                 "global_load_lds_dwordx4 %4, %1 offset:2048\n\t"
                 "global_load_lds_dwordx4 %5, %1 offset:3072"
                 :: "v"(ofs[0]), "s"(row0), "s"(lds), "v"(ofs[1]), "v"(ofs[2]), "v"(ofs[3]) : "memory");
  }
  // 8 rows, the first or the second ones of 16 (their offsets: two of the four; row0, lds: of the 16, plus 2048 for the second)
  __device__ static inline void rows8(const char *row0, unsigned ofs0, unsigned ofs1, unsigned lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\t"
                 "global_load_lds_dwordx4 %0, %1\n\t"
                 "global_load_lds_dwordx4 %3, %1 offset:1024"
                 :: "v"(ofs0), "s"(row0), "s"(lds), "v"(ofs1) : "memory");
  }
  // 32 rows from kb on into the tile at lds
  __device__ static inline void tile(const char *h, unsigned rb, const unsigned (&ofs)[4], int kb, unsigned lds) {
#pragma unroll
    for (int half = 0; half < 2; ++half) rows16(h + (uint64_t)(unsigned)(kb + 16 * half) * rb, ofs, lds + 4096 * half);
  }
  // some row sees every slot kb .. end - 1
  template <class Walk>
  __device__ static inline bool all_seen(int kb, int end, const Walk &w) { return end <= w.len && (kb >= w.lo || end <= w.e1); }
  // BLOCKS times four rows of the tile at kb, from row `first` on, one by one: slots that no row of the call sees are
  // replaced by one that some row does
  template <int BLOCKS, class Walk>
  __device__ static inline void rows_in_part(const char *h, unsigned rb, int kb, int first, const Walk &w, unsigned lds, int lane) {
    const int rl = lane >> 4, cpos = lane & 15;
#pragma unroll
    for (int blk = 0; blk < BLOCKS; ++blk) {
      const int r = first + 4 * blk + rl;
      int key = kb + r;
      if (key >= w.e1) key = max(key, w.lo);
      key = min(key, w.len - 1);
      dma16(h + (uint64_t)(unsigned)key * rb + ((cpos ^ swz_f(r)) << 4), lds + (first + 4 * blk) * ROW_BYTES);
    }
  }
  // ... and, where those rows of V are there, by zeros: P = 0 times an infinity of the one that took their place is NaN.
  // (Nothing of this may be kept in registers through a loop over tiles, which nearly never takes it: with the zeros and
  // addresses held the tile loop of 128 rows had its operands read one by one, the prefix of 128K 101 -> 116 us.)
  template <int BLOCKS, class Walk>
  __device__ static inline void zero_unseen(char *tV, int kb, int first, const Walk &w, int lane) {
    unsigned zero = 0;
    asm volatile("" : "+v"(zero), "+v"(lane));
#pragma unroll
    for (int blk = 0; blk < BLOCKS; ++blk) {
      const int key = kb + first + 4 * blk + (lane >> 4);
      if (key >= w.len || (key >= w.e1 && key < w.lo))
        *reinterpret_cast<uint4 *>(tV + (first + 4 * blk) * ROW_BYTES + 16 * lane) = uint4{zero, zero, zero, zero};
    }
  }
  __device__ inline void fetch(int kb, const SeqWalk &w, unsigned lds, int lane) const {
    if (all_seen(kb, kb + CACHE_TILE, w)) {
      tile(kh, k_rb, kofs, kb, lds);
      tile(vh, v_rb, vofs, kb, lds + HALF_BYTES);
    } else {
      rows_in_part<8>(kh, k_rb, kb, 0, w, lds, lane);
      rows_in_part<8>(vh, v_rb, kb, 0, w, lds + HALF_BYTES, lane);
    }
  }
};

// Two waves per SIMD fit (256 registers): with more to hand out the compiler moves O between register files
// in every tile.
template <int NB>
__global__ __launch_bounds__(64 * CACHE_WAVES, NB == 1 ? 2 : 1) void cache_attn_kernel(CacheCall) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  CacheArgs *args = (CacheArgs *)__builtin_amdgcn_kernarg_segment_ptr();
  const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6);
  const int worker = blockIdx.x * CACHE_WAVES + wave;
  char *ring = lds + wave * CACHE_RING;
  const unsigned ring_at = uni(lds_addr_of(ring));

  int first_place, g, g1, share;             // place of the current part's first tile, end of this worker's places
  const int mine = first_lens(*args, lane);
  CachePart cur;
  {
    CacheArgs &x = args_again(args);
    const int pre = prefix_walk(x).places() * x.n_kv * x.p_row_tiles;
    int all, before;
    count_places(x, 0, mine, lane, all, before);
    const int total = pre + all * x.n_kv * x.row_tiles;
    share = worker_share(total, x.workers);
    first_place = g = worker * share;
    g1 = min(g + share, total);
    if (g >= g1) return;
    cur = seek(x, g, g1, pre, mine, lane);
    if (cur.t0 >= cur.t1) return;
  }
  CacheSource src;
  CacheRows<NB> st;
  CacheQ<NB> q;                              // rows of the next part, loaded ahead of its first tile (loads return in order)
  {
    CacheArgs &x = args_again(args);
    src.strides(x, cur.prefix, lane);
    src.heads(x, cur);
    load_queries<NB>(x, cur, st.q, lane);
  }
  src.fetch(cur.w.base(cur.t0), cur.w, ring_at, lane);
  CacheLane lo;
  lo.init(lane);
  const float c_log2 = args->c_log2;
  unsigned slot = 0;
  // The compiler waits for the rows where they are used first.  Here, once: inside the loop it would wait for all
  // loads in every iteration, the tiles' too.
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) asm volatile("" : "+v"(st.q.q[nb][ks]));
  CacheLogits out;
  out.room = lds + CACHE_WAVES * CACHE_RING + wave * CACHE_LOGITS;
  out.used = 0;
  for (;;) {                                 // part by part
    const int left = g1 - g - (cur.t1 - cur.t0) - SEGMENT_COST;        // tiles of the next one at most
    CachePart nxt;
    CacheMask mask;
    bool keep;
    {
      CacheArgs &x = args_again(args);
      if (left > 0) nxt = next_part(x, cur, left, mine);
      begin_part<NB>(x, cur, st, lane);
      mask.n_init = cur.prefix ? 0 : x.n_init;
      mask.n_local = cur.prefix ? x.p_cap : x.n_local;
      mask.first_pos = cur.prefix ? cur.w.len - 1 : cur.w.i0;
      mask.last_pos = cur.w.len - 1;
      mask.n_tok = cur.prefix ? 1 : x.n_new;
      keep = NB == 1 && x.logits && !cur.prefix;
      out.tile_bytes = x.rows * CACHE_TILE * 4;
      out.to = reinterpret_cast<char *>(x.logits) +
               (((int64_t)cur.b * x.n_kv + cur.kvh) * x.max_tiles + cur.t0) * out.tile_bytes;
    }
    for (int t = cur.t0, kb = cur.w.base(t); t < cur.t1; ++t) {
      const int kb_next = t + 1 == cur.w.T1 ? cur.w.s2 : kb + CACHE_TILE;
      const bool more = t + 1 < cur.t1 || left > 0;
      if (t + 1 < cur.t1) {
        src.fetch(kb_next, cur.w, ring_at + (slot ^ 2 * HALF_BYTES), lane);
      } else if (left > 0) {
        CacheArgs &x = args_again(args);
        if (nxt.prefix != cur.prefix) src.strides(x, nxt.prefix, lane);
        src.heads(x, nxt);
        load_queries<NB>(x, nxt, q, lane);
        src.fetch(nxt.w.base(0), nxt.w, ring_at + (slot ^ 2 * HALF_BYTES), lane);
      }
      if (more) MINF_WAIT_VMCNT(24); else MINF_WAIT_VMCNT(8);     // K has landed
      char *tK = ring + slot;
      auto wait_v = [&](bool edge) {
        if (more) MINF_WAIT_VMCNT(16); else MINF_WAIT_VMCNT(0);
        if (edge && !src.all_seen(kb, kb + CACHE_TILE, cur.w)) src.zero_unseen<8>(tK + HALF_BYTES, kb, 0, cur.w, lane);
      };
      if (mask.whole<CACHE_TILE>(kb)) cache_tile<NB, false>(mask, st, lo, c_log2, kb, tK, tK + HALF_BYTES, keep, out, lane, wait_v);
      else cache_tile<NB, true>(mask, st, lo, c_log2, kb, tK, tK + HALF_BYTES, keep, out, lane, wait_v);
      __builtin_amdgcn_s_waitcnt(0xC07F);    // LDS reads done: the slot may be filled again
      slot ^= 2 * HALF_BYTES;
      kb = kb_next;
    }
    {
      CacheArgs &x = args_again(args);
      if (keep) out.flush(lane);
      const int t0 = g - cur.t0;
      if (group_inside(blockIdx.x, t0, t0 + cur.w.tiles, share)) {     // the four waves' only part
        end_group<NB>(x, cur, st, lds, lane);
        break;
      }
      const bool whole = cur.t0 == 0 && cur.t1 == cur.w.tiles;
      end_part<NB>(x, cur, st, whole, whole ? 2 * x.workers + segment_of(x, cur) : 2 * worker + (g > first_place ? 1 : 0), lane);
    }
    if (left <= 0) break;
    g += cur.t1 - cur.t0 + SEGMENT_COST;
    st.q = q;
    cur = nxt;
  }
}

// ---- many rows (from 17 or 33 on) -----------------------------------------------------------------------
// HALVES = 2: eight waves share 64-key tiles (a ring of four: loads go out three tiles ahead, one barrier a tile); four
// take the first 32 keys and four the others, 16 NB rows each, 64 or 128 rows a workgroup; at the end the two halves' sums
// are joined in LDS.  So a SIMD has two waves, one's exponentials beside the other's products, and no operand is read from
// LDS more often than with four.  The barrier of every tile would keep both in the same phase; priority pulls them apart:
// of a prefix the first half's waves have it, else the wave in its exponentials (the calls of the two sizes below,
// neither 137 and 74.3 us, the first half 130 and 73.9, the exponentials 133 and 73.5).
// HALVES = 1: four waves, 32-key tiles, two workgroups a CU, which overlap each other's starts and ends.  Taken of 128 rows
// a workgroup where there are more workgroups than CUs (4 heads of 32 sequences of 32K, 128 and 256 rows: 479 and 842 us with
// two halves, 438 and 784 with one; of up to 32K 282 and 492, 288 and 457; 64 rows 409 and 391, 126 short sequences 98 and 100).
// Memory bounds 128 rows (32 KiB a tile take a CU 1.4 us), the arithmetic more of them.
// (128 rows, 8 heads of 128K tokens, and 256 rows, 4 heads of 40K: 107 and 37 us; four waves with all 64 keys 120 and
// 44; HALVES = 1 109 and 39, and twice the pieces to join, 3 us more; eight waves of 16 rows, which read every operand
// twice as often, 132 us for the 128 rows; the 256-row loop of cache_prefix_kernel 142.)
// P in two bf16 up to 64 rows.  Beyond in one, as in the prefill kernels: off by 2^-8 of a probability at most, which is
// what O itself is rounded by, and the errors of many keys cancel in part; the product of its rest would cost the same two
// calls 27 and 8 us.
// A workgroup takes one part (of x.*_sh.splits) of the tiles that its rows see; a segment in one part is final, of
// others reference, sum and unnormalised O go to the workspace for cache_join_kernel.
// Launch order: the row tiles that read the same slots run on one XCD, one after the other.
constexpr int SHARED_ROOM = 4096;                                            // per wave: update_by_token
constexpr int shared_waves(int halves) { return 4 * halves; }
constexpr int shared_ring(int halves) { return 4 * 2 * HALF_BYTES * halves; }
template <int NB, bool PREFIX, int HALVES>
__global__ __launch_bounds__(64 * shared_waves(HALVES), 2) void cache_shared_kernel(CacheCall x) {
  constexpr int KEYS = CACHE_TILE * HALVES, BYTES = HALF_BYTES * HALVES;     // of a tile
  constexpr int W = 4, PARTS = NB == 1 ? 2 : 1, prefix = PREFIX;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wave = to_sgpr(threadIdx.x >> 6);
  const int half = to_sgpr(wave / W), row_wave = wave - half * W;            // of a tile's keys; of the rows
  const SharedPart &sh = prefix ? x.p_sh : x.own_sh;
  const int splits = sh.splits, tile_rows = 16 * NB * W;
  const int per_xcd = blockIdx.x >> 3, turn = to_sgpr(per_xcd / sh.row_tiles), rt = per_xcd - turn * sh.row_tiles;
  const int group = turn * 8 + (blockIdx.x & 7);                             // (K/V head of a sequence, part of the tiles)
  const int heads = (prefix ? 1 : x.batch) * x.n_kv;
  if (group >= heads * splits) return;
  const int head = to_sgpr(group / splits), part = group - head * splits;
  CachePart c;
  c.prefix = prefix;
  c.b = prefix ? 0 : to_sgpr(head / x.n_kv);
  c.kvh = head - c.b * x.n_kv;
  c.rt = rt * W + row_wave;                                                  // row tile of 16 NB rows
  const int last_row = min((rt + 1) * tile_rows, sh.rows) - 1;
  const int len = to_sgpr(prefix ? x.p_lens[0] : x.lens[c.b]);
  const TileWalk<SHARED_TILE> w = prefix ? tile_walk<SHARED_TILE>(len, x.p_cap, 1, 0, x.p_cap)
                                         : rows_walk(rt * tile_rows, last_row, x.group, len, x.capacity, x.n_new, x.n_init, x.n_local);
  const bool final = !prefix && x.direct && splits == 1;
  const int per = to_sgpr(part_tiles(w.tiles, splits)), t0 = part * per, n = min(per, w.tiles - t0);
  if (n <= 0 && !final) return;

  CacheMask mask;
  mask.n_init = prefix ? 0 : x.n_init;
  mask.n_local = prefix ? x.p_cap : x.n_local;
  mask.first_pos = prefix ? w.len - 1 : min(max(len, 0), x.capacity) - x.n_new + rt * tile_rows / x.group;
  mask.last_pos = w.len - 1;
  mask.n_tok = prefix ? 1 : last_row / x.group - rt * tile_rows / x.group + 1;
  CacheSource src;
  src.strides(x, prefix, lane);
  src.heads(x, c);
  const unsigned ring = uni(lds_addr_of(lds));
  const int upper = wave & 1, tiles = n * (SHARED_TILE / KEYS);
  auto base = [&](int i) { return HALVES == 2 ? w.base(t0 + i) : w.base(t0 + (i >> 1)) + CACHE_TILE * (i & 1); };
  const unsigned k0 = upper ? src.kofs[2] : src.kofs[0], k1 = upper ? src.kofs[3] : src.kofs[1];
  const unsigned v0 = upper ? src.vofs[2] : src.vofs[0], v1 = upper ? src.vofs[3] : src.vofs[1];
  auto fetch = [&](int i) {                                                  // a wave: 8 rows of K and of V
    const unsigned to = ring + (i & 3) * (2 * BYTES);
    const int kb = base(min(i, tiles - 1));
    if (src.all_seen(kb, kb + KEYS, w)) {
      const int row = kb + 16 * (wave >> 1);
      const unsigned at = to_sgpr(to + 2048 * wave);
      src.rows8(src.kh + (uint64_t)(unsigned)row * src.k_rb + 2048 * upper, k0, k1, at);
      src.rows8(src.vh + (uint64_t)(unsigned)row * src.v_rb + 2048 * upper, v0, v1, at + BYTES);
    } else {
      src.template rows_in_part<2>(src.kh, src.k_rb, kb, 8 * wave, w, to, lane);
      src.template rows_in_part<2>(src.vh, src.v_rb, kb, 8 * wave, w, to + BYTES, lane);
    }
  };
  CacheRows<NB> st;
  load_queries<NB>(x, c, st.q, lane);
  // (awaited here: behind the tiles' loads the wait would be for all three tiles, 1.5 us more)
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) asm volatile("" : "+v"(st.q.q[nb][ks]));
  if (n > 0) {
    fetch(0);
    fetch(1);
    fetch(2);
  }
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int t = block_row<NB>(x, c, nb, lane).t;
    st.tok[nb] = prefix ? 0 : t - rt * tile_rows / x.group;
    st.pos[nb] = mask.first_pos + st.tok[nb];
    st.m[nb] = -INFINITY;
    st.l[nb] = 0.f;
#pragma unroll
    for (int db = 0; db < 8; ++db) st.o[nb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  CacheLane lo;
  lo.init(lane);
  const float c_log2 = x.c_log2;
  if (PREFIX && half == 0) __builtin_amdgcn_s_setprio(1);
  for (int i = 0; i < tiles; ++i) {
    MINF_WAIT_VMCNT(8);                        // this wave's part of tile i; those of i + 1 and i + 2 may run
    if (!src.all_seen(base(i), base(i) + KEYS, w))
      src.template zero_unseen<2>(lds + (i & 3) * (2 * BYTES) + BYTES, base(i), 8 * wave, w, lane);
    __syncthreads();                           // all of tile i is there; all waves are done with tile i - 1
    fetch(i + 3);                              // behind the last tile it is repeated: every tile issues as many loads
    const char *tK = lds + (i & 3) * (2 * BYTES) + half * HALF_BYTES, *tV = tK + BYTES;
    const int kb = base(i) + CACHE_TILE * half;
    f32x4 s[2][NB];                            // [16 keys][row block]
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        const bf16x8 a = lds_read_k(tK, lo.k[ks] + kt * HALF_TILE_ROWS);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
          s[kt][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, st.q.q[nb][ks], ks == 0 ? zero : s[kt][nb], 0, 0, 0);
        }
      }
    if (!PREFIX) __builtin_amdgcn_s_setprio(1);
    const bool edge = !mask.whole<CACHE_TILE>(kb);
    if (edge) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          s[e >> 2][nb][e & 3] = cache_visible(kb + 16 * (e >> 2) + 4 * (lane >> 4) + (e & 3), st.pos[nb], mask.n_init, mask.n_local)
                                     ? s[e >> 2][nb][e & 3] : -INFINITY;
    }
    bool outgrown = false;
    float mx[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      mx[nb] = s[0][nb][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) mx[nb] = fmaxf(mx[nb], s[e >> 2][nb][e & 3]);
      outgrown = outgrown || mx[nb] * c_log2 > st.m[nb];
    }
    if (__builtin_amdgcn_ballot_w64(outgrown) != 0) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float most = fmaxf(mx[nb], __shfl_xor(mx[nb], 16));
        most = fmaxf(most, __shfl_xor(most, 32)) * c_log2;
        const float m_new = fmaxf(st.m[nb], most + REF_ROOM);
        const float f = m_new == -INFINITY ? 1.f : fast_exp2(st.m[nb] - m_new);
        st.m[nb] = m_new;
        st.l[nb] *= f;
#pragma unroll
        for (int db = 0; db < 8; ++db) st.o[nb][db] *= f;
      }
    }
    bf16x8 p[NB][PARTS];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const float m = st.m[nb] == -INFINITY ? 0.f : st.m[nb];
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const f32x4 &v4 = s[e >> 2][nb];
        const f32x2 v = {fast_exp2(fmaf(v4[e & 3], c_log2, -m)), fast_exp2(fmaf(v4[(e & 3) + 1], c_log2, -m))};
        sum += v[0] + v[1];
        bf16x2 two[PARTS];
        split_p<PARTS>(v, two);
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
          p[nb][part][e] = two[part][0];
          p[nb][part][e + 1] = two[part][1];
        }
      }
      st.l[nb] += sum;
    }
    if (!PREFIX) __builtin_amdgcn_s_setprio(0);
    if (!PREFIX && edge && mask.n_tok > 1 && tile_not_finite<HALF_BYTES>(tV, lane)) {
      update_by_token<NB, PARTS>(st, p, tV, lds + shared_ring(HALVES) + wave * SHARED_ROOM, kb, mask, lane);
    } else {
#pragma unroll
      for (int db = 0; db < 8; ++db) {
        const bf16x8 a = lds_read_vt(tV, lo.v[db], lo.v[db] + HALF_TILE_ROWS);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int part = 0; part < PARTS; ++part)
            st.o[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p[nb][part], st.o[nb][db], 0, 0, 0);
      }
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);        // LDS reads done
  }
  MINF_WAIT_VMCNT(0);                          // the repeated loads
  if (HALVES == 2) {
    // The two halves' sums, in the place of the ring: the same lane has the same row and the same d of both.
    __syncthreads();
    f32x4 *other_o = reinterpret_cast<f32x4 *>(lds) + row_wave * (NB * 8 * 64) + lane;
    float2 *other_ml = reinterpret_cast<float2 *>(lds + W * NB * 8 * 64 * 16) + row_wave * (NB * 64) + lane;
    if (half == 1) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        other_ml[64 * nb] = float2{st.m[nb], st.l[nb]};
#pragma unroll
        for (int db = 0; db < 8; ++db) other_o[64 * (8 * nb + db)] = st.o[nb][db];
      }
    }
    __syncthreads();
    if (half == 1) return;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const float2 ml = other_ml[64 * nb];
      const float m = fmaxf(st.m[nb], ml.x);
      // (-inf: no key was seen, the sums are 0)
      const float f0 = st.m[nb] == -INFINITY ? 1.f : fast_exp2(st.m[nb] - m), f1 = ml.x == -INFINITY ? 1.f : fast_exp2(ml.x - m);
      st.m[nb] = m;
      st.l[nb] = st.l[nb] * f0 + ml.y * f1;
#pragma unroll
      for (int db = 0; db < 8; ++db) st.o[nb][db] = st.o[nb][db] * f0 + other_o[64 * (8 * nb + db)] * f1;
    }
  }
  const int64_t item = ((int64_t)head * sh.row_tiles + rt) * splits + part;
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int in_tile = (row_wave * NB + nb) * 16 + (lane & 15), row = rt * tile_rows + in_tile;
    float l = st.l[nb] + __shfl_xor(st.l[nb], 16);
    l += __shfl_xor(l, 32);
    if (row >= sh.rows) continue;
    if (final) {
      store_row<NB>(x, c, st, nb, row, l, lane);
      continue;
    }
    const int64_t at = item * tile_rows + in_tile;
    if (lane < 16) sh.ml[at] = float2{st.m[nb], l};
    float *to = sh.o + at * D + 4 * (lane >> 4);
#pragma unroll
    for (int db = 0; db < 8; ++db) *reinterpret_cast<f32x4 *>(to + 16 * db) = st.o[nb][db];
  }
}

// ---- joining the pieces ---------------------------------------------------------------------------------
// o = sum_p 2^(m_p - M) O_p / sum_p 2^(m_p - M) l_p over the pieces of the row's own segment and of the prefix's.
// Four waves share a row (W = 4: every fourth piece each) or, of many rows, each wave takes one (W = 1); eight pieces at
// a time with all their loads in flight.  Rows without a visible key, or without a token, give zeros.
// Further workgroups give the slots their weights (where the logits were kept): they need the references and sums
// of a K/V head's rows, which they join themselves, rather than wait for another launch.
constexpr int JOIN_WAVES = 4, JOIN_AHEAD = 8;

// The pieces that the workers left of a segment.
struct PieceList {
  SegmentPieces p;
  int t0, share, segment;
  int64_t base;                            // row of slot 0
  int slot_rows, workers;
  __device__ inline int count() const { return p.first == p.last ? 1 : p.count(); }
  __device__ inline int64_t at(int i) const {
    const int slot = p.first == p.last ? 2 * workers + segment : piece_slot(p.worker(i), t0, share);
    return (int64_t)slot * slot_rows + base;
  }
};

// SHARED: with rows that several waves took together (without them the code is smaller, which a short call notices).
template <int W, bool SHARED>
__global__ __launch_bounds__(64 * JOIN_WAVES) void cache_join_kernel(CacheCall x, int tile_rows, int joins) {
  const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6);
  const bool joining = (int)blockIdx.x < joins;
  // joining: the row of a K/V head of a sequence; else 1024 slots of one
  const int per_head = joining ? x.rows : (x.capacity + 1023) / 1024;
  const int id = !joining ? blockIdx.x - joins : W == 4 ? blockIdx.x : blockIdx.x * JOIN_WAVES + wave;
  if (joining && W == 1 && id >= x.batch * x.n_kv * x.rows) return;
  const int seg = id / per_head, item = id - seg * per_head;
  const int b = seg / x.n_kv, kvh = seg - b * x.n_kv;
  const int mine = first_lens(x, lane);
  const SeqWalk pw = prefix_walk(x);
  const int pre = pw.places() * x.n_kv * x.p_row_tiles;                // row tiles of rows that are not the workers': 0
  const int heads = x.n_kv * x.row_tiles;
  int all, before;
  count_places(x, b, mine, lane, all, before);
  const int share = worker_share(pre + all * heads, x.workers);
  const SeqWalk w = walk_of(x, b, mine);
  auto own_pieces = [&](int row) {
    const int rt = row / tile_rows;
    PieceList l;
    l.t0 = pre + before * heads + (kvh * x.row_tiles + rt) * w.places() + SEGMENT_COST;
    l.p = segment_pieces(l.t0, l.t0 + w.tiles, share);
    l.share = share; l.segment = x.n_kv * x.p_row_tiles + seg * x.row_tiles + rt;
    l.base = row - rt * tile_rows; l.slot_rows = x.slot_rows; l.workers = x.workers;
    return l;
  };

  if (!joining) {
    // weights of 1024 slots, four of a tile a thread (slots and tiles are aligned alike); up to 16 rows
    if (item * 1024 >= w.len) return;
    __shared__ float2 stat[16];
    const PieceList l = own_pieces(0);
    const bool whole = w.tiles > 0 && l.p.first == l.p.last;
    for (int row = wave; row < x.rows; row += JOIN_WAVES) {
      float m = -INFINITY, sum = 0.f;
      const int n = l.count();
      for (int i0 = 0; i0 < n; i0 += 64) {
        float2 ml = float2{-INFINITY, 0.f};
        if (i0 + lane < n) ml = whole ? x.stat[(int64_t)seg * x.rows + row] : x.piece_ml[l.at(i0 + lane) + row];
        float mx = ml.x;
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
        mx = fmaxf(mx, m);
        sum = m == -INFINITY && sum == 0.f ? 0.f : sum * fast_exp2(m - mx);
        float f = ml.x == -INFINITY && ml.y == 0.f ? 0.f : ml.y * fast_exp2(ml.x - mx);
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) f += __shfl_xor(f, d);
        sum += f;
        m = mx;
      }
      if (lane == 0) stat[row] = float2{m, sum > 0.f || sum != sum ? 1.0f / sum : 0.f};
    }
    __syncthreads();
    const int slot = item * 1024 + 4 * threadIdx.x;
    if (slot >= w.len) return;
    const int tau = w.tile_of(slot);
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    if (tau >= 0) {
      const float *s = x.logits + ((int64_t)seg * x.max_tiles + tau) * (x.rows * CACHE_TILE) + (slot - w.base(tau));
#pragma unroll 4
      for (int r = 0; r < x.rows; ++r) {
        const f32x4 v = *reinterpret_cast<const f32x4 *>(s + r * CACHE_TILE);
        const float2 ml = stat[r];
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += v[i] == -INFINITY ? 0.f : fast_exp2(v[i] - ml.x) * ml.y;
      }
    }
    float *to = x.weight + b * x.w_sb + kvh * x.w_sh + slot;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (slot + i < w.len) to[i] = x.add_weights ? to[i] + sum[i] : sum[i];
    return;
  }

  const int row = item, t = row / x.group;
  const bool token = w.i0 + t >= 0;
  const bool workers = !SHARED || !x.own_sh.on;
  PieceList own = {};
  if (workers) {
    own = own_pieces(row);
    if (x.direct && w.tiles > 0 && own.p.first == own.p.last) return;  // written by the worker itself
  }
  // The row's pieces in one list: of its own cache, then of the prefix, either the workers' or parts that several
  // waves took together.
  const SharedPart &osh = x.own_sh, &psh = x.p_sh;
  const int prow = b * x.rows + row;
  int64_t own0 = 0, pre0 = 0;
  int n_own = 0, n_psh = 0, n = 0;
  PieceList pre_pieces = own;
  if (token) {
    if (workers) {
      n_own = w.tiles > 0 ? own.count() : 0;
    } else {
      const int rt = row / osh.tile_rows, r0 = rt * osh.tile_rows, r1 = min(r0 + osh.tile_rows, x.rows) - 1;
      n_own = part_count(rows_walk(r0, r1, x.group, w.len, x.capacity, x.n_new, x.n_init, x.n_local).tiles, osh.splits);
      own0 = ((int64_t)seg * osh.row_tiles + rt) * osh.splits * osh.tile_rows + (row - r0);
    }
    if (SHARED && psh.on) {
      const int rt = prow / psh.tile_rows, len = pw.len + (psh.tile_rows == 256 ? 0 : SHARED_TILE - 1);
      n_psh = part_count(len / SHARED_TILE, psh.splits);
      pre0 = ((int64_t)kvh * psh.row_tiles + rt) * psh.splits * psh.tile_rows + (prow - rt * psh.tile_rows);
    }
    n = n_own + n_psh;
    if (x.p_row_tiles > 0 && pw.tiles > 0) {
      const int prt = prow / tile_rows;
      pre_pieces.t0 = (kvh * x.p_row_tiles + prt) * pw.places() + SEGMENT_COST;
      pre_pieces.p = segment_pieces(pre_pieces.t0, pre_pieces.t0 + pw.tiles, share);
      pre_pieces.segment = kvh * x.p_row_tiles + prt;
      pre_pieces.base = prow - prt * tile_rows;
      pre_pieces.share = share; pre_pieces.slot_rows = x.slot_rows; pre_pieces.workers = x.workers;
      n += pre_pieces.count();
    }
  }
  float m = -INFINITY, l = 0.f;
  f32x2 o = {0.f, 0.f};
  for (int i0 = W == 4 ? wave : 0; i0 < n; i0 += W * JOIN_AHEAD) {
    float2 ml[JOIN_AHEAD];
    f32x2 po[JOIN_AHEAD];
#pragma unroll
    for (int j = 0; j < JOIN_AHEAD; ++j) {
      const int i = min(i0 + W * j, n - 1);
      const bool mine = i < n_own, shared = SHARED && (mine ? osh.on : i < n_own + n_psh);
      const SharedPart &sh = mine ? osh : psh;
      const int64_t at = mine ? (shared ? own0 + (int64_t)i * sh.tile_rows : own.at(i))
                              : shared ? pre0 + (int64_t)(i - n_own) * sh.tile_rows : pre_pieces.at(i - n_own - n_psh);
      ml[j] = (shared ? sh.ml : x.piece_ml)[at];
      po[j] = *reinterpret_cast<const f32x2 *>((shared ? sh.o : x.piece_o) + at * D + 2 * lane);
    }
    float mx = m;
#pragma unroll
    for (int j = 0; j < JOIN_AHEAD; ++j) {
      if (i0 + W * j >= n) ml[j] = float2{-INFINITY, 0.f};
      mx = fmaxf(mx, ml[j].x);
    }
    const float f = m == -INFINITY && l == 0.f ? 0.f : fast_exp2(m - mx);
    m = mx;
    l *= f;
    o *= f;
#pragma unroll
    for (int j = 0; j < JOIN_AHEAD; ++j) {
      // a piece without a visible key (reference and sum as at its start) counts for nothing
      const bool none = ml[j].x == -INFINITY && ml[j].y == 0.f;
      const float g = none ? 0.f : fast_exp2(ml[j].x - m);
      l += none ? 0.f : ml[j].y * g;
      o[0] += none ? 0.f : po[j][0] * g;
      o[1] += none ? 0.f : po[j][1] * g;
    }
  }
  if (W == 4) {
    __shared__ float sm[JOIN_WAVES], sl[JOIN_WAVES];
    __shared__ f32x2 so[JOIN_WAVES][64];
    if (lane == 0) { sm[wave] = m; sl[wave] = l; }
    so[wave][lane] = o;
    __syncthreads();
    if (wave != 0) return;
    m = -INFINITY; l = 0.f;
    o = f32x2{0.f, 0.f};
#pragma unroll
    for (int i = 0; i < JOIN_WAVES; ++i) m = fmaxf(m, sm[i]);
#pragma unroll
    for (int i = 0; i < JOIN_WAVES; ++i) {
      if (sm[i] == -INFINITY && sl[i] == 0.f) continue;
      const float f = fast_exp2(sm[i] - m);
      l += sl[i] * f;
      o[0] += so[i][lane][0] * f;
      o[1] += so[i][lane][1] * f;
    }
  }
  const float inv = l > 0.f || l != l ? 1.0f / l : 0.f;
  const f32x2 r = {o[0] * inv, o[1] * inv};
  bf16_t *to = x.o + b * x.o_sb + (int64_t)(kvh * x.group + row - t * x.group) * x.o_sh + t * x.o_st;
  *reinterpret_cast<unsigned *>(to + 2 * lane) = __builtin_bit_cast(unsigned, __builtin_convertvector(r, bf16x2));
  if (x.stat && lane == 0) x.stat[(int64_t)seg * x.rows + row] = float2{m, l};
}

// Weights of more than 16 rows, whose logits would be more bytes than the keys: they are computed anew.  A wave takes
// 16 KT keys (K as A operands, in registers) and all rows, 16 at a time; per row block 4 KT MFMAs and 4 KT exponentials a
// lane.  The four waves of a workgroup share the rows: each brings one of four blocks into LDS, as operands, while
// the four before are used.  (Every wave with loads of its own: 256 rows, 4 heads of 40K tokens, 35 us, half of it
// for the loads.)
// KT = 2 where that gives 512 workgroups, two per CU, 1 otherwise, when the time is a wave's latency: the call with 256 rows,
// 4 heads of 40K, 74 and 82 us (KT = 4: 76), the kernel with 464 rows, 8 heads of 511 tokens, 17 and 16 (28).
template <int KT>
__global__ __launch_bounds__(256, 3) void cache_column_kernel(CacheCall x) {
  __shared__ bf16x8 rows_q[2][4][4][64];                        // [buffer][row block][k step][lane]
  __shared__ float rows_m[2][64];
  const int kvh = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4, kb = blockIdx.x * (64 * KT) + wave * (16 * KT);
  const int len = uni(min(max(x.lens[b], 0), x.capacity)), i0 = len - x.n_new;
  if ((int)blockIdx.x * (64 * KT) >= len) return;
  const int64_t head = (int64_t)b * x.n_kv + kvh;
  // every row sees every key / no row sees a key
  const bool whole = kb + 16 * KT - 1 <= i0 && (kb + 16 * KT - 1 < x.n_init || len - 1 - kb < x.n_local);
  const bool hidden = kb >= len || (kb >= x.n_init && i0 - (kb + 16 * KT - 1) >= x.n_local);
  bf16x8 k[KT][4];                                               // [16 keys][k step]
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    const bf16_t *row = x.k + b * x.k_sb + kvh * x.k_sh + (int64_t)min(kb + 16 * kt + n, len - 1) * x.k_st + 8 * g;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) k[kt][ks] = *reinterpret_cast<const bf16x8 *>(row + 32 * ks);
  }
  bf16x8 q[4];                                                  // this wave's block of the next four
  float m;
  auto load = [&](int r0) {
    const int at = r0 + 16 * wave + n, row = min(at, x.rows - 1), t = row / x.group;
    const bf16_t *from = x.q + b * x.q_sb + (int64_t)(kvh * x.group + row - t * x.group) * x.q_sh + t * x.q_st + 8 * g;
    const float2 ml = x.stat[head * x.rows + row];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) q[ks] = *reinterpret_cast<const bf16x8 *>(from + 32 * ks);
    // p = 2^(c s - m) / l = 2^(c s - (m + log2 l)); a row without a key, or behind the last: 2^-inf
    m = at >= x.rows || (ml.x == -INFINITY && ml.y == 0.f) ? INFINITY : ml.x + __builtin_amdgcn_logf(ml.y);
  };
  auto store = [&](int buf) {
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) rows_q[buf][wave][ks][lane] = q[ks];
    if (g == 0) rows_m[buf][16 * wave + n] = m;
  };
  float sum[4 * KT];
#pragma unroll
  for (int i = 0; i < 4 * KT; ++i) sum[i] = 0.f;
  load(0);
  store(0);
  __syncthreads();
  for (int r0 = 0, buf = 0; r0 < x.rows; r0 += 64, buf ^= 1) {
    const bool more = r0 + 64 < x.rows;
    if (more) load(r0 + 64);
    for (int blk = 0; blk < 4 && r0 + 16 * blk < x.rows && !hidden; ++blk) {
      const float ref = rows_m[buf][16 * blk + n];
      f32x4 s[KT];
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        const bf16x8 qf = rows_q[buf][blk][ks][lane];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
          const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
          s[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[kt][ks], qf, ks == 0 ? zero : s[kt], 0, 0, 0);
        }
      }
      if (whole) {
#pragma unroll
        for (int i = 0; i < 4 * KT; ++i) sum[i] += fast_exp2(fmaf(s[i >> 2][i & 3], x.c_log2, -ref));
        continue;
      }
      const int t = min(r0 + 16 * blk + n, x.rows - 1) / x.group;
#pragma unroll
      for (int i = 0; i < 4 * KT; ++i) {
        const bool sees = cache_visible(kb + 16 * (i >> 2) + 4 * g + (i & 3), i0 + t, x.n_init, x.n_local);
        const float p = fast_exp2(fmaf(s[i >> 2][i & 3], x.c_log2, -ref));
        sum[i] += sees ? p : 0.f;
      }
    }
    if (more) store(buf ^ 1);                                   // last read a barrier ago
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4 * KT; ++i)
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) sum[i] += __shfl_xor(sum[i], d);
  if (n != 0) return;
  float *to = x.weight + b * x.w_sb + kvh * x.w_sh;
#pragma unroll
  for (int i = 0; i < 4 * KT; ++i) {
    const int key = kb + 16 * (i >> 2) + 4 * g + (i & 3);
    if (key < len) to[key] = x.add_weights ? to[key] + sum[i] : sum[i];
  }
}

// ---- eviction ---------------------------------------------------------------------------------------------
// Order of the weights as unsigned numbers: NaN lowest, -0 and 0 equal.  0 is no weight's.
__device__ inline unsigned weight_key(float v) {
  if (v != v) return 1u;
  const unsigned u = v == 0.f ? 0u : __builtin_bit_cast(unsigned, v);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int SELECT_THREADS = 1024, SELECT_WAVES = SELECT_THREADS / 64;
constexpr int SELECT_BINS = 2048, SELECT_COPIES = 4, SELECT_AHEAD = 8;   // AHEAD: loads in flight a lane
// The kept weight of rank `want` is found digit by digit: 11, 11 and 10 bits from the most significant one.
__device__ constexpr int select_shift(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
__device__ constexpr int select_bins(int pass) { return pass == 2 ? 1024 : 2048; }
__device__ constexpr unsigned select_mask(int pass) { return pass == 0 ? 0u : ~0u << select_shift(pass - 1); }

// Sum of v over the lower threads of the workgroup, and over all of them.
__device__ inline int block_scan(int v, int *part, int &all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int incl = wave_scan(v, lane);
  __syncthreads();
  if (lane == 63) part[wave] = incl;
  __syncthreads();
  int before = 0;
  all = 0;
#pragma unroll
  for (int i = 0; i < SELECT_WAVES; ++i) {
    const int p = part[i];
    if (i < wave) before += p;
    all += p;
  }
  return before + incl - v;
}

// One sequence and K/V head.
struct SelectRow {
  const float *w;
  int len, first, last;          // tokens; slots first .. last - 1 are chosen by weight
  int want;                      // ... so many of them
  __device__ inline SelectRow(const EvictCall &x, int row) {
    const int b = row / x.n_kv, kvh = row - b * x.n_kv;
    w = x.weight + b * x.w_sb + kvh * x.w_sh;
    len = min(max(x.lens[b], 0), x.capacity);
    first = x.n_init; last = len - x.n_recent;
    want = x.keep - x.n_init - x.n_recent;
  }
};

struct SelectLds {
  int hist[SELECT_COPIES][SELECT_BINS];
  int part[SELECT_WAVES], pick[3];
};

// The keys of the slots from .. to - 1 (at most 32768) in registers, loaded once: a wave takes consecutive ones, so
// that it can also number them.
struct SelectKeys {
  static constexpr int BATCHES = 32768 / SELECT_THREADS / SELECT_AHEAD;
  unsigned k[BATCHES][SELECT_AHEAD];
  int w0, w1;                      // this wave's slots; 0: not to be chosen by weight
  __device__ inline int slot(int t, int j, int lane) const { return w0 + 64 * (t * SELECT_AHEAD + j) + lane; }
  __device__ inline bool batch(int t) const { return w0 + 64 * SELECT_AHEAD * t < w1; }
  __device__ inline void load(const SelectRow &r, int from, int to) {
    const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6);
    const int per = (to - from + SELECT_THREADS - 1) / SELECT_THREADS * 64;
    w0 = from + wave * per;
    w1 = min(w0 + per, min(to, r.last));
#pragma unroll
    for (int t = 0; t < BATCHES; ++t) {
      if (!batch(t)) break;
      float v[SELECT_AHEAD];
#pragma unroll
      for (int j = 0; j < SELECT_AHEAD; ++j) v[j] = r.w[min(slot(t, j, lane), w1 - 1)];
#pragma unroll
      for (int j = 0; j < SELECT_AHEAD; ++j) {
        const int i = slot(t, j, lane);
        k[t][j] = i >= r.first && i < w1 ? weight_key(v[j]) : 0u;
      }
    }
  }
};

// Histogram of the pass's digit over the keys whose higher digits are those of `prefix`.  Lanes add into four
// copies: weights cluster, and lanes that meet in a bin go one after the other.
template <int PASS>
__device__ inline void select_count(const SelectKeys &keys, unsigned prefix, SelectLds &s) {
  const int tid = threadIdx.x;
  for (int i = tid; i < SELECT_COPIES * SELECT_BINS; i += SELECT_THREADS) (&s.hist[0][0])[i] = 0;
  __syncthreads();
#pragma unroll
  for (int t = 0; t < SelectKeys::BATCHES; ++t) {
    if (!keys.batch(t)) break;
#pragma unroll
    for (int j = 0; j < SELECT_AHEAD; ++j) {
      const unsigned k = keys.k[t][j];
      if (k != 0u && (k & select_mask(PASS)) == prefix)
        atomicAdd(&s.hist[tid & (SELECT_COPIES - 1)][(k >> select_shift(PASS)) & (select_bins(PASS) - 1)], 1);
    }
  }
  __syncthreads();
}

// The digit of rank `want` from this thread's two bins (2047 - 2 tid and the one below: descending), and the
// number of slots above it: in all, and in the chunks before this one (n_before).  Lowers `want` to the rank
// among the slots with that digit.
__device__ inline unsigned select_pick(const int (&n)[2], const int (&n_before)[2], int bins, int &want, int &gt_before,
                                       int &eq_before, SelectLds &s) {
  const int hi = bins - 1 - 2 * (int)threadIdx.x;
  int all;
  const int above = block_scan(n[0] + n[1], s.part, all);
  if (above < want && want <= above + n[0] + n[1]) {
    const int lower = above + n[0] < want;
    s.pick[0] = hi - lower;
    s.pick[1] = above + (lower ? n[0] : 0);
    s.pick[2] = n_before[lower];
  }
  __syncthreads();
  const int d = s.pick[0];
  eq_before = s.pick[2];
  want -= s.pick[1];
  block_scan((hi > d ? n_before[0] : 0) + (hi - 1 > d ? n_before[1] : 0), s.part, gt_before);
  return (unsigned)d;
}

// Writes the kept slots among from .. to - 1 behind the `gt` larger and `eq` equal ones of lower slots; of the equal
// ones the first `want` stay.
__device__ inline void select_emit(const SelectRow &r, const SelectKeys &keys, int from, int to, unsigned key, int want, int gt,
                                   int eq, int32_t *kept, int keep, SelectLds &s) {
  const int tid = threadIdx.x, lane = tid & 63;
  auto rank = [](unsigned long long mask, int base) {              // base + set bits of the lower lanes
    return (int)__builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, base));
  };
  int ng = 0, ne = 0;
#pragma unroll
  for (int t = 0; t < SelectKeys::BATCHES; ++t) {
    if (!keys.batch(t)) break;
#pragma unroll
    for (int j = 0; j < SELECT_AHEAD; ++j) {
      ng += keys.k[t][j] > key;
      ne += keys.k[t][j] == key;
    }
  }
  int all;
  const int before_g = block_scan(ng, s.part, all), before_e = block_scan(ne, s.part, all);
  gt += uni(before_g);                                             // (the first lane's: those of the waves before)
  eq += uni(before_e);
#pragma unroll
  for (int t = 0; t < SelectKeys::BATCHES; ++t) {
    if (!keys.batch(t)) break;
#pragma unroll
    for (int j = 0; j < SELECT_AHEAD; ++j) {
      const unsigned k = keys.k[t][j];
      const unsigned long long g = __builtin_amdgcn_ballot_w64(k > key), e = __builtin_amdgcn_ballot_w64(k == key);
      if ((g | e) == 0) continue;
      const int gr = rank(g, gt), er = rank(e, eq);
      if (k > key || (k == key && er < want)) kept[r.first + gr + min(er, want)] = keys.slot(t, j, lane);
      gt += __popcll(g);
      eq += __popcll(e);
    }
  }
  // the first and the last slots stay whatever they weigh
  for (int i = from + tid; i < min(to, r.first); i += SELECT_THREADS) kept[i] = i;
  for (int i = max(from, r.last) + tid; i < min(to, r.len); i += SELECT_THREADS) kept[keep - (r.len - i)] = i;
}

__device__ inline void select_all(int len, int32_t *kept, int keep, int from, int step) {
  for (int i = from; i < keep; i += step) kept[i] = i < len ? i : -1;
}

// Short rows: one workgroup per sequence and K/V head, one launch.
__global__ __launch_bounds__(SELECT_THREADS) void cache_select_kernel(EvictCall x) {
  __shared__ SelectLds s;
  const int row = blockIdx.x, tid = threadIdx.x;
  const SelectRow r(x, row);
  int32_t *kept = x.kept + (int64_t)row * x.keep;
  if (tid == 0) x.counts[row] = min(r.len, x.keep);
  if (r.len <= x.keep) return select_all(r.len, kept, x.keep, tid, SELECT_THREADS);
  unsigned key = ~0u;                         // above every weight: nothing to choose
  int want = r.want, gt = 0, eq = 0;
  SelectKeys keys;
  keys.load(r, 0, r.len);
  if (want > 0) {
    key = 0;
    auto pass = [&](auto p) {
      constexpr int P = decltype(p)::value;
      select_count<P>(keys, key, s);
      int n[2] = {0, 0};
      const int none[2] = {0, 0}, hi = select_bins(P) - 1 - 2 * tid;
      if (hi > 0)
        for (int c = 0; c < SELECT_COPIES; ++c) {
          n[0] += s.hist[c][hi];
          n[1] += s.hist[c][hi - 1];
        }
      key |= select_pick(n, none, select_bins(P), want, gt, eq, s) << select_shift(P);
    };
    pass(std::integral_constant<int, 0>{});
    pass(std::integral_constant<int, 1>{});
    pass(std::integral_constant<int, 2>{});
  }
  select_emit(r, keys, 0, r.len, key, want, 0, 0, kept, x.keep, s);
}

// Long rows: a row in chunks, a workgroup each.  Pass p counts its digit per chunk; the workgroups of the next
// launch each add up the row's counts and pick the digit themselves (no atomics on memory, nothing to clear).
// The row and chunk of a workgroup.  Workgroups go round the eight XCDs: a row's are put on as few of them as keep
// all busy, since they read each other's counts, through the XCD's L2.
struct SelectPlace {
  int row, chunk;
  __device__ inline explicit SelectPlace(const EvictCall &x) {
    const int rows = x.batch * x.n_kv, id = blockIdx.x, xcd = id & 7, turn = id >> 3;
    if (rows % 8 == 0) {
      row = turn / x.chunks * 8 + xcd;
      chunk = turn % x.chunks;
    } else if (8 % rows == 0) {
      row = xcd % rows;
      chunk = turn * (8 / rows) + xcd / rows;
    } else {
      row = id / x.chunks;
      chunk = id % x.chunks;
    }
  }
};

template <int PASS>
__device__ inline void select_from_counts(const EvictCall &x, int row, int chunk, unsigned &key, int &want, int &gt, int &eq,
                                          SelectLds &s) {
  const int hi = select_bins(PASS) - 1 - 2 * (int)threadIdx.x;
  int n[2] = {0, 0}, before[2] = {0, 0};
  if (hi > 0) {
    const unsigned *h = x.hist + (((int64_t)PASS * x.batch * x.n_kv + row) * x.chunks * SELECT_BINS + (hi - 1)) / 2;
#pragma unroll 8
    for (int c = 0; c < x.chunks; ++c) {
      const unsigned two = h[(int64_t)c * (SELECT_BINS / 2)];
      n[0] += two >> 16;
      n[1] += two & 0xffff;
      before[0] += c < chunk ? two >> 16 : 0;
      before[1] += c < chunk ? two & 0xffff : 0;
    }
  }
  int above;
  key |= select_pick(n, before, select_bins(PASS), want, above, eq, s) << select_shift(PASS);
  gt += above;
}

template <int PASS>
__global__ __launch_bounds__(SELECT_THREADS) void cache_count_kernel(EvictCall x) {
  __shared__ SelectLds s;
  const SelectPlace at(x);
  const int row = at.row, chunk = at.chunk, tid = threadIdx.x;
  if (chunk >= x.chunks) return;
  const SelectRow r(x, row);
  const int from = chunk * x.chunk_slots, to = min(from + x.chunk_slots, r.len);
  if (r.len <= x.keep || r.want == 0) return;
  // digits so far, rank left, larger slots in the chunks before this one
  SelectState *state = x.state + (int64_t)row * x.chunks + chunk;
  SelectKeys keys;
  keys.load(r, from, max(to, from));
  unsigned key = 0;
  int want = r.want, gt = 0, eq = 0;
  if (PASS == 2) { key = state->key; want = state->want; gt = state->gt; }
  if (PASS > 0) {
    select_from_counts<PASS == 0 ? 0 : PASS - 1>(x, row, chunk, key, want, gt, eq, s);
    if (tid == 0) *state = SelectState{key, want, gt};
  }
  select_count<PASS>(keys, key, s);
  unsigned *h = x.hist + (((int64_t)PASS * x.batch * x.n_kv + row) * x.chunks + chunk) * (SELECT_BINS / 2);
  for (int i = tid; i < select_bins(PASS) / 2; i += SELECT_THREADS) {
    int a = 0, b = 0;
#pragma unroll
    for (int c = 0; c < SELECT_COPIES; ++c) { a += s.hist[c][2 * i]; b += s.hist[c][2 * i + 1]; }
    h[i] = (unsigned)b << 16 | (unsigned)a;
  }
}

__global__ __launch_bounds__(SELECT_THREADS) void cache_emit_kernel(EvictCall x) {
  __shared__ SelectLds s;
  const SelectPlace at(x);
  const int row = at.row, chunk = at.chunk, tid = threadIdx.x;
  if (chunk >= x.chunks) return;
  const SelectRow r(x, row);
  int32_t *kept = x.kept + (int64_t)row * x.keep;
  if (chunk == 0 && tid == 0) x.counts[row] = min(r.len, x.keep);
  if (r.len <= x.keep) return select_all(r.len, kept, x.keep, chunk * SELECT_THREADS + tid, x.chunks * SELECT_THREADS);
  const int from = chunk * x.chunk_slots, to = min(from + x.chunk_slots, r.len);
  if (from >= to) return;
  SelectKeys keys;
  keys.load(r, from, to);
  unsigned key = ~0u;
  int want = 0, gt = 0, eq = 0;
  if (r.want > 0) {
    const SelectState st = x.state[(int64_t)row * x.chunks + chunk];
    key = st.key; want = st.want; gt = st.gt;
    select_from_counts<2>(x, row, chunk, key, want, gt, eq, s);
  }
  select_emit(r, keys, from, to, key, want, gt, eq, kept, x.keep, s);
}

// Moves the kept rows to the slots 0, 1, ...  In place a workgroup owns one slice of 64 bytes of the rows of K or V of
// one sequence and K/V head (slices 0..3: K, 4..7: V), or its weights (the last slice), and walks them in ascending
// order, a chunk into registers, then out: the kept slots ascend, so the rows of a later chunk, which are loaded
// ahead, lie behind everything that this chunk overwrites.  Into another cache whole rows (slices K, V, weights) in
// any order.  (8 heads, 16K of 1M and 64K of 128K slots kept: 24 and 105 us into another cache, at 5.4 TB/s; in place 194
// and 756, a chain of 64 and 256 dependent chunks on 72 workgroups.)
constexpr int MOVE_ROWS = 4;                                     // a thread, at a time
template <bool IN_PLACE>
__global__ __launch_bounds__(256) void cache_move_kernel(EvictCall x) {
  constexpr int LANES = IN_PLACE ? 4 : 16, SLICES = 16 / LANES, CHUNK = MOVE_ROWS * 256 / LANES;
  const int slice = blockIdx.x, row = blockIdx.y, b = row / x.n_kv, kvh = row - b * x.n_kv, tid = threadIdx.x;
  const int n = x.counts[row], step = CHUNK * gridDim.z;
  const int32_t *kept = x.kept + (int64_t)row * x.keep;
  if (slice == 2 * SLICES) {
    const float *from = x.weight + b * x.w_sb + kvh * x.w_sh;
    float *to = x.to_weight + b * x.tw_sb + kvh * x.tw_sh;
    for (int i0 = blockIdx.z * 256; i0 < n; i0 += 256 * gridDim.z) {
      const int i = i0 + tid;
      float v = 0.f;
      if (i < n) v = from[kept[i]];
      asm volatile("" : "+v"(v));
      if (IN_PLACE) __syncthreads();                             // every weight of the chunk has been read
      if (i < n) to[i] = v;
    }
    if (IN_PLACE) __syncthreads();
    for (int i = n + (int)blockIdx.z * 256 + tid; i < x.to_capacity; i += 256 * gridDim.z) to[i] = 0.f;
    if (kvh == 0 && blockIdx.z == 0 && tid == 0) x.to_lens[b] = n;
    return;
  }
  const bool is_v = slice >= SLICES;
  const int64_t f_st = is_v ? x.v_st : x.k_st, t_st = is_v ? x.tv_st : x.tk_st;
  const int col = 8 * (LANES * (slice % SLICES) + tid % LANES), lane_row = tid / LANES;
  const bf16_t *from = (is_v ? x.v + b * x.v_sb + kvh * x.v_sh : x.k + b * x.k_sb + kvh * x.k_sh) + col;
  bf16_t *to = (is_v ? x.to_v + b * x.tv_sb + kvh * x.tv_sh : x.to_k + b * x.tk_sb + kvh * x.tk_sh) + col;
  auto load = [&](int i0, uint4 (&v)[MOVE_ROWS]) {
#pragma unroll
    for (int j = 0; j < MOVE_ROWS; ++j) {
      const int i = i0 + 256 / LANES * j + lane_row;
      if (i < n) v[j] = *reinterpret_cast<const uint4 *>(from + kept[i] * f_st);
    }
  };
  int i0 = blockIdx.z * CHUNK;
  if (IN_PLACE) {                                                // chunks in front of which nothing was evicted stay
    for (int same = 256; same == 256 && i0 < n; i0 += same * CHUNK) {
      const int at = i0 + tid * CHUNK, last = min(at + CHUNK, n) - 1;
      same = __syncthreads_count(at < n && kept[last] == last);
    }
  }
  uint4 v[MOVE_ROWS], next[MOVE_ROWS];
#pragma unroll
  for (int j = 0; j < MOVE_ROWS; ++j) v[j] = next[j] = uint4{0u, 0u, 0u, 0u};
  load(i0, v);
  for (; i0 < n; i0 += step) {
    load(i0 + step, next);
#pragma unroll
    for (int j = 0; j < MOVE_ROWS; ++j) asm volatile("" : "+v"(v[j].x), "+v"(v[j].y), "+v"(v[j].z), "+v"(v[j].w));
    if (IN_PLACE) __syncthreads();                               // every row of the chunk has been read
#pragma unroll
    for (int j = 0; j < MOVE_ROWS; ++j) {
      const int i = i0 + 256 / LANES * j + lane_row;
      if (i < n) *reinterpret_cast<uint4 *>(to + i * t_st) = v[j];
      v[j] = next[j];
    }
  }
}

// ---- host-side launches -------------------------------------------------------------------------------------
template <int NB>
static hipError_t launch_workers(const CacheCall &x, hipStream_t st) {
  const size_t lds = CACHE_WAVES * (CACHE_RING + (x.logits ? CACHE_LOGITS : 0));
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(cache_attn_kernel<NB>),
                                     hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(cache_attn_kernel<NB>, dim3(x.workers / CACHE_WAVES), dim3(64 * CACHE_WAVES), lds, st, x);
  return hipGetLastError();
}

constexpr int SHARED_ROUND = 256;                               // workgroups that fill a CU each
template <int NB, bool PREFIX, int HALVES>
static hipError_t launch_shared_as(const CacheCall &x, const SharedPart &sh, hipStream_t st) {
  const size_t lds = shared_ring(HALVES) + shared_waves(HALVES) * SHARED_ROOM;
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(cache_shared_kernel<NB, PREFIX, HALVES>),
                                     hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  const int groups = (PREFIX ? 1 : x.batch) * x.n_kv * sh.splits;
  hipLaunchKernelGGL((cache_shared_kernel<NB, PREFIX, HALVES>), dim3((groups + 7) / 8 * 8 * sh.row_tiles),
                     dim3(64 * shared_waves(HALVES)), lds, st, x);
  return hipGetLastError();
}
template <bool PREFIX>
static hipError_t launch_shared(const CacheCall &x, const SharedPart &sh, hipStream_t st) {
  if (!sh.on) return hipSuccess;
  if (sh.tile_rows == 256) return launch_cache_prefix(x, st);
  if (sh.tile_rows == 64) return launch_shared_as<1, PREFIX, 2>(x, sh, st);
  if (!PREFIX && (int64_t)x.batch * x.n_kv * sh.splits * sh.row_tiles > SHARED_ROUND) return launch_shared_as<2, false, 1>(x, sh, st);
  return launch_shared_as<2, PREFIX, 2>(x, sh, st);
}

hipError_t launch_cache_attn(const CacheCall &x, hipStream_t st) {
  hipError_t e = launch_shared<true>(x, x.p_sh, st);
  if (e == hipSuccess) e = launch_shared<false>(x, x.own_sh, st);
  if (e == hipSuccess && (x.row_tiles > 0 || x.p_row_tiles > 0)) e = x.row_blocks == 1 ? launch_workers<1>(x, st) : launch_workers<2>(x, st);
  if (e != hipSuccess) return e;
  const bool final = x.direct && x.own_sh.on && x.own_sh.splits == 1;  // nothing to join
  // Four waves per row while that is a round of the chip's waves or less (calls of 1024 rows, 32 pieces each, 74 us with
  // four and 76.5 with one, few pieces each 37.0 and 36.2; 2048 rows of few 115 and 110; 256 rows the same)
  const int rows = x.batch * x.n_kv * x.rows, weigh = x.logits ? x.batch * x.n_kv * ((x.capacity + 1023) / 1024) : 0;
  if (!final) {
    const bool four = rows <= 1024;
    const int joins = four ? rows : (rows + JOIN_WAVES - 1) / JOIN_WAVES, tile_rows = 16 * x.row_blocks;
    auto join = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3(joins + weigh), dim3(64 * JOIN_WAVES), 0, st, x, tile_rows, joins);
    };
    if (x.own_sh.on || x.p_sh.on) four ? join(cache_join_kernel<4, true>) : join(cache_join_kernel<1, true>);
    else four ? join(cache_join_kernel<4, false>) : join(cache_join_kernel<1, false>);
  }
  if ((e = hipGetLastError()) != hipSuccess || !x.weight || x.logits) return e;
  const int wide = (x.capacity + 127) / 128;
  if (wide * x.n_kv * x.batch >= 512) hipLaunchKernelGGL(cache_column_kernel<2>, dim3(wide, x.n_kv, x.batch), dim3(256), 0, st, x);
  else hipLaunchKernelGGL(cache_column_kernel<1>, dim3((x.capacity + 63) / 64, x.n_kv, x.batch), dim3(256), 0, st, x);
  return hipGetLastError();
}

hipError_t launch_cache_evict(const EvictCall &x, bool in_place, hipStream_t st) {
  const int rows = x.batch * x.n_kv;
  if (x.chunks == 0) {
    hipLaunchKernelGGL(cache_select_kernel, dim3(rows), dim3(SELECT_THREADS), 0, st, x);
  } else {
    const int groups = rows % 8 != 0 && 8 % rows == 0 ? (x.chunks * rows + 7) / 8 * 8 : x.chunks * rows;
    const dim3 grid(groups);
    hipLaunchKernelGGL(cache_count_kernel<0>, grid, dim3(SELECT_THREADS), 0, st, x);
    hipLaunchKernelGGL(cache_count_kernel<1>, grid, dim3(SELECT_THREADS), 0, st, x);
    hipLaunchKernelGGL(cache_count_kernel<2>, grid, dim3(SELECT_THREADS), 0, st, x);
    hipLaunchKernelGGL(cache_emit_kernel, grid, dim3(SELECT_THREADS), 0, st, x);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (in_place) {
    hipLaunchKernelGGL(cache_move_kernel<true>, dim3(9, rows), dim3(256), 0, st, x);
  } else {
    const int chunks = (x.keep + 16 * MOVE_ROWS - 1) / (16 * MOVE_ROWS);
    hipLaunchKernelGGL(cache_move_kernel<false>, dim3(3, rows, chunks < 1024 ? chunks : 1024), dim3(256), 0, st, x);
  }
  return hipGetLastError();
}

}  // namespace minf
