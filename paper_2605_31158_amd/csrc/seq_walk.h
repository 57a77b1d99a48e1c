// How the attention over packed sequences (seq_attn.hip, seq_token.hip) is shared out.
//
// A unit is a run of at most TB query tokens of one sequence with the GH query heads of one head
// group: R = TB GH packed rows (row r is token r / GH, head r % GH), which all read the same keys.
// A head group is the G query heads of a key head, or, where G > R, a part of at most R of them.
// A unit weighs the keys that its last token sees, and `extra` for what it costs to start and to end
// one (a row that sees nothing is written too).  The units, in the order (sequence, head group, run of
// tokens), are laid end to end on one line of weights, and workgroup l of P takes the stretch
// [l share, (l + 1) share): equal shares whatever the lengths are, with no plan in memory and no launch
// for one.  A stretch covers the end of one unit, whole units and the start of another; a place inside
// a unit, less the extra, is rounded up to tiles of 64 keys, on both sides of a cut alike, so every
// tile belongs to exactly one piece.  A cut costs a piece more, so a border no further than a 64th of a
// share (or `extra`) from a unit's start or end is moved there, again on both sides alike; with few keys
// to share, where a piece costs more to start than to work off, it is moved to the nearest one in units of
// up to two shares (256-row units: 48 prompts of 1 to 300 tokens 24.4 -> 19.9 us, 4 of 500 tokens 38 -> 27;
// in larger ones shares would differ by as much as themselves: 2164 queries over 3041 keys, 8 heads, 64 us
// with it, 54 without).  The runs of a
// causal sequence come from both ends in turn, the longest, the shortest, the second longest, ..:
// pairs weigh the same, and where they fill the shares evenly no unit is cut at all (8192 tokens, 4
// key heads: 512 units for 256 workgroups; in ascending order nearly every workgroup cut two, 34 MB of
// partials written and read).
//
// Where a unit starts on the line has a closed form (causal runs of a sequence weigh off + TB,
// off + 2 TB, ..), so a wave finds its first unit with one scan over the sequences and a 64-way
// search over the runs, in registers.
#pragma once

#include <math.h>

#include "la_internal.h"

namespace la {

struct SeqGeom {
  const int32_t* cu_q;     // [S + 1] first query token of every sequence
  const int32_t* ks;       // [S + 1] first key (packed keys), or [S] lengths (a cache)
  int S, Tq, Kcap;         // Kcap: packed keys, or the most keys of a sequence in the cache
  int lq_min, lq_max;      // sequences with other numbers of query tokens are left out
  int Hq, Hkv, G, GH, GS;  // query heads, key heads, Hq / Hkv, heads of a group, groups of a key head
  int gh_magic;            // r / GH of a packed row r < 256 is r gh_magic >> 16: ceil(2^16 / GH)
  int TB;                  // tokens of a unit
  int causal;
  uint32_t extra;          // weight of a unit beside its keys, >= 1
  uint32_t cuts;           // 0: no unit is cut, the workgroup whose share holds its end does all of it
  uint32_t whole;          // shares below this end where the nearest small unit does
  uint32_t min_share;      // more than two tiles, so that a share among a unit's keys is never empty
};

struct Seq {
  int q0, lq, k0, lk;
};

struct SeqIo {
  const uint16_t *q, *k, *v;
  uint16_t* o;
  float* lse;
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head, o_tok, o_head;   // strides in elements
  float* part_o;           // [2 P][R][d]: O of the piece that a stretch starts in (0) or ends in (1)
  float* part_m;           // [2 P][R]
  float* part_l;
  int4* cut;               // [2 P]: the unit whose piece a slot holds (unit_record), or w = 0
  float scale_log2;
};

// Distances that a tile of 64 x 32 pairs can have beyond the bias' first or last one while it still needs the table.
constexpr int kBiasPad = 96;
constexpr int kBiasMost = 513;                              // distances
constexpr int kBiasPitch = kBiasMost + 2 * kBiasPad;
constexpr int kBiasHeads = 4, kBiasRows = 128;              // of a unit of la_prompt_attn_bias
constexpr float kBiasWeight = 16384.f;                      // the largest finite weight

// A learned bias by relative position (la_rel_bias).
struct SeqBias {
  const int32_t* bucket;
  const void* weight;      // [buckets][Hq], fp32 or bf16
  int bf16, buckets, lo, hi;
};

namespace {

// The bias of bucket bucket[i] and head h in base 2.  Finite weights are held to 2^14 (a type's lowest value as a mask, or
// -1e9): a row that sees nothing but such keys has all of it in its logits and in its lse, and must still tell the logits
// apart and get its probabilities back from the lse, of which the gradients have one float.  Next to 2^14 that float's
// half step is worth 0.1 % of a probability, the logits' the same; next to 2^24 both are worth whole factors (row sums of
// P from 0.25 to 4).  As a mask 2^14 is enough for logits that lie up to 16000 apart.
__device__ __forceinline__ float bias_log2(const SeqBias& b, int i, int Hq, int h) {
  const int n = b.bucket[min(max(i, 0), b.hi - b.lo)];
  if (n < 0 || n >= b.buckets) return 0.f;
  const size_t at = (size_t)n * Hq + h;
  float w = b.bf16 ? __uint_as_float((uint32_t)((const uint16_t*)b.weight)[at] << 16) : ((const float*)b.weight)[at];
  if (fabsf(w) > kBiasWeight && w != -INFINITY) w = copysignf(kBiasWeight, w);
  return w * 1.4426950408889634f;
}

template <bool CACHE>
__device__ __forceinline__ Seq load_seq(const SeqGeom& g, int s) {
  Seq q;
  q.q0 = min(max(g.cu_q[s], 0), g.Tq);
  q.lq = min(max(g.cu_q[s + 1], q.q0), g.Tq) - q.q0;
  if (q.lq < g.lq_min || q.lq > g.lq_max) q.lq = 0;
  if (CACHE) {
    q.k0 = 0;
    q.lk = min(max(g.ks[s], 0), g.Kcap);
  } else {
    q.k0 = min(max(g.ks[s], 0), g.Kcap);
    q.lk = min(max(g.ks[s + 1], q.k0), g.Kcap) - q.k0;
  }
  return q;
}

// Weight of the runs before run b (b < the sequence's runs), for one head group.
__device__ __forceinline__ uint64_t weight_before(const SeqGeom& g, const Seq& q, int b) {
  const uint64_t extra = (uint64_t)b * g.extra;
  if (!g.causal) return extra + (uint64_t)b * (uint32_t)q.lk;
  const int off = q.lk - q.lq;                         // token i sees the keys up to i + off
  const int b0 = off < 0 ? min(b, -off / g.TB) : 0;    // runs whose last token sees nothing
  const int64_t n = b - b0;
  return extra + (uint64_t)(n * off + (int64_t)g.TB * (n * (b0 + 1 + (int64_t)b) / 2));
}

// Keys that the last token of run b sees.
__device__ __forceinline__ int run_keys(const SeqGeom& g, const Seq& q, int b) {
  if (!g.causal) return q.lk;
  return max(0, min(q.lk, q.lk - q.lq + (int)min((int64_t)q.lq, ((int64_t)b + 1) * g.TB)));
}

__device__ __forceinline__ int runs_of(const SeqGeom& g, const Seq& q) { return (q.lq + g.TB - 1) / g.TB; }

// Weight of all runs of a sequence, for one head group.
__device__ __forceinline__ uint64_t seq_weight(const SeqGeom& g, const Seq& q) {
  const int nb = runs_of(g, q);
  return nb == 0 ? 0 : weight_before(g, q, nb - 1) + (uint32_t)q.lk + g.extra;
}

// The j-th run of a sequence on the line, and the weight of those before it.
__device__ __forceinline__ int run_at(const SeqGeom& g, int nb, int j) {
  return g.causal ? ((j & 1) ? j >> 1 : nb - 1 - (j >> 1)) : j;
}
__device__ __forceinline__ uint64_t line_before(const SeqGeom& g, const Seq& q, int nb, uint64_t all, int j) {
  if (!g.causal) return weight_before(g, q, j);
  const int m = j >> 1;                                // m runs of either end
  uint64_t w = weight_before(g, q, m);
  if (m > 0) w += all - weight_before(g, q, nb - m);
  if (j & 1) w += (uint32_t)run_keys(g, q, nb - 1 - m) + g.extra;
  return w;
}

// A wave's place on the line; everything in it is uniform.
struct Walk {
  uint64_t pos, end;       // the stretch still to do
  uint64_t unit0;          // where the present unit starts
  uint32_t snap;           // borders this near a unit's start or end lie there,
  uint32_t small;          // and in units of at most this weight, those nearer than a quarter of it
  int s, kvh, part;        // sequence, key head, part of its group
  int j, b, nb;            // place of the run among the sequence's, run, runs
  Seq q;
  __device__ __forceinline__ bool more() const { return pos < end; }
};

__device__ __forceinline__ uint64_t first_lane_u64(uint64_t x) { return read_lane_u64(x, 0); }

template <bool CACHE>
__device__ __forceinline__ Seq load_seq_uniform(const SeqGeom& g, int s) {
  Seq q = load_seq<CACHE>(g, s);
  q.q0 = __builtin_amdgcn_readfirstlane(q.q0);
  q.lq = __builtin_amdgcn_readfirstlane(q.lq);
  q.k0 = __builtin_amdgcn_readfirstlane(q.k0);
  q.lk = __builtin_amdgcn_readfirstlane(q.lk);
  return q;
}

// How near a border has to lie to an end of a unit of this weight to be moved there.
__device__ __forceinline__ uint32_t near_ends(const Walk& w, uint32_t weight) {
  return weight <= w.small ? w.small / 4 : w.snap;
}

// The part of the present unit that the stretch covers: tiles [ta, tb) of n, none if ta == tb.
struct Piece {
  int keys;                // keys that the unit's last token sees
  int ta, tb, n;
};

__device__ __forceinline__ Piece walk_piece(const SeqGeom& g, const Walk& w, uint64_t* unit_end) {
  Piece p;
  p.keys = run_keys(g, w.q, w.b);
  *unit_end = w.unit0 + (uint32_t)p.keys + g.extra;
  p.n = p.keys == 0 ? 1 : (int)(((uint32_t)p.keys + 63u) >> 6);
  const uint32_t xa = (uint32_t)(w.pos - w.unit0);
  p.ta = xa <= g.extra ? 0 : (int)((xa - g.extra + 63u) >> 6);
  p.tb = p.n;
  if (w.end < *unit_end) {
    const uint32_t xb = (uint32_t)(w.end - w.unit0), near = near_ends(w, (uint32_t)p.keys + g.extra);
    if (xb <= near) p.tb = 0;                           // the unit is the next workgroup's
    else if (*unit_end - w.end > near) p.tb = xb <= g.extra ? 0 : (int)((xb - g.extra + 63u) >> 6);
  }
  p.ta = __builtin_amdgcn_readfirstlane(p.ta);
  p.tb = __builtin_amdgcn_readfirstlane(max(p.ta, p.tb));
  return p;
}

// On to the next unit.
template <bool CACHE>
__device__ __forceinline__ void walk_on(const SeqGeom& g, Walk& w, uint64_t unit_end) {
  w.pos = w.unit0 = unit_end;
  if (w.pos >= w.end) return;
  if (++w.j >= w.nb) {
    w.j = 0;
    if (++w.part >= g.GS) {
      w.part = 0;
      if (++w.kvh >= g.Hkv) {
        w.kvh = 0;
        do {
          if (++w.s >= g.S) {                           // not reached while pos < end
            w.pos = w.end;
            return;
          }
          w.q = load_seq_uniform<CACHE>(g, w.s);
        } while (w.q.lq == 0);
        w.nb = runs_of(g, w.q);
      }
    }
  }
  w.b = run_at(g, w.nb, w.j);
}

// Start of the stretch of workgroup l of P.
template <bool CACHE>
__device__ __forceinline__ Walk start_walk(const SeqGeom& g, int l, int P) {
  const int lane = threadIdx.x & 63;
  const int NH = g.Hkv * g.GS;
  const int C = (g.S + 63) / 64;
  uint64_t sum = 0;
  Seq mine{0, 0, 0, 0};
  for (int i = 0; i < C; ++i) {
    const int s = lane * C + i;
    if (s < g.S) {
      mine = load_seq<CACHE>(g, s);
      sum += seq_weight(g, mine);
    }
  }
  sum *= (uint32_t)NH;
  const uint64_t incl = wave_incl_scan(sum);
  const uint64_t total = read_lane_u64(incl, 63);
  uint64_t share = (total + (uint32_t)P - 1) / (uint32_t)P;
  if (share < g.min_share) share = g.min_share;
  Walk w;
  w.pos = first_lane_u64((uint64_t)(uint32_t)l * share);
  w.end = w.pos + share < total ? w.pos + share : total;
  w.snap = !g.cuts ? ~0u : (uint32_t)(share / 64 < g.extra ? share / 64 : g.extra);
  w.small = g.cuts && share < g.whole ? 2 * (uint32_t)share : 0;
  w.s = w.kvh = w.part = w.j = w.b = w.nb = 0;
  w.unit0 = 0;
  w.q = Seq{0, 0, 0, 0};
  if (w.pos >= w.end) return w;
  // the lane whose sequences hold pos, then the sequence among them
  const uint64_t held = __ballot(incl - sum <= w.pos && w.pos < incl);
  const int L = __builtin_ctzll(held);
  uint64_t at = read_lane_u64(incl - sum, L);
  int s = __builtin_amdgcn_readfirstlane(L * C);
  Seq q;
  if (C == 1) {
    q.q0 = __builtin_amdgcn_readlane(mine.q0, L);
    q.lq = __builtin_amdgcn_readlane(mine.lq, L);
    q.k0 = __builtin_amdgcn_readlane(mine.k0, L);
    q.lk = __builtin_amdgcn_readlane(mine.lk, L);
  } else {
    q = load_seq_uniform<CACHE>(g, s);
  }
  uint64_t ws = seq_weight(g, q);
  while (w.pos >= at + ws * (uint32_t)NH && s + 1 < g.S) {
    at += ws * (uint32_t)NH;
    q = load_seq_uniform<CACHE>(g, ++s);
    ws = seq_weight(g, q);
  }
  const int hg = (int)((w.pos - at) / ws);
  at += ws * (uint32_t)hg;
  const uint64_t rem = w.pos - at;
  const int nb = runs_of(g, q);
  int lo = 0, n = nb;
  while (n > 1) {                                       // the run's place is in [lo, lo + n)
    const int step = (n + 63) / 64;
    const int64_t j = (int64_t)lo + (int64_t)lane * step;
    const bool below = j < lo + n && line_before(g, q, nb, ws, (int)j) <= rem;
    const int i = __popcll(__ballot(below)) - 1;        // lane 0 is always below
    lo += i * step;
    n = min(step, n - i * step);
  }
  w.s = __builtin_amdgcn_readfirstlane(s);
  w.kvh = __builtin_amdgcn_readfirstlane(hg / g.GS);
  w.part = __builtin_amdgcn_readfirstlane(hg % g.GS);
  w.j = __builtin_amdgcn_readfirstlane(lo);
  w.b = run_at(g, nb, w.j);
  w.nb = nb;
  w.q = q;
  w.unit0 = first_lane_u64(at + line_before(g, q, nb, ws, w.j));
  const uint32_t weight = (uint32_t)run_keys(g, q, w.b) + g.extra, near = near_ends(w, weight);
  const uint64_t unit_end = w.unit0 + weight;
  if (w.pos - w.unit0 <= near) w.pos = w.unit0;
  else if (unit_end - w.pos <= near) walk_on<CACHE>(g, w, unit_end);
  return w;
}

// Packed row r of a unit: its token (of the sequence) and query head, or ok == false.
struct Row {
  int token, head;
  bool ok;
};
__device__ __forceinline__ int unit_head0(const SeqGeom& g, const Walk& w) { return w.kvh * g.G + w.part * g.GH; }
__device__ __forceinline__ int unit_heads(const SeqGeom& g, const Walk& w) { return min(g.GH, g.G - w.part * g.GH); }
__device__ __forceinline__ Row unit_row(const SeqGeom& g, const Walk& w, int r) {
  const int t = (int)(((uint32_t)r * (uint32_t)g.gh_magic) >> 16), j = r - t * g.GH;
  Row x;
  x.token = w.b * g.TB + t;
  x.head = unit_head0(g, w) + j;
  x.ok = t < min(g.TB, w.q.lq - w.b * g.TB) && j < unit_heads(g, w);
  return x;
}

// What a merge has to know of a unit: its first row of q and o, tokens, first head, heads.  The first and
// the third name the unit.
__device__ __forceinline__ int4 unit_record(const SeqGeom& g, const Walk& w) {
  return int4{w.q.q0 + w.b * g.TB, min(g.TB, w.q.lq - w.b * g.TB), unit_head0(g, w), unit_heads(g, w)};
}

// Keys that token t of the sequence sees.
__device__ __forceinline__ int token_keys(const SeqGeom& g, const Seq& q, int t) {
  return g.causal ? max(0, min(q.lk, q.lk - q.lq + t + 1)) : q.lk;
}

}  // namespace
}  // namespace la
