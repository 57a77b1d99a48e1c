// How the gradients of the attention over packed sequences (seq_grad.hip) are shared out.
//
// A unit is a run of 128 rows: of keys of one sequence and key head (the kernel of dK and dV, whose inner
// axis is the G query heads of that key head, one after the other, with the queries that see the run), or of
// packed query rows (token, head) of one sequence and head group (the kernel of dQ, whose inner axis is the
// keys that the run's last token sees).  A unit weighs its inner axis and `extra` for what starting and
// ending it costs.  As in seq_walk.h the units lie end to end on one line, workgroup l of P takes
// the stretch [l share, (l + 1) share) and finds it in closed form, a cut inside a unit goes to the next
// border of its inner tiles on both sides alike, and one that lies near a unit's start or end goes there.  A causal
// sequence's runs come from both ends in turn (8192 tokens, 16 heads over 4: dQ 341 -> 329 us, its units uncut).
//
// The order is (head, sequence, run): a head weighs the same as any other, so head h lies at h times the
// weight of one, and workgroup l meets the heads from floor(l share / that) on: the pairs (l, h) that occur
// form a staircase, along which l + h takes every value once (slots of the bias' gradient).
#pragma once

#include "la_internal.h"
#include "seq_walk.h"

namespace la {

constexpr int kGradRows = 128;

struct GradGeom {
  const int32_t* cu_q;     // [S + 1] first query token of every sequence
  const int32_t* cu_k;     // [S + 1] first key
  int S, Tq, Tk;
  int Hq, Hkv, G;
  int GH, GS, gh_magic;    // dQ: heads of a unit's rows, head groups of a key head, as in SeqGeom
  int TB;                  // tokens (dQ) or keys (dK, dV) of a unit
  int NH;                  // head groups (dQ) or key heads: times a sequence lies on the line
  int causal;
  uint32_t extra, cuts, whole, min_share;
};

struct GradIo {
  const uint16_t *q, *k, *v, *dout;
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head, do_tok, do_head;      // strides in elements
  uint16_t *out0, *out1;   // dQ; or dK and dV
  int64_t out0_tok, out0_head, out1_tok, out1_head;
  const float2* stat;      // [Hq][Tq]: log2-sum-exp2 of a row (+inf where it sees nothing), and delta
  float* part;             // [2 P][arrays][128][d]: sums of the piece that a stretch starts in (0) or ends in (1)
  int4* cut;               // [2 P]: the unit whose piece a slot holds, or w = 0
  float scale, scale_log2;
  const float* table;      // [Hq][bias_pitch]: the bias times log2 e by distance - (bias_lo - kBiasPad); first, whether any is -inf
  int bias_lo, bias_hi, bias_pitch;
  float* dist;             // [P + NH][bias_pitch]: the sums of dS of workgroup l and head h by distance, in l + h
  uint64_t* line;          // a head's weight, and a share
};

// One call of the gradients.
struct GradCall {
  bool rows, keys, has_bias;         // there are query rows; keys; a bias
  int rows_p, keys_p;      // workgroups
  GradGeom rows_g, keys_g;
  GradIo rows_io, keys_io;
  int Tq;
  const uint16_t* o;
  int64_t o_tok, o_head;
  const float *lse, *dlse;
  SeqBias bias;
  void* dweight;
};

namespace {

__device__ __forceinline__ int64_t ceil_div_i64(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Run j of a sequence weighs clamp(c0 + c1 j, 0, cap) times mult, and extra.
struct GradLine {
  int64_t c0, c1, cap;
  int64_t ja, jb;          // runs [ja, jb) weigh c0 + c1 j; those before and behind 0 or cap
  int nb;
  uint32_t mult;
};

// QT: query rows of an inner tile of the kernel of dK and dV; 0: the kernel of dQ.
template <int QT>
__device__ __forceinline__ GradLine grad_line(const GradGeom& g, const Seq& q) {
  GradLine w;
  const int64_t off = (int64_t)q.lk - q.lq;                  // token i sees the keys up to i + off
  if (QT == 0) {
    w.nb = (q.lq + g.TB - 1) / g.TB;
    w.mult = 1;
    w.cap = q.lk;
    w.c1 = g.causal ? g.TB : 0;
    w.c0 = g.causal ? off + g.TB : w.cap;
  } else {
    constexpr int T = QT == 0 ? 1 : QT;
    w.nb = (q.lk + g.TB - 1) / g.TB;
    w.mult = (uint32_t)g.G;
    w.cap = ((int64_t)q.lq + T - 1) / T * T;
    // key n is seen by the queries from n - off on; the first tile of run j starts at TB j - off rounded down
    const int64_t first = -off >= 0 ? -off / T * T : -(off + T - 1) / T * T;
    w.c1 = g.causal ? -g.TB : 0;
    w.c0 = g.causal ? w.cap - first : w.cap;
  }
  if (w.c1 > 0) {
    w.ja = w.c0 > 0 ? 0 : -w.c0 / w.c1 + 1;
    w.jb = w.c0 >= w.cap ? 0 : ceil_div_i64(w.cap - w.c0, w.c1);
  } else if (w.c1 < 0) {
    w.ja = w.c0 < w.cap ? 0 : (w.c0 - w.cap) / -w.c1 + 1;
    w.jb = w.c0 <= 0 ? 0 : ceil_div_i64(w.c0, -w.c1);
  } else {
    w.ja = w.jb = 0;
  }
  if (w.jb < w.ja) w.jb = w.ja;
  return w;
}

// What run j weighs beside extra, for one of mult heads.
__device__ __forceinline__ uint32_t grad_seen(const GradLine& w, int j) {
  const int64_t x = w.c0 + w.c1 * j;
  return (uint32_t)(x < 0 ? 0 : (x > w.cap ? w.cap : x));
}

// Weight of the runs before run b.
__device__ __forceinline__ uint64_t grad_before(const GradGeom& g, const GradLine& w, int b) {
  int64_t sum;
  if (w.c1 == 0) {
    sum = w.cap * b;
  } else {
    const int64_t a = w.ja < b ? w.ja : b, e = w.jb < b ? w.jb : b;
    sum = (e - a) * w.c0;
    if (e > a) sum += w.c1 * ((a + e - 1) * (e - a) / 2);
    sum += w.cap * (w.c1 > 0 ? b - e : a);
  }
  return (uint64_t)sum * w.mult + (uint64_t)b * g.extra;
}

// The j-th run of a sequence on the line, and the weight of those before it: the runs of a causal sequence come from
// both ends in turn (see seq_walk.h).
__device__ __forceinline__ int grad_run(const GradGeom& g, int nb, int j) {
  return g.causal ? ((j & 1) ? j >> 1 : nb - 1 - (j >> 1)) : j;
}
__device__ __forceinline__ uint64_t grad_line_before(const GradGeom& g, const GradLine& w, uint64_t all, int j) {
  if (!g.causal) return grad_before(g, w, j);
  const int m = j >> 1;                                     // m runs of either end
  uint64_t x = grad_before(g, w, m);
  if (m > 0) x += all - grad_before(g, w, w.nb - m);
  if (j & 1) x += (uint64_t)grad_seen(w, w.nb - 1 - m) * w.mult + g.extra;
  return x;
}

__device__ __forceinline__ Seq grad_seq(const GradGeom& g, int s) {
  Seq q;
  q.q0 = min(max(g.cu_q[s], 0), g.Tq);
  q.lq = min(max(g.cu_q[s + 1], q.q0), g.Tq) - q.q0;
  q.k0 = min(max(g.cu_k[s], 0), g.Tk);
  q.lk = min(max(g.cu_k[s + 1], q.k0), g.Tk) - q.k0;
  q.q0 = __builtin_amdgcn_readfirstlane(q.q0);
  q.lq = __builtin_amdgcn_readfirstlane(q.lq);
  q.k0 = __builtin_amdgcn_readfirstlane(q.k0);
  q.lk = __builtin_amdgcn_readfirstlane(q.lk);
  return q;
}

// A workgroup's place on the line; everything in it is uniform.
struct GradWalk {
  uint64_t pos, end;       // the stretch still to do
  uint64_t unit0;          // where the present unit starts
  uint64_t head;           // weight of a head
  uint32_t snap, small;    // as in Walk, but in units of up to 5/4 shares a border within half a share of an end goes there
  int h, s, j, b;          // head group, sequence, place of the run among the sequence's, run
  Seq q;
  GradLine line;
  __device__ __forceinline__ bool more() const { return pos < end; }
};

__device__ __forceinline__ uint32_t grad_near(const GradWalk& w, uint64_t weight) {
  return weight <= w.small ? w.small * 2 / 5 : w.snap;
}

// The part of the present unit that the stretch covers: inner tiles [ta, tb) of n, none if ta == tb.  A unit
// of nothing has one tile too, which is empty.
struct GradPiece {
  int64_t ta, tb, n;
};

// TS: what an inner tile weighs.
template <int TS>
__device__ __forceinline__ GradPiece grad_piece(const GradGeom& g, const GradWalk& w, uint64_t* unit_end) {
  const uint64_t seen = (uint64_t)grad_seen(w.line, w.b) * w.line.mult;
  *unit_end = w.unit0 + seen + g.extra;
  GradPiece p;
  p.n = seen == 0 ? 1 : (int64_t)((seen + TS - 1) / TS);
  const uint64_t xa = w.pos - w.unit0;
  p.ta = xa <= g.extra ? 0 : (int64_t)((xa - g.extra + TS - 1) / TS);
  p.tb = p.n;
  if (w.end < *unit_end) {
    const uint64_t xb = w.end - w.unit0;
    const uint32_t near = grad_near(w, seen + g.extra);
    if (xb <= near) p.tb = 0;                               // the unit is the next workgroup's
    else if (*unit_end - w.end > near) p.tb = xb <= g.extra ? 0 : (int64_t)((xb - g.extra + TS - 1) / TS);
  }
  if (p.tb < p.ta) p.tb = p.ta;
  return p;
}

// On to the next unit.
template <int QT>
__device__ __forceinline__ void grad_on(const GradGeom& g, GradWalk& w, uint64_t unit_end) {
  w.pos = w.unit0 = unit_end;
  if (w.pos >= w.end) return;
  if (++w.j < w.line.nb) {
    w.b = grad_run(g, w.line.nb, w.j);
    return;
  }
  w.j = 0;
  do {
    if (++w.s >= g.S) {
      w.s = 0;
      if (++w.h >= g.NH) {                                  // not reached while pos < end
        w.pos = w.end;
        return;
      }
    }
    w.q = grad_seq(g, w.s);
    w.line = grad_line<QT>(g, w.q);
  } while (w.line.nb == 0);
  w.b = grad_run(g, w.line.nb, 0);
}

// Start of the stretch of workgroup l of P; *share is what a workgroup takes.
template <int QT>
__device__ __forceinline__ GradWalk grad_start(const GradGeom& g, int l, int P, uint64_t* share_out) {
  const int lane = threadIdx.x & 63;
  const int C = (g.S + 63) / 64;
  uint64_t sum = 0;
  for (int i = 0; i < C; ++i) {
    const int s = lane * C + i;
    if (s < g.S) {
      Seq q;
      q.q0 = min(max(g.cu_q[s], 0), g.Tq);
      q.lq = min(max(g.cu_q[s + 1], q.q0), g.Tq) - q.q0;
      q.k0 = min(max(g.cu_k[s], 0), g.Tk);
      q.lk = min(max(g.cu_k[s + 1], q.k0), g.Tk) - q.k0;
      const GradLine w = grad_line<QT>(g, q);
      sum += grad_before(g, w, w.nb);
    }
  }
  const uint64_t incl = wave_incl_scan(sum);
  GradWalk w;
  w.head = read_lane_u64(incl, 63);
  const uint64_t total = w.head * (uint32_t)g.NH;
  uint64_t share = (total + (uint32_t)P - 1) / (uint32_t)P;
  if (share < g.min_share) share = g.min_share;
  *share_out = share;
  w.pos = first_lane_u64((uint64_t)(uint32_t)l * share);
  w.end = w.pos + share < total ? w.pos + share : total;
  w.snap = !g.cuts ? ~0u : (uint32_t)(share / 64 < g.extra ? share / 64 : g.extra);
  w.small = g.cuts && share < g.whole ? (uint32_t)share * 5 / 4 : 0;
  w.h = w.s = w.j = w.b = 0;
  w.unit0 = 0;
  w.q = Seq{0, 0, 0, 0};
  w.line = GradLine{0, 0, 0, 0, 0, 0, 0};
  if (w.pos >= w.end) return w;
  w.h = (int)(w.pos / w.head);
  const uint64_t in_head = w.pos - w.head * (uint32_t)w.h;
  // the lane whose sequences hold the place, then the sequence among them
  const uint64_t held = __ballot(incl - sum <= in_head && in_head < incl);
  const int L = __builtin_ctzll(held);
  uint64_t at = read_lane_u64(incl - sum, L);
  int s = __builtin_amdgcn_readfirstlane(L * C);
  w.q = grad_seq(g, s);
  w.line = grad_line<QT>(g, w.q);
  uint64_t ws = grad_before(g, w.line, w.line.nb);
  while (in_head >= at + ws && s + 1 < g.S) {
    at += ws;
    w.q = grad_seq(g, ++s);
    w.line = grad_line<QT>(g, w.q);
    ws = grad_before(g, w.line, w.line.nb);
  }
  w.s = s;
  const uint64_t rem = in_head - at;
  int lo = 0, n = w.line.nb;
  while (n > 1) {                                           // the run's place is in [lo, lo + n)
    const int step = (n + 63) / 64;
    const int64_t j = (int64_t)lo + (int64_t)lane * step;
    const bool below = j < lo + n && grad_line_before(g, w.line, ws, (int)j) <= rem;
    const int i = __popcll(__ballot(below)) - 1;            // lane 0 is always below
    lo += i * step;
    n = min(step, n - i * step);
  }
  w.j = __builtin_amdgcn_readfirstlane(lo);
  w.b = grad_run(g, w.line.nb, w.j);
  w.unit0 = first_lane_u64(w.head * (uint32_t)w.h + at + grad_line_before(g, w.line, ws, w.j));
  const uint64_t weight = (uint64_t)grad_seen(w.line, w.b) * w.line.mult + g.extra;
  const uint32_t near = grad_near(w, weight);
  const uint64_t unit_end = w.unit0 + weight;
  if (w.pos - w.unit0 <= near) w.pos = w.unit0;
  else if (unit_end - w.pos <= near) grad_on<QT>(g, w, unit_end);
  return w;
}

}  // namespace
}  // namespace la
