// Host side of the entry points over packed sequences (include/la.h): validation, the shapes that
// the kernels take, workspaces and launches.  Nothing here allocates device memory.
#include <math.h>

#include "grad_walk.h"
#include "kv4.h"
#include "la_internal.h"
#include "seq_walk.h"

using namespace la;

namespace {

bool misaligned(const void* p) { return ((uintptr_t)p & 15u) != 0; }

bool bad_strides(int64_t token, int64_t head, int d, bool written) {
  return token < d || token >= (int64_t(1) << 24) || head < (written ? 1 : 0) || ((token | head) & 7);
}

// The most sequences, rows and cached tokens: 64 times a tile's number, and what is read ahead of a tile (8 of
// them), stay below 2^31.
constexpr int kMaxTokens = 0x7ffff000;
// The most rows of la_kv4_append and la_kv4_read: 256 threads for 16 or 32 rows, and a grid has at most
// 2^32 - 1 threads along an axis.
constexpr int kMaxCacheRows = (1 << 28) - 32;

// Fields that every call uses.  Hq is 0 where there are no queries; else it has to fit Hkv.
la_status check_rows(const la_seqs* s) {
  if (!s) return LA_ERR_ARG;
  if (s->S < 0 || s->Tk < 0 || s->S > kMaxTokens || s->Tk > kMaxTokens) return LA_ERR_SHAPE;
  if (s->Hkv < 1 || s->Hkv > 65535 || s->Hq < 0 || s->Hq > 65535 || s->Hq % s->Hkv) return LA_ERR_SHAPE;
  if (s->d != 64 && s->d != 128) return LA_ERR_SHAPE;
  return LA_OK;
}

// Those of the calls that have queries; the strides of q, k and v only where the call has such rows.
la_status check_seqs(const la_seqs* s) {
  const la_status st = check_rows(s);
  if (st != LA_OK) return st;
  if (s->Hq < 1 || s->Tq < 0 || s->Tq > kMaxTokens || (s->causal != 0 && s->causal != 1)) return LA_ERR_SHAPE;
  return LA_OK;
}

constexpr int kRows = 256;              // packed rows of a workgroup (seq_attn.hip)
// What starting and ending a unit costs, and the smallest share of a workgroup, in keys.
constexpr uint32_t kRowsExtra = 512, kTokenExtra = 384, kRowsShare = 512, kTokenShare = 256;
constexpr int kMaxWorkgroups = 256;

// Where no sequence can have more keys than this (a cache's: than its table holds, since the lengths are on
// the GPU), units are not cut: nothing to join, so no workspace and no second launch.  kTokenWhole is set for
// eager calls, whose host side takes 11 us without the join's launch and 14.3 with it: one token over 256, 512,
// 1000 keys takes 11.0, 11.0, 11.1 us a call uncut and 14.4, 14.4, 14.3 cut, 32 sequences of 500 to 1000 keys 14.0
// and 14.9.  On the GPU alone (a captured call) the two meet near 800 keys: 256 keys 6.4 us (cut 9.3), 512 8.0 (9.7),
// 768 9.3 (9.8), 896 10.3 (9.9), 1000 11.0 (10.1), 2000 16.2 (10.5); 32 sequences of 256 to 512 keys 10.5 (12.5), of
// 500 to 1000 15.0 (14.7), of 2000 21.4 (16.3): a captured call over 800 to 1024 keys pays up to 0.9 us.
// kRowsWhole, on the GPU: a prompt of 256 tokens 16.0 us (cut 17.4), of 512 21.0 (22.4).
constexpr int kTokenWhole = 1024, kRowsWhole = 512;

SeqGeom seq_geom(const la_seqs& s, int rows, int kcap, uint32_t extra, uint32_t whole, uint32_t share, int uncut,
                 int heads = kRows) {
  SeqGeom g{};
  g.S = s.S;
  g.Tq = s.Tq;
  g.Kcap = kcap;
  g.lq_min = 1;
  g.lq_max = 0x7fffffff;
  g.Hq = s.Hq;
  g.Hkv = s.Hkv;
  g.G = s.Hq / s.Hkv;
  g.GH = g.G < rows ? g.G : rows;
  if (g.GH > heads) g.GH = heads;
  g.GS = ceil_div(g.G, g.GH);
  g.gh_magic = (65536 + g.GH - 1) / g.GH;
  g.TB = rows / g.GH;
  g.causal = s.causal;
  g.extra = extra;
  g.whole = whole;
  g.cuts = kcap > uncut;
  g.min_share = share;
  return g;
}

double most_units(const SeqGeom& g) {
  return (double)g.Hkv * g.GS * ((double)g.Tq / g.TB + (g.S < g.Tq ? g.S : g.Tq));
}

// Workgroups worth starting: no more than smallest shares of the most work there can be (sequences of
// at most kcap keys, kall in all).
int workgroups(const SeqGeom& g, int64_t kall, int most) {
  const double shares = ceil(most_units(g) * ((double)kall + g.extra) / g.min_share);
  const int want = shares < most ? (int)shares : most;
  return (want + 7) / 8 * 8;
}

struct PartLayout {
  int4* cut;
  float *m, *l, *o;
  size_t bytes;
};

PartLayout part_layout(const SeqGeom& g, int P, int rows, int d, void* ws) {
  PartLayout w{};
  if (!g.cuts) return w;
  char* p = (char*)ws;
  size_t at = 0;
  auto take = [&](size_t n) {
    char* r = p ? p + at : nullptr;
    at += align256(n);
    return r;
  };
  w.cut = (int4*)take((size_t)2 * P * sizeof(int4));
  w.m = (float*)take((size_t)2 * P * rows * sizeof(float));
  w.l = (float*)take((size_t)2 * P * rows * sizeof(float));
  w.o = (float*)take((size_t)2 * P * rows * d * sizeof(float));
  w.bytes = at;
  return w;
}

void set_parts(SeqIo* io, const PartLayout& w) {
  io->cut = w.cut;
  io->part_m = w.m;
  io->part_l = w.l;
  io->part_o = w.o;
}

SeqIo seq_io(const la_seqs& s, const void* q, void* o, float* lse, float scale) {
  SeqIo io{};
  io.q = (const uint16_t*)q;
  io.o = (uint16_t*)o;
  io.lse = lse;
  io.q_tok = s.q_token; io.q_head = s.q_head;
  io.o_tok = s.o_token; io.o_head = s.o_head;
  io.k_tok = s.k_token; io.k_head = s.k_head;
  io.v_tok = s.v_token; io.v_head = s.v_head;
  io.scale_log2 = (scale > 0.0f ? scale : 1.0f / sqrtf((float)s.d)) * 1.4426950408889634f;
  return io;
}

// Workgroups that the device runs at once, `per_cu` to a CU: CUs rounded down to a multiple of 8 (the XCDs).
int device_workgroups(int per_cu) {
  const int p = device_cu_count() / 8 * 8;
  return (p < 8 ? 8 : (p > kMaxWorkgroups ? kMaxWorkgroups : p)) * per_cu;
}

// The gradients' units (seq_grad.hip): what starting and ending one costs (of keys, and of query rows) and the
// smallest share of a workgroup, in rows of the inner axis; shares below kGradSnap end at the end of a unit of up to 5/4
// shares that lies within half a share; and nothing is cut where the inner axis has at most kGradWhole rows.  Chosen over
// 98 calls, 90 of them drawn: all three at 512 are 3.2 % slower (48 prompts of 1 to 300 tokens, 16 heads over 4, d 64, 39.5 us, with
// these 36.4), extras of 256 for both 2.2 %, a smallest share of 256 or 144 0.9 %; a snap of 4096 or none costs five
// prompts of 100 to 2100 (12 heads over 4, a bias) 120 instead of 115.
// A CU runs one workgroup of dK and dV and one of dQ at a time: 256 of each instead of 512 have half the cuts, and two
// kinds on a CU cover each other better than two of one kind that start together (the prompts above 73 -> 63 us and
// 130 -> 121; six of 150 to 3300, 24 heads over 8, d 128, 493 -> 466; a 480P chunk over its context 1806 -> 1765; one
// of 8192, 16 heads over 4, 818 either way).
constexpr uint32_t kGradKeysExtra = 256, kGradRowsExtra = 512, kGradShare = 192, kGradSnap = 2048;
constexpr int kGradWhole = 512, kGradPerCu = 1;

GradGeom grad_geom(const la_seqs& s, bool keys, bool bias) {
  GradGeom g{};
  g.S = s.S;
  g.Tq = s.Tq;
  g.Tk = s.Tk;
  g.Hq = s.Hq;
  g.Hkv = s.Hkv;
  g.G = s.Hq / s.Hkv;
  // the pairs' distances are added up head by head, so that a unit of a call with a bias has one
  g.GH = keys || bias ? 1 : (g.G < kGradRows ? g.G : kGradRows);
  g.GS = keys ? 1 : ceil_div(g.G, g.GH);
  g.gh_magic = (65536 + g.GH - 1) / g.GH;
  g.TB = kGradRows / g.GH;
  g.NH = s.Hkv * g.GS;
  g.causal = s.causal;
  g.extra = keys ? kGradKeysExtra : kGradRowsExtra;
  g.whole = kGradSnap;
  g.min_share = kGradShare;
  g.cuts = (keys ? (double)s.Tq * g.G : (double)s.Tk) > kGradWhole;
  return g;
}

int grad_workgroups(const GradGeom& g, bool keys) {
  const int rows = keys ? g.Tk : g.Tq;
  const double units = (double)g.NH * ((double)rows / g.TB + (g.S < rows ? g.S : rows));
  const double inner = keys ? (double)g.G * (g.Tq + 64.0 * (g.S < g.Tq ? g.S : g.Tq)) : (double)g.Tk;
  const double shares = ceil(units * (inner + g.extra) / g.min_share);
  const int most = kMaxWorkgroups * kGradPerCu, want = shares < most ? (int)shares : most;
  return (want + 7) / 8 * 8;
}

bool bad_bias(const la_rel_bias* b) {
  return b->lo > b->hi || b->lo < -(1 << 20) || b->hi > (1 << 20) || b->hi - b->lo >= kBiasMost || b->buckets < 1 ||
         b->buckets > (1 << 20);
}
int bias_pitch(const la_rel_bias* b) { return b->hi - b->lo + 1 + 2 * kBiasPad; }

struct GradLayout {
  float2* stat;
  float *table, *dist;
  uint64_t* line;
  int4 *keys_cut, *rows_cut;
  float *keys_part, *rows_part;
  size_t bytes;
};

GradLayout grad_layout(const la_seqs& s, const la_rel_bias* bias, void* ws) {
  GradLayout w{};
  char* p = (char*)ws;
  size_t at = 0;
  auto take = [&](size_t n) {
    char* r = p ? p + at : nullptr;
    at += align256(n);
    return r;
  };
  const GradGeom r = grad_geom(s, false, bias != nullptr), k = grad_geom(s, true, false);
  const size_t rp = grad_workgroups(r, false), kp = grad_workgroups(k, true);
  w.stat = (float2*)take(((size_t)s.Hq * s.Tq + 1) * sizeof(float2));     // read two at a time
  if (bias) {
    w.table = (float*)take((size_t)s.Hq * bias_pitch(bias) * sizeof(float));
    w.dist = (float*)take((rp + r.NH) * bias_pitch(bias) * sizeof(float));
    w.line = (uint64_t*)take(2 * sizeof(uint64_t));
  }
  const size_t rcut = r.cuts ? 2 * rp : 0, kcut = k.cuts ? 2 * kp : 0;
  w.keys_cut = (int4*)take(kcut * sizeof(int4));
  w.rows_cut = (int4*)take(rcut * sizeof(int4));
  w.keys_part = (float*)take(2 * kcut * kGradRows * s.d * sizeof(float));
  w.rows_part = (float*)take(rcut * kGradRows * s.d * sizeof(float));
  w.bytes = at;
  return w;
}

// The logits are formed as scale (q.k + bias / scale): the quotient of the largest bias is finite above this scale.
constexpr float kBiasScale = 0x1p-60f;

la_status check_bias(const la_rel_bias* bias, const int32_t* bucket, const void* weight, float scale) {
  if (bad_bias(bias)) return LA_ERR_SHAPE;
  if (scale > 0.0f && scale < kBiasScale) return LA_ERR_ARG;
  if (bias->dtype != LA_DTYPE_F32 && bias->dtype != LA_DTYPE_BF16) return LA_ERR_ARG;
  const uintptr_t word = bias->dtype == LA_DTYPE_F32 ? 3u : 1u;
  if (!bucket || !weight || ((uintptr_t)bucket & 3u) || ((uintptr_t)weight & word)) return LA_ERR_ARG;
  return LA_OK;
}

// How a call over whole prompts is made.  With a bias, sequences of up to kBiasKeys keys on average go to the kernel of
// 128 rows (bias_rows_kernel), whose starts and ends cost less, and longer ones to that of 256: d 64, 16 heads, 20 prompts
// of 100 tokens 11 against 19 us, 16 of 256 15 against 17, 4 of 1024 30 either way, 6 of 1024 54 against 52, 4 of 2048 93
// against 89; d 128, 8 of 512 27.5 against 32, 4 of 2048 140 against 132, 8192 causal tokens 270 against 230.  A unit has
// at most kBiasHeads heads then, whose tables are in LDS.
// Its units are not cut in calls of up to kBiasWhole keys, which saves the join.  Up to kBiasWholeShort keys it goes by
// how uneven the work can be, as the lengths are on the GPU: one sequence may have nearly all keys, and its units walk 60
// tiles, 50 to 70 us.  With a mean of up to 256 keys, units are whole up to kBiasWholeMost keys (20 prompts of 100 tokens, 4
// heads, 14.4 -> 9.7 us; one of 1900 with 7 of 28, 4 heads, would take 31 instead of 26).  Beyond, where there is a run of
// queries for every 16 keys, as 8 heads have: then the long sequence has many units too (16 prompts of 60 to 512 tokens, 16
// heads, 25 -> 21 us, 8 heads 22 -> 17; one of 3800 among 15 of 10 60 to 90 -> 69 to 79, with 8 heads 44 to 58 -> 71).  With
// fewer they are cut: that one with 4 heads takes 31 to 38 us instead of 52 to 72, 16 single tokens, of which one has 3900
// keys, 17 instead of 50, for 2 to 4 us more in even batches (16 over 250 keys 10.6 -> 13).  Continuations of a few queries
// (more than one a sequence, fewer than a sixteenth of the keys) are whole: 6 a sequence over 256 keys, 8 heads over 2, d 128,
// take 13.7 us instead of 15.8, but 71 instead of 22 where one sequence has nearly all keys.  A mean of up to 512 keys asks
// for 256 units too (8 of 512, 8 heads, d 128, 33 -> 25).  Calls of more keys are cut: whole units would save 1.5 to 4 us in
// even batches (32 prompts of 60 to 512 tokens 34 -> 32, 64 60 -> 56).
constexpr int kBiasKeys = 1024, kBiasWhole = 1024, kBiasWholeMost = 2048, kBiasWholeShort = 4096, kBiasPerCu = 2;
constexpr uint32_t kBiasExtra = 512, kBiasSnap = 2048, kBiasShare = 256;
struct PromptPlan {
  SeqGeom g;
  int rows, most;          // packed rows of a unit; workgroups (before the device's limit)
};
PromptPlan prompt_plan(const la_seqs& s, const la_rel_bias* bias) {
  PromptPlan p{};
  if (bias && s.Tk <= (int64_t)kBiasKeys * s.S) {
    p.g = seq_geom(s, kBiasRows, s.Tk, kBiasExtra, kBiasSnap, kBiasShare, kBiasWhole, kBiasHeads);
    const double mean = (double)s.Tk / s.S, runs = (double)p.g.Hkv * p.g.GS * p.g.Tq / p.g.TB;
    const bool fill = 16 * runs >= s.Tk, few = s.Tq > s.S && 16 * (int64_t)s.Tq < s.Tk;
    const bool whole = mean <= 256 ? s.Tk <= kBiasWholeMost || fill || few : mean <= 512 && fill && most_units(p.g) >= 256;
    if (s.Tk <= kBiasWholeShort && whole) p.g.cuts = 0;
    p.rows = kBiasRows;
  } else {
    p.g = seq_geom(s, kRows, s.Tk, kRowsExtra, 2 * kRowsExtra, kRowsShare, kRowsWhole, bias ? kBiasHeads : kRows);
    p.rows = kRows;
  }
  p.most = workgroups(p.g, s.Tk, kMaxWorkgroups * (p.rows == kRows ? 1 : kBiasPerCu));
  return p;
}

bool bad_kv4(const la_kv4* kv) {
  return kv->n_pages < 1 || kv->max_pages < 1 || kv->page < 16 || kv->page > 1024 || (kv->page & (kv->page - 1));
}

CacheGeom cache_geom(const la_seqs& s, const la_kv4& kv, const void* cache, const int32_t* table) {
  CacheGeom cg{(const uint8_t*)cache, table, kv.n_pages, kv.max_pages, 0, s.Hkv};
  while ((1 << cg.log_p) < kv.page) ++cg.log_p;
  return cg;
}

// How a call over a cache is made: sequences of at most lq_token query tokens by token_attn_kernel with
// `rows` packed rows a unit, those of more by seq_attn_kernel.  The first reads the cache once for every
// 32 rows, the second converts a tile once for 256 but takes longer to start a unit: over 6000 tokens, 4
// key heads of 4 query heads, 8 sequences of 128 rows 37 against 55 us, 2 of 256 rows 33 against 46, 32 of
// 128 rows 73 against 100, 32 of 256 rows 133 against 114.  Where all rows over all that the table holds
// are few products (kTokenWork query rows times keys) the first takes them whatever their length is: 539
// rows over 986 keys 13.8 against 28.4 us, 5580 rows over 5825 keys 41 against 53, 9600 over 6000 56 against
// 60; 17300 over 3041 57.5 against 54.3, 20200 over 3287 65 against 58.  The lengths are on the GPU, so a table
// that is wider than the sequences are long leaves their rows with the second kernel.
constexpr int kTokenRows = 192;
constexpr double kTokenWork = 50e6;
constexpr int kTokenPerCu = 2;
struct CachePlan {
  int lq_token, rows;
  bool few, many;          // there may be sequences of at most, and of more than, lq_token tokens
  SeqGeom token, many_rows;
  int p_token, p_many;     // workgroups (before the device's limit)
  size_t bytes;
};

CachePlan cache_plan(const la_seqs& s, const la_kv4& kv, int max_q) {
  CachePlan c{};
  const int G = s.Hq / s.Hkv;
  const int64_t cap64 = (int64_t)kv.max_pages * kv.page;
  const int cap = cap64 < kMaxTokens ? (int)cap64 : kMaxTokens;
  if (max_q > s.Tq) max_q = s.Tq;
  c.lq_token = G >= kTokenRows ? 1 : kTokenRows / G;
  if ((double)s.Tq * s.Hq * cap <= kTokenWork && max_q > c.lq_token) c.lq_token = max_q;
  c.many = max_q > c.lq_token;
  // a single sequence has all rows, so that it is one of many (or, where rows behind it are spare, may be
  // made like one); saves two launches, 9 us
  c.few = !(c.many && s.S == 1);
  c.rows = (int64_t)(c.many ? c.lq_token : max_q) * G <= 16 ? 16 : 32;
  c.token = seq_geom(s, c.rows, cap, kTokenExtra, 0, kTokenShare, kTokenWhole);
  c.token.lq_max = c.many ? c.lq_token : max_q;
  c.p_token = workgroups(c.token, cap, kMaxWorkgroups * kTokenPerCu);
  c.bytes = part_layout(c.token, c.p_token, c.rows, s.d, nullptr).bytes;
  if (c.many) {
    c.many_rows = seq_geom(s, kRows, cap, kRowsExtra, 2 * kRowsExtra, kRowsShare, kRowsWhole);
    c.many_rows.lq_min = c.few ? c.lq_token + 1 : 1;
    c.many_rows.lq_max = max_q;
    c.p_many = workgroups(c.many_rows, cap, kMaxWorkgroups);
    const size_t b = part_layout(c.many_rows, c.p_many, kRows, s.d, nullptr).bytes;
    if (b > c.bytes) c.bytes = b;
  }
  return c;
}

la_status check_cache_rows(const la_seqs* s, const la_kv4* kv, const void* k, const void* v, const int32_t* cu,
                           const int32_t* lens, const int32_t* table, const void* cache, bool written) {
  const la_status st = check_rows(s);
  if (st != LA_OK) return st;
  if (!kv) return LA_ERR_ARG;
  if (bad_kv4(kv) || s->Tk > kMaxCacheRows) return LA_ERR_SHAPE;
  if (s->S == 0 || s->Tk == 0) return LA_OK;
  if (bad_strides(s->k_token, s->k_head, s->d, written) || bad_strides(s->v_token, s->v_head, s->d, written))
    return LA_ERR_SHAPE;
  if (!k || !v || !cu || !lens || !table || !cache) return LA_ERR_ARG;
  if (misaligned(k) || misaligned(v) || misaligned(cache)) return LA_ERR_ARG;
  if (((uintptr_t)cu | (uintptr_t)lens | (uintptr_t)table) & 3u) return LA_ERR_ARG;
  return LA_OK;
}

}  // namespace

extern "C" {

size_t la_prompt_ws_bytes(const la_seqs* seqs) { return la_prompt_bias_ws_bytes(seqs, nullptr); }

size_t la_prompt_bias_ws_bytes(const la_seqs* seqs, const la_rel_bias* bias) {
  if (check_seqs(seqs) != LA_OK || (bias && bad_bias(bias)) || seqs->S == 0 || seqs->Tq == 0) return 0;
  const PromptPlan p = prompt_plan(*seqs, bias);
  return part_layout(p.g, p.most, p.rows, seqs->d, nullptr).bytes;
}

la_status la_prompt_attn(const la_seqs* seqs, const void* q, const void* k, const void* v, const int32_t* cu_q,
                         const int32_t* cu_k, float scale, void* o, float* lse, void* ws, size_t ws_bytes,
                         void* stream) {
  return la_prompt_attn_bias(seqs, nullptr, q, k, v, cu_q, cu_k, nullptr, nullptr, scale, o, lse, ws, ws_bytes, stream);
}

la_status la_prompt_attn_bias(const la_seqs* seqs, const la_rel_bias* bias, const void* q, const void* k, const void* v,
                              const int32_t* cu_q, const int32_t* cu_k, const int32_t* bucket, const void* weight,
                              float scale, void* o, float* lse, void* ws, size_t ws_bytes, void* stream) {
  la_status st = check_seqs(seqs);
  if (st != LA_OK) return st;
  if (isnan(scale) || isinf(scale)) return LA_ERR_ARG;
  if (bias) {
    if (bad_bias(bias)) return LA_ERR_SHAPE;
    if (bias->dtype != LA_DTYPE_F32 && bias->dtype != LA_DTYPE_BF16) return LA_ERR_ARG;
  }
  if (seqs->S == 0 || seqs->Tq == 0) return LA_OK;
  if (bad_strides(seqs->q_token, seqs->q_head, seqs->d, false) || bad_strides(seqs->o_token, seqs->o_head, seqs->d, true))
    return LA_ERR_SHAPE;
  if (seqs->Tk > 0 && (bad_strides(seqs->k_token, seqs->k_head, seqs->d, false) ||
                       bad_strides(seqs->v_token, seqs->v_head, seqs->d, false)))
    return LA_ERR_SHAPE;
  if (!q || !o || !cu_q || !cu_k || (seqs->Tk > 0 && (!k || !v))) return LA_ERR_ARG;
  if (misaligned(q) || misaligned(o) || misaligned(k) || misaligned(v)) return LA_ERR_ARG;
  if (((uintptr_t)cu_q | (uintptr_t)cu_k | (uintptr_t)lse) & 3u) return LA_ERR_ARG;
  SeqBias b{};
  if (bias) {
    st = check_bias(bias, bucket, weight, scale);
    if (st != LA_OK) return st;
    b = SeqBias{bucket, weight, bias->dtype == LA_DTYPE_BF16, bias->buckets, bias->lo, bias->hi};
  }
  PromptPlan p = prompt_plan(*seqs, bias);
  p.g.cu_q = cu_q;
  p.g.ks = cu_k;
  const PartLayout w = part_layout(p.g, p.most, p.rows, seqs->d, ws);
  if (w.bytes > 0 && (!ws || ws_bytes < w.bytes || ((uintptr_t)ws & 255u))) return LA_ERR_WORKSPACE;
  SeqIo io = seq_io(*seqs, q, o, lse, scale);
  io.k = (const uint16_t*)k;
  io.v = (const uint16_t*)v;
  set_parts(&io, w);
  const int have = device_workgroups(p.rows == kRows ? 1 : kBiasPerCu);
  const hipError_t e = launch_prompt_attn(p.g, io, bias ? &b : nullptr, seqs->d, p.rows, p.most < have ? p.most : have,
                                          (hipStream_t)stream);
  return e == hipSuccess ? LA_OK : LA_ERR_HIP;
}

size_t la_kv4_page_bytes(int32_t d, int32_t page) {
  const la_kv4 kv{1, page, 1};
  if ((d != 64 && d != 128) || bad_kv4(&kv)) return 0;
  return (size_t)page * (d + d / 16);
}

la_status la_kv4_append(const la_seqs* seqs, const la_kv4* kv, const void* k, const void* v, const int32_t* cu,
                        const int32_t* lens, const int32_t* table, void* cache, void* stream) {
  const la_status st = check_cache_rows(seqs, kv, k, v, cu, lens, table, cache, false);
  if (st != LA_OK || seqs->S == 0 || seqs->Tk == 0) return st;
  const CacheGeom cg = cache_geom(*seqs, *kv, cache, table);
  const hipError_t e = launch_kv4_append(*seqs, cg, k, v, cu, lens, cache, (hipStream_t)stream);
  return e == hipSuccess ? LA_OK : LA_ERR_HIP;
}

la_status la_kv4_read(const la_seqs* seqs, const la_kv4* kv, const void* cache, const int32_t* cu, const int32_t* lens,
                      const int32_t* table, void* k, void* v, void* stream) {
  const la_status st = check_cache_rows(seqs, kv, k, v, cu, lens, table, cache, true);
  if (st != LA_OK || seqs->S == 0 || seqs->Tk == 0) return st;
  const CacheGeom cg = cache_geom(*seqs, *kv, cache, table);
  const hipError_t e = launch_kv4_read(*seqs, cg, cu, lens, k, v, (hipStream_t)stream);
  return e == hipSuccess ? LA_OK : LA_ERR_HIP;
}

size_t la_kv4_ws_bytes(const la_seqs* seqs, const la_kv4* kv, int32_t max_q) {
  if (check_seqs(seqs) != LA_OK || !kv || bad_kv4(kv) || max_q < 1 || seqs->S == 0 || seqs->Tq == 0) return 0;
  return cache_plan(*seqs, *kv, max_q).bytes;
}

la_status la_kv4_attn(const la_seqs* seqs, const la_kv4* kv, int32_t max_q, const void* q, const void* cache,
                      const int32_t* cu_q, const int32_t* lens, const int32_t* table, float scale, void* o, float* lse,
                      void* ws, size_t ws_bytes, void* stream) {
  la_status st = check_seqs(seqs);
  if (st != LA_OK) return st;
  if (!kv || max_q < 0 || isnan(scale) || isinf(scale)) return LA_ERR_ARG;
  if (bad_kv4(kv)) return LA_ERR_SHAPE;
  if (seqs->S == 0 || seqs->Tq == 0 || max_q == 0) return LA_OK;
  if (bad_strides(seqs->q_token, seqs->q_head, seqs->d, false) || bad_strides(seqs->o_token, seqs->o_head, seqs->d, true))
    return LA_ERR_SHAPE;
  if (!q || !o || !cache || !cu_q || !lens || !table) return LA_ERR_ARG;
  if (misaligned(q) || misaligned(o) || misaligned(cache)) return LA_ERR_ARG;
  if (((uintptr_t)cu_q | (uintptr_t)lens | (uintptr_t)table | (uintptr_t)lse) & 3u) return LA_ERR_ARG;
  CachePlan c = cache_plan(*seqs, *kv, max_q);
  if (c.bytes > 0 && (!ws || ws_bytes < c.bytes || ((uintptr_t)ws & 255u))) return LA_ERR_WORKSPACE;
  const CacheGeom cg = cache_geom(*seqs, *kv, cache, table);
  SeqIo io = seq_io(*seqs, q, o, lse, scale);
  c.token.cu_q = c.many_rows.cu_q = cu_q;
  c.token.ks = c.many_rows.ks = lens;
  // one after the other on the stream, so they may use the same scratch
  set_parts(&io, part_layout(c.token, c.p_token, c.rows, seqs->d, ws));
  hipError_t e = hipSuccess;
  if (c.few) {
    const int have = device_workgroups(kTokenPerCu);
    e = launch_cache_tokens(c.token, io, cg, seqs->d, c.rows, c.p_token < have ? c.p_token : have, (hipStream_t)stream);
  }
  if (e == hipSuccess && c.many) {
    set_parts(&io, part_layout(c.many_rows, c.p_many, kRows, seqs->d, ws));
    const int have = device_workgroups(1);
    e = launch_cache_rows(c.many_rows, io, cg, seqs->d, c.p_many < have ? c.p_many : have, (hipStream_t)stream);
  }
  return e == hipSuccess ? LA_OK : LA_ERR_HIP;
}

size_t la_prompt_bwd_ws_bytes(const la_seqs* seqs, const la_rel_bias* bias) {
  if (check_seqs(seqs) != LA_OK || (bias && bad_bias(bias)) || seqs->S == 0) return 0;
  return grad_layout(*seqs, bias, nullptr).bytes;
}

la_status la_prompt_attn_bwd(const la_seqs* seqs, const la_prompt_grads* grads, const la_rel_bias* bias,
                             const void* dout, const void* q, const void* k, const void* v, const void* o,
                             const float* lse, const float* dlse, const int32_t* cu_q, const int32_t* cu_k,
                             const int32_t* bucket, const void* weight, float scale, void* dq, void* dk, void* dv,
                             void* dweight, void* ws, size_t ws_bytes, void* stream) {
  la_status st = check_seqs(seqs);
  if (st != LA_OK) return st;
  if (!grads || isnan(scale) || isinf(scale)) return LA_ERR_ARG;
  if (bias) {
    st = check_bias(bias, bucket, weight, scale);
    if (st != LA_OK) return st;
    if (!dweight || ((uintptr_t)dweight & (bias->dtype == LA_DTYPE_F32 ? 3u : 1u))) return LA_ERR_ARG;
  }
  const la_seqs& s = *seqs;
  const bool rows = s.S > 0 && s.Tq > 0, keys = s.S > 0 && s.Tk > 0;
  if (rows && (bad_strides(s.q_token, s.q_head, s.d, false) || bad_strides(s.o_token, s.o_head, s.d, false) ||
               bad_strides(grads->do_token, grads->do_head, s.d, false) ||
               bad_strides(grads->dq_token, grads->dq_head, s.d, true)))
    return LA_ERR_SHAPE;
  if (keys && (bad_strides(s.k_token, s.k_head, s.d, false) || bad_strides(s.v_token, s.v_head, s.d, false) ||
               bad_strides(grads->dk_token, grads->dk_head, s.d, true) ||
               bad_strides(grads->dv_token, grads->dv_head, s.d, true)))
    return LA_ERR_SHAPE;
  if (!rows && !keys && !bias) return LA_OK;
  if (rows && (!dout || !q || !o || !lse || !dq)) return LA_ERR_ARG;
  if (keys && (!k || !v || !dk || !dv)) return LA_ERR_ARG;
  if ((rows || keys) && (!cu_q || !cu_k)) return LA_ERR_ARG;
  if (misaligned(dout) || misaligned(q) || misaligned(k) || misaligned(v) || misaligned(o) || misaligned(dq) ||
      misaligned(dk) || misaligned(dv))
    return LA_ERR_ARG;
  if (((uintptr_t)cu_q | (uintptr_t)cu_k | (uintptr_t)lse | (uintptr_t)dlse) & 3u) return LA_ERR_ARG;
  GradLayout w{};
  if (rows || keys) {
    w = grad_layout(s, bias, ws);
    if (w.bytes > 0 && (!ws || ws_bytes < w.bytes || ((uintptr_t)ws & 255u))) return LA_ERR_WORKSPACE;
  }
  GradCall c{};
  c.rows = rows;
  c.keys = keys;
  c.has_bias = bias != nullptr;
  c.rows_g = grad_geom(s, false, bias != nullptr);
  c.keys_g = grad_geom(s, true, false);
  c.rows_g.cu_q = c.keys_g.cu_q = cu_q;
  c.rows_g.cu_k = c.keys_g.cu_k = cu_k;
  const int have = device_workgroups(kGradPerCu);
  c.rows_p = grad_workgroups(c.rows_g, false);
  c.keys_p = grad_workgroups(c.keys_g, true);
  if (c.rows_p > have) c.rows_p = have;
  if (c.keys_p > have) c.keys_p = have;
  GradIo io{};
  io.q = (const uint16_t*)q;
  io.k = (const uint16_t*)k;
  io.v = (const uint16_t*)v;
  io.dout = (const uint16_t*)dout;
  io.q_tok = s.q_token; io.q_head = s.q_head;
  io.k_tok = s.k_token; io.k_head = s.k_head;
  io.v_tok = s.v_token; io.v_head = s.v_head;
  io.do_tok = grads->do_token; io.do_head = grads->do_head;
  io.stat = w.stat;
  io.scale = scale > 0.0f ? scale : 1.0f / sqrtf((float)s.d);
  io.scale_log2 = io.scale * 1.4426950408889634f;
  if (bias) {
    io.table = w.table;
    io.bias_lo = bias->lo;
    io.bias_hi = bias->hi;
    io.bias_pitch = bias_pitch(bias);
    io.dist = w.dist;
    io.line = w.line;
    c.bias = SeqBias{bucket, weight, bias->dtype == LA_DTYPE_BF16, bias->buckets, bias->lo, bias->hi};
    c.dweight = dweight;
  }
  c.rows_io = c.keys_io = io;
  c.rows_io.part = w.rows_part;
  c.rows_io.cut = w.rows_cut;
  c.keys_io.part = w.keys_part;
  c.keys_io.cut = w.keys_cut;
  c.rows_io.out0 = (uint16_t*)dq;
  c.rows_io.out0_tok = grads->dq_token; c.rows_io.out0_head = grads->dq_head;
  c.keys_io.out0 = (uint16_t*)dk;
  c.keys_io.out0_tok = grads->dk_token; c.keys_io.out0_head = grads->dk_head;
  c.keys_io.out1 = (uint16_t*)dv;
  c.keys_io.out1_tok = grads->dv_token; c.keys_io.out1_head = grads->dv_head;
  c.Tq = s.Tq;
  c.o = (const uint16_t*)o;
  c.o_tok = s.o_token; c.o_head = s.o_head;
  c.lse = lse;
  c.dlse = dlse;
  const hipError_t e = launch_prompt_bwd(c, s.d, (hipStream_t)stream);
  return e == hipSuccess ? LA_OK : LA_ERR_HIP;
}

}  // extern "C"
