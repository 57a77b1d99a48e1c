// Host side of the entry points over packed sequences (include/la.h): validation, the shapes that
// the kernels take, workspaces and launches.  Nothing here allocates device memory.
#include <math.h>

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

SeqGeom seq_geom(const la_seqs& s, int rows, int kcap, uint32_t extra, uint32_t whole, uint32_t share, int uncut) {
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

// Workgroups worth starting: no more than smallest shares of the most work there can be (sequences of
// at most kcap keys, kall in all).
int workgroups(const SeqGeom& g, int64_t kall, int most) {
  const double units = (double)g.Hkv * g.GS * ((double)g.Tq / g.TB + (g.S < g.Tq ? g.S : g.Tq));
  const double shares = ceil(units * ((double)kall + g.extra) / g.min_share);
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

size_t la_prompt_ws_bytes(const la_seqs* seqs) {
  if (check_seqs(seqs) != LA_OK || seqs->S == 0 || seqs->Tq == 0) return 0;
  const SeqGeom g = seq_geom(*seqs, kRows, seqs->Tk, kRowsExtra, 2 * kRowsExtra, kRowsShare, kRowsWhole);
  return part_layout(g, workgroups(g, seqs->Tk, kMaxWorkgroups), kRows, seqs->d, nullptr).bytes;
}

la_status la_prompt_attn(const la_seqs* seqs, const void* q, const void* k, const void* v, const int32_t* cu_q,
                         const int32_t* cu_k, float scale, void* o, float* lse, void* ws, size_t ws_bytes,
                         void* stream) {
  la_status st = check_seqs(seqs);
  if (st != LA_OK) return st;
  if (isnan(scale) || isinf(scale)) return LA_ERR_ARG;
  if (seqs->S == 0 || seqs->Tq == 0) return LA_OK;
  if (bad_strides(seqs->q_token, seqs->q_head, seqs->d, false) || bad_strides(seqs->o_token, seqs->o_head, seqs->d, true))
    return LA_ERR_SHAPE;
  if (seqs->Tk > 0 && (bad_strides(seqs->k_token, seqs->k_head, seqs->d, false) ||
                       bad_strides(seqs->v_token, seqs->v_head, seqs->d, false)))
    return LA_ERR_SHAPE;
  if (!q || !o || !cu_q || !cu_k || (seqs->Tk > 0 && (!k || !v))) return LA_ERR_ARG;
  if (misaligned(q) || misaligned(o) || misaligned(k) || misaligned(v)) return LA_ERR_ARG;
  if (((uintptr_t)cu_q | (uintptr_t)cu_k | (uintptr_t)lse) & 3u) return LA_ERR_ARG;
  SeqGeom g = seq_geom(*seqs, kRows, seqs->Tk, kRowsExtra, 2 * kRowsExtra, kRowsShare, kRowsWhole);
  g.cu_q = cu_q;
  g.ks = cu_k;
  const int most = workgroups(g, seqs->Tk, kMaxWorkgroups);
  const PartLayout w = part_layout(g, most, kRows, seqs->d, ws);
  if (w.bytes > 0 && (!ws || ws_bytes < w.bytes || ((uintptr_t)ws & 255u))) return LA_ERR_WORKSPACE;
  SeqIo io = seq_io(*seqs, q, o, lse, scale);
  io.k = (const uint16_t*)k;
  io.v = (const uint16_t*)v;
  set_parts(&io, w);
  const int have = device_workgroups(1);
  const hipError_t e = launch_prompt_attn(g, io, seqs->d, most < have ? most : have, (hipStream_t)stream);
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

}  // extern "C"
