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

// Shared checks of a la_seqs; the strides of k and v only where the call has such rows.
la_status check_seqs(const la_seqs* s) {
  if (!s) return LA_ERR_ARG;
  if (s->S < 0 || s->Tq < 0 || s->Tk < 0 || s->Hq < 1 || s->Hkv < 1 || s->Hq % s->Hkv) return LA_ERR_SHAPE;
  if (s->Hq > 65535 || (s->d != 64 && s->d != 128)) return LA_ERR_SHAPE;
  if (s->causal != 0 && s->causal != 1) return LA_ERR_SHAPE;
  return LA_OK;
}

constexpr int kRows = 256;              // packed rows of a workgroup (seq_attn.hip)
constexpr uint32_t kMinShare = 256;     // keys
constexpr int kMaxWorkgroups = 256;

SeqGeom seq_geom(const la_seqs& s, int rows, int kcap) {
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
  g.TB = rows / g.GH;
  g.causal = s.causal;
  g.min_share = kMinShare;
  return g;
}

// Workgroups worth starting: no more than smallest shares of the most work there can be (sequences of
// at most kcap keys, kall in all).
int workgroups(const SeqGeom& g, int64_t kall, int most) {
  const double units = (double)g.Hkv * g.GS * ((double)g.Tq / g.TB + (g.S < g.Tq ? g.S : g.Tq));
  const double shares = ceil(units * (double)(kall > 0 ? kall : 1) / g.min_share);
  const int want = shares < most ? (int)shares : most;
  return (want + 7) / 8 * 8;
}

struct PartLayout {
  int4* cut;
  float *m, *l, *o;
  size_t bytes;
};

PartLayout part_layout(int P, int rows, int d, void* ws) {
  PartLayout w{};
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

// Workgroups that the device runs at once: CUs rounded down to a multiple of 8 (the XCDs).
int device_workgroups() {
  const int cus = device_cu_count();
  const int p = cus / 8 * 8;
  return p < 8 ? 8 : (p > kMaxWorkgroups ? kMaxWorkgroups : p);
}

}  // namespace

extern "C" {

size_t la_prompt_ws_bytes(const la_seqs* seqs) {
  if (check_seqs(seqs) != LA_OK || seqs->S == 0 || seqs->Tq == 0) return 0;
  const SeqGeom g = seq_geom(*seqs, kRows, seqs->Tk);
  return part_layout(workgroups(g, seqs->Tk, kMaxWorkgroups), kRows, seqs->d, nullptr).bytes;
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
  SeqGeom g = seq_geom(*seqs, kRows, seqs->Tk);
  g.cu_q = cu_q;
  g.ks = cu_k;
  const int most = workgroups(g, seqs->Tk, kMaxWorkgroups);
  const PartLayout w = part_layout(most, kRows, seqs->d, ws);
  if (!ws || ws_bytes < w.bytes || ((uintptr_t)ws & 255u)) return LA_ERR_WORKSPACE;
  SeqIo io = seq_io(*seqs, q, o, lse, scale);
  io.k = (const uint16_t*)k;
  io.v = (const uint16_t*)v;
  set_parts(&io, w);
  const int have = device_workgroups();
  const hipError_t e = launch_prompt_attn(g, io, seqs->d, most < have ? most : have, (hipStream_t)stream);
  return e == hipSuccess ? LA_OK : LA_ERR_HIP;
}

}  // extern "C"
