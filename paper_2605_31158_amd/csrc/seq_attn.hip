// Attention over packed sequences on gfx950: queries [T, Hq, d] of sequences of different lengths,
// each over its own keys, causal (the last query sees the last key) or not, with grouped heads.
// Keys and values are bf16 rows (the attention over a whole prompt) or the pages of a 4-bit cache
// (many query tokens over a cache; few of them: seq_token.hip).
//
// Per query row: one pass over the keys in tiles of 64 with a running maximum m and sum l,
//   m' = max(m, s);  O = 2^(m - m') O + sum 2^(s - m') v;  l = 2^(m - m') l + sum 2^(s - m')
// and o = O / l, lse = m + log l at the end; the tile core is that of the block-sparse attention
// (attn_core.h, and attn.hip for its phases: two groups of four waves take turns at the matrix
// pipeline and at the softmax).  A workgroup has 256 packed rows: the rows of a group's heads share
// K and V, so grouped heads cost no more reads than one.  The work is cut into equal shares over
// one persistent workgroup per CU (seq_walk.h); a unit cut between two leaves (O, m, l) partials that
// seq_merge joins, in a fixed order.
//
// The weights 2^(s - m) are rounded to bf16 for the product with V (by at most 2^-8 of themselves), since the
// matrix pipeline takes bf16 operands at 16 times the rate of fp32 ones; m, l and O stay in fp32, and l adds the
// weights before they are rounded.  Relative rms error of o against 64 bits 0.0018 to 0.0023; its own rounding to
// bf16 alone makes 0.0016.
//
// A relative bias costs where a tile lies within its reach: its accumulators start from the bias instead of 0 (read
// from LDS, in units of q.k), while the tiles beyond have one number a row, by which the maximum they are formed
// against is moved.  16 prompts of 60 to 512 tokens, 16 heads, d 64, take 28.5 us here (without a bias 26.2; short
// sequences go to bias_rows_kernel), 8192 causal tokens as below 225 (221); added behind the product it was 32.6 and
// 251 (copies of the logits where the two kinds of tiles meet), and two calls of the softmax, one for each kind, spill.
//
// Differences from attn.hip: the tiles of a piece are consecutive, so nothing is read to know the
// next one (no records); K and V rows have a stride; and the loop ends with the piece, so a piece
// pays one load latency of its own.
//
// Bound by the matrix pipeline under the card's power limit where pieces are long: 8192 causal tokens, 16
// query heads over 4, d 128, in 213 us, 1.29 PFLOP/s of the 1.36 that a large bf16 product of random data
// reaches here (1.63 us a tile of 256 x 64); 6240 queries over 12480 tokens of a 4-bit cache, 16 heads, in
// 520 us, 1.23 PFLOP/s.  A piece costs about 8 us beside its tiles: the 128 KB of Q and O that every
// workgroup moves at the same time, and the latency of the first tiles; one workgroup to a CU (96 KB of LDS at
// d 128) has nothing to cover it with.  64-wide heads do the same vector work a logit for half the products:
// 8192 tokens as above take 155 us, 0.89 PFLOP/s.  Sequences of 150 to 3300 tokens
// (6, 24 heads over 8) take 124 us where their products alone take 77.  Holding the next piece's Q in LDS,
// with its tiles issued before the results are written, was right and no faster (registers, and the
// bytes are the same).
#include <math.h>

#include <type_traits>

#include "attn_core.h"
#include "kv4.h"
#include "seq_walk.h"

namespace la {
namespace {

// One wave's running piece.
template <int D>
struct PieceState {
  using X = Mma<D>;
  typename X::Acc oacc[D / X::MR][X::QT];
  typename X::Acc sacc[KT / X::MR][X::QT];
  bf16x8 pb[KT / X::KC][X::QT];
  bf16x8 qreg[D / X::KC][X::QT];
  float m_run[X::QT], l_run[X::QT];
  int seen;                // keys that some row of the wave sees, 0 when it has no rows
};

// The source of one group's tiles (V: the group that loads V, else K), bf16 rows: asynchronous
// loads to LDS, their descriptors end at the sequence's last key, so tiles read zeros behind it.
template <int D, bool V>
struct RowTiles {
  const uint16_t* base;
  int64_t step;            // elements from tile to tile
  uint64_t at;             // byte offset of the next tile to issue
  uint32_t stride;         // bytes from row to row
  int left;                // keys from the next tile on
  uint32_t off[Tile<D>::PER];
  int lw;

  __device__ __forceinline__ void init(const SeqIo& io, const CacheGeom&, int lw_, int lane) {
    base = V ? io.v : io.k;
    lw = lw_;
    stride = (uint32_t)(V ? io.v_tok : io.k_tok) * 2u;
#pragma unroll
    for (int i = 0; i < Tile<D>::PER; ++i) off[i] = slot_offset<D, V>(lw, i, lane, stride);
  }
  // a piece's first tile into d0, its second into d1 where there is one
  __device__ __forceinline__ void prime(const SeqIo& io, const Walk& wk, int kvh, int ta, int tb, unsigned char* d0,
                                        unsigned char* d1) {
    const Seq& q = wk.q;
    const int64_t tok = V ? io.v_tok : io.k_tok, head = V ? io.v_head : io.k_head;
    at = first_lane_u64((uint64_t)(((int64_t)q.k0 + 64 * (int64_t)ta) * tok + kvh * head) * 2u);
    left = __builtin_amdgcn_readfirstlane(min(q.lk, 64 * tb) - 64 * ta);
    issue(d0);
    if (d1) issue(d1);
  }
  // the next tile into LDS; behind the piece's last one nothing is read (its rows come as zeros)
  __device__ __forceinline__ void issue(unsigned char* dst) {
    const uint32_t nrec = __builtin_amdgcn_readfirstlane((uint32_t)min(max(left, 0), KT) * stride);
    issue_tile<D>(dst + lw * (Tile<D>::BYTES / 4), base, first_lane_u64(at), nrec, off);
    at += (uint64_t)KT * stride;
    left -= KT;
  }
  // all but the tile issued last have landed
  __device__ __forceinline__ void wait() { wait_vmem<Tile<D>::PER>(); }
};

// The same from the pages of a 4-bit cache: a thread holds the codes of one tile more in registers
// (16 bytes, 8 for d = 64, and their scales) and turns them into bf16 where the tile is due; the page
// numbers are read a tile before the codes.  Keys at the sequence's end and on pages that do not
// exist come as zeros.
template <int D, bool V>
struct CacheTiles {
  using F = Kv4<D>;
  using T = Tile<D>;
  typedef typename std::conditional<D == 128, u32x4, u32x2>::type Codes;
  CacheGeom cg;
  const int32_t* row;      // the sequence's pages
  int kvh, lk, tb;
  int key;                 // first key of the tile that the next codes are loaded for
  int id;                  // this thread's page of it
  int at_tile;             // this thread's first key inside a tile
  int nv;                  // of its keys (K: 1, V: 4) in `codes`, those that exist
  Codes codes;
  uint32_t scales;
  int part;                // K: which quarter of the row; V: which chunk
  uint32_t dst0;

  __device__ __forceinline__ void init(const SeqIo&, const CacheGeom& cg_, int lw, int lane) {
    cg = cg_;
    const int gt = lw * 64 + lane;
    // row r = at_tile + j of a V tile, or slot (d / 32) part + j of a K row, is swizzled by an exclusive or
    // of j's bits with those of j = 0, at which `dst0` points
    if (V) {
      constexpr int CB = 2 * Mma<D>::MR;                    // bytes that are permuted as one
      at_tile = 4 * (gt >> 4);
      part = gt & 15;
      const int lo = part * (D / 8);
      dst0 = (uint32_t)(at_tile * T::STRIDE + ((lo / CB) ^ T::vswz(at_tile)) * CB + lo % CB);
    } else {
      at_tile = gt >> 2;
      part = gt & 3;
      dst0 = (uint32_t)(at_tile * T::STRIDE + (((D / 32) * part) ^ T::kswz(at_tile)) * 16);
    }
  }
  __device__ __forceinline__ uint32_t dst_off(int j) const {
    return V ? (dst0 ^ (uint32_t)((D == 128 ? j : j >> 1) * 2 * Mma<D>::MR)) + (uint32_t)(j * T::STRIDE)
             : dst0 ^ (uint32_t)(16 * j);
  }
  __device__ __forceinline__ void load_id() {
    const int idx = min((key + at_tile) >> cg.log_p, cg.max_pages - 1);
    id = row[idx];
  }
  // codes of the next tile; page numbers of the one behind it
  __device__ __forceinline__ void load() {
    const int P = 1 << cg.log_p, k = key + at_tile, in = k & (P - 1);
    bool ok;
    const uint8_t* pg = page_of<D>(cg, id, kvh, &ok);
    const int most = key < 64 * tb ? lk - k : 0;
    nv = ok ? min(max(most, 0), V ? 4 : 1) : 0;
    if (V) {
      codes = *(const Codes*)(pg + F::v_code(P) + ((in >> 2) * 16 + part) * (4 * F::WB));
      scales = *(const uint32_t*)(pg + F::v_scale(P) + (part * D / 512) * P + in);
    } else {
      codes = *(const Codes*)(pg + in * F::ROW + part * (F::ROW / 4));
      scales = pg[F::k_scale(P) + (part * D / 128) * P + in];
    }
    key += KT;
    load_id();
  }
  __device__ __forceinline__ void write(unsigned char* dst) {
    if (V) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float sc = j < nv ? scale_of(scales, j) : 1.0f;
        if constexpr (D == 128) {
          *(u32x4*)(dst + dst_off(j)) = fp4x8(j < nv ? codes[j] : 0u, sc);
        } else {
          const uint32_t w = j < nv ? codes[j >> 1] >> (16 * (j & 1)) : 0u;
          *(u32x2*)(dst + dst_off(j)) = u32x2{fp4x2<0>(w, sc), fp4x2<1>(w, sc)};
        }
      }
    } else {
      const float sc = nv ? scale_of(scales, 0) : 1.0f;
#pragma unroll
      for (int j = 0; j < D / 32; ++j) *(u32x4*)(dst + dst_off(j)) = fp4x8(nv ? codes[j] : 0u, sc);
    }
  }
  __device__ __forceinline__ void prime(const SeqIo&, const Walk& wk, int kvh_, int ta, int tb_, unsigned char* d0,
                                        unsigned char* d1) {
    row = cg.table + (int64_t)wk.s * cg.max_pages;
    kvh = kvh_;
    lk = wk.q.lk;
    tb = tb_;
    key = 64 * ta;
    load_id();
    load();
    write(d0);
    load();
    if (d1) {
      write(d1);
      load();
    }
  }
  __device__ __forceinline__ void issue(unsigned char* dst) {
    write(dst);
    load();
  }
  // the tile stored last is in LDS
  __device__ __forceinline__ void wait() {
    asm volatile("" ::: "memory");                      // the compiler moves no store behind the wait
    __builtin_amdgcn_s_waitcnt(0xC07F);                 // lgkmcnt(0)
  }
};

// Starts a piece: O and l zero, the maximum at -inf, the wave's Q rows and how far each sees.
template <int D>
__device__ __forceinline__ void start_rows(PieceState<D>& st, WaveCtx& w, const SeqGeom& g, const SeqIo& io,
                                           const Walk& wk, int r_off, int c, int lg) {
  using X = Mma<D>;
  int seen = 0;
#pragma unroll
  for (int qt = 0; qt < X::QT; ++qt) {
    st.m_run[qt] = -INFINITY;
    st.l_run[qt] = 0.f;
#pragma unroll
    for (int dt = 0; dt < D / X::MR; ++dt)
#pragma unroll
      for (int i = 0; i < X::AR; ++i) st.oacc[dt][qt][i] = 0.f;
    const Row row = unit_row(g, wk, r_off + X::MR * qt + c);
    const uint16_t* src = io.q + (int64_t)(wk.q.q0 + row.token) * io.q_tok + (int64_t)row.head * io.q_head + 8 * lg;
#pragma unroll
    for (int ks = 0; ks < D / X::KC; ++ks) {
      u32x4 qw = u32x4{0u, 0u, 0u, 0u};
      if (row.ok) qw = *(const u32x4*)(src + X::KC * ks);
      st.qreg[ks][qt] = __builtin_bit_cast(bf16x8, qw);
    }
    const int keys = token_keys(g, wk.q, row.token);
    w.klimit[qt] = row.ok ? keys : 0x7fffffff;      // rows that do not exist are not worth a mask
    seen = max(seen, row.ok ? keys : 0);
  }
#pragma unroll
  for (int m = 1; m < X::MR; m <<= 1) seen = max(seen, __shfl_xor(seen, m));
  st.seen = __builtin_amdgcn_readfirstlane(seen);
}

// Ends a piece: bf16 rows (and lse) where the piece is the whole unit, else the partial.
template <int D, int R = QR>
__device__ __forceinline__ void end_rows(const PieceState<D>& st, const SeqGeom& g, const SeqIo& io, const Walk& wk,
                                         const Piece& pc, int slot0, int r_off, int c, int lg) {
  using X = Mma<D>;
  const bool whole = pc.ta == 0 && pc.tb == pc.n;
  const int slot = slot0 + (pc.ta == 0 ? 1 : 0);
  if (!whole && threadIdx.x == 0) io.cut[slot] = unit_record(g, wk);
#pragma unroll
  for (int qt = 0; qt < X::QT; ++qt) {
    float l = st.l_run[qt];
    if constexpr (X::NG == 4) l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    const int r = r_off + X::MR * qt + c;
    const Row row = unit_row(g, wk, r);
    u32x4 y[D / (8 * X::NG)];
    if (whole) out_words<D>(st.oacc, qt, l > 0.f ? 1.0f / l : (l == 0.f ? 0.f : l), y);   // a NaN stays one
    if (!row.ok) {
    } else if (whole) {
      uint16_t* dst = io.o + (int64_t)(wk.q.q0 + row.token) * io.o_tok + (int64_t)row.head * io.o_head;
#pragma unroll
      for (int i = 0; i < D / (8 * X::NG); ++i) *(u32x4*)(dst + out_col<D>(i, lg)) = y[i];
      if (io.lse && lg == 0)
        io.lse[(int64_t)(wk.q.q0 + row.token) * g.Hq + row.head] =
            l == 0.f ? -INFINITY : (st.m_run[qt] + log2f(l)) * 0.69314718055994531f;
    } else {
      const size_t prow = (size_t)slot * R + r;
      float* po = io.part_o + prow * D + 4 * lg;
#pragma unroll
      for (int dt = 0; dt < D / X::MR; ++dt) {
        const typename X::Acc x = st.oacc[dt][qt];
#pragma unroll
        for (int i = 0; i < X::AR; i += 4)
          *(f32x4*)(po + X::MR * dt + X::acc_row(i)) = f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]};
      }
      if (lg == 0) {
        io.part_m[prow] = st.m_run[qt];
        io.part_l[prow] = l;
      }
    }
  }
}

struct SeqArgs {
  SeqGeom g;
  SeqIo io;
  CacheGeom cg;
  SeqBias bias;
};

// A wave's relative bias: a table by distance in LDS for each head of the unit, from distance lo - kBiasPad on, so
// that the tiles that need it (near) read it without a clamp; where all distances of a tile are beyond one end the
// bias is one number a row, which the softmax takes as a shift.
template <int D>
struct WaveBias {
  using X = Mma<D>;
  uint32_t at[X::QT];                // index of key 0's distance in the tables, for this lane's first key (mod 2^32)
  int row[X::QT];                    // the row's table
  float lo[X::QT], hi[X::QT];        // beyond the ends
  int first, last;                   // the first and last place of the wave's rows among the keys
};

// Where the wave's rows lie; the tables are whole behind the barrier that follows.
template <int D>
__device__ __forceinline__ void start_bias(WaveBias<D>& wb, const SeqArgs& a, const Walk& wk, int r_off, int c, int lg) {
  using X = Mma<D>;
  const int off = wk.q.lk - wk.q.lq, t0 = wk.b * a.g.TB;
  // the tokens of the wave's 32 rows, as unit_row has them
  const int last = min(a.g.TB, wk.q.lq - t0) - 1;
  wb.first = off + t0 + min((int)(((uint32_t)r_off * (uint32_t)a.g.gh_magic) >> 16), last);
  wb.last = off + t0 + min((int)(((uint32_t)(r_off + 31) * (uint32_t)a.g.gh_magic) >> 16), last);
#pragma unroll
  for (int qt = 0; qt < X::QT; ++qt) {
    const Row row = unit_row(a.g, wk, r_off + X::MR * qt + c);
    const int head = row.ok ? row.head - unit_head0(a.g, wk) : 0;
    // rows that do not exist read the places of one that does
    const int place = row.ok ? row.token + off : wb.first;
    wb.row[qt] = head * kBiasPitch;
    wb.at[qt] = (uint32_t)(wb.row[qt] + 4 * lg + kBiasPad - a.bias.lo) - (uint32_t)place;
  }
}
// The bias beyond the ends, from the tables.
template <int D>
__device__ __forceinline__ void far_bias(WaveBias<D>& wb, const float* table, int distances, float scale_log2) {
#pragma unroll
  for (int qt = 0; qt < Mma<D>::QT; ++qt) {
    wb.lo[qt] = table[wb.row[qt] + kBiasPad] * scale_log2;
    wb.hi[qt] = table[wb.row[qt] + kBiasPad + distances] * scale_log2;
  }
}

// The unit's tables, by all threads.
template <int THREADS>
__device__ __forceinline__ void fill_bias(float (*table)[kBiasPitch], const SeqArgs& a, const Walk& wk) {
  const int heads = unit_heads(a.g, wk), head0 = unit_head0(a.g, wk), n = a.bias.hi - a.bias.lo + 1 + 2 * kBiasPad;
  const float inv = 1.0f / a.io.scale_log2;
  for (int h = 0; h < heads; ++h)
    for (int i = threadIdx.x; i < n; i += THREADS) table[h][i] = bias_log2(a.bias, i - kBiasPad, a.g.Hq, head0 + h) * inv;
}

// The bias of a tile that needs the table, where the logits are added to.
template <int D>
__device__ __forceinline__ void near_bias(const WaveBias<D>& wb, const float* table,
                                          typename Mma<D>::Acc (*sacc)[Mma<D>::QT], int key0) {
  using X = Mma<D>;
#pragma unroll
  for (int qt = 0; qt < X::QT; ++qt) {
    const float* at = table + (int)(wb.at[qt] + (uint32_t)key0);
#pragma unroll
    for (int kt = 0; kt < KT / X::MR; ++kt)
#pragma unroll
      for (int i = 0; i < X::AR; ++i) sacc[kt][qt][i] = at[X::MR * kt + X::acc_row(i)];
  }
}

// The arguments of seq_attn_kernel, read anew: 50 scalar registers that a piece needs at its ends must
// not be held over its loop, which needs nearly all there are.
__device__ __forceinline__ SeqArgs fresh_args() {
  typedef const __attribute__((address_space(4))) SeqArgs CArgs;
  CArgs* p = (CArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const SeqArgs*)p;
}

template <int D, bool CACHE, bool BIAS>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void seq_attn_kernel(SeqArgs) {
  using T = Tile<D>;
  using X = Mma<D>;
  __shared__ __attribute__((aligned(1024))) unsigned char ring[6 * T::BYTES];
  __shared__ float table[BIAS ? kBiasHeads : 1][BIAS ? kBiasPitch : 1];

  // workgroups of one XCD take consecutive stretches: they walk the same head's K and V
  const int P = gridDim.x;
  const int lambda = (blockIdx.x & 7) * (P >> 3) + (blockIdx.x >> 3);
  const int tid = threadIdx.x, lane = tid & 63;
  Walk wk;
  float scale_log2;
  {
    const SeqArgs a = fresh_args();
    if (a.g.cuts && tid == 0) a.io.cut[2 * lambda] = a.io.cut[2 * lambda + 1] = int4{0, 0, 0, 0};
    wk = start_walk<CACHE>(a.g, lambda, P);
    scale_log2 = a.io.scale_log2;
  }
  if (!wk.more()) return;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lw = wave & 3;
  const int c = lane % X::MR, lg = lane / X::MR;
  const int r_off = lw * 64 + (wave >> 2) * QW;      // the two waves of a SIMD: halves of 64 rows

  WaveCtx w;
  w.kbase = c * T::STRIDE + 16 * (lg ^ T::kswz(c));
  {
    const int vrow = 4 * lg + ((lane & 15) >> 2);
    w.vbase = 3 * T::BYTES + vrow * T::STRIDE + 2 * X::MR * T::vswz(vrow) + (X::MR == 32 ? 2 * (lane & 16) : 0) +
              8 * (lane & 3);
  }
  w.g4 = 4 * lg;
  w.scale_log2 = scale_log2;
  PieceState<D> st;
  typename std::conditional<BIAS, WaveBias<D>, int>::type wb;
  int bias_lo = 0, bias_hi = 0, table_head = -1;       // table_head: the first head of the tables in LDS
  if constexpr (BIAS) {
    const SeqArgs a = fresh_args();
    bias_lo = a.bias.lo;
    bias_hi = a.bias.hi;
  }

  // Iteration i of a piece's tiles (phases as in attn.hip): tile i lies in stage i % 3.  Group 0
  // loads K(i + 2) and group 1 V(i + 1) at the end of their V phases, and both wait at the end of
  // the iteration for what they issued in the one before.
  auto run = [&](auto G1) {
    constexpr bool IS_G1 = decltype(G1)::value;
    constexpr int VOFF = 3 * T::BYTES;
    typename std::conditional<CACHE, CacheTiles<D, IS_G1>, RowTiles<D, IS_G1>>::type src;
    {
      const SeqArgs a = fresh_args();
      src.init(a.io, a.cg, lw, lane);
    }
    unsigned char* const s0 = ring;
    unsigned char* const s1 = ring + T::BYTES;
    unsigned char* const s2 = ring + 2 * T::BYTES;
    while (wk.more()) {
      uint64_t unit_end;
      Piece pc;
      {
        const SeqArgs a = fresh_args();
        pc = walk_piece(a.g, wk, &unit_end);
      }
      const int N = pc.tb - pc.ta;
      if (N > 0) {
        int key_open;                                 // first tile that some row of the unit does not see whole
        {
          const SeqArgs a = fresh_args();
          src.prime(a.io, wk, wk.kvh, pc.ta, pc.tb, IS_G1 ? s0 + VOFF : s0, IS_G1 ? nullptr : s1);
          start_rows<D>(st, w, a.g, a.io, wk, r_off, c, lg);
          if constexpr (BIAS) {
            // consecutive units mostly have the same heads; the waves read no table of the piece before any more, as
            // its last iteration ended with a barrier
            const int heads = unit_head0(a.g, wk);
            if (heads != table_head) fill_bias<kThreads>(table, a, wk);
            table_head = heads;
            start_bias<D>(wb, a, wk, r_off, c, lg);
          }
          const int open = a.g.causal ? max(0, wk.q.lk - wk.q.lq + wk.b * a.g.TB + 1) : wk.q.lk;
          key_open = min(open, wk.q.lk) - 63;
        }
        __builtin_amdgcn_s_waitcnt(0);
        phase_barrier();
        if constexpr (BIAS) far_bias<D>(wb, &table[0][0], bias_hi - bias_lo, w.scale_log2);
        auto m_phase = [&](int i, const unsigned char* kcur, const unsigned char* vprev) {
          const int key0 = 64 * (pc.ta + i);
          if (i > 0 && key0 - 64 < st.seen) pv_tile<D>(vprev, st.pb, st.oacc, w.vbase);
          if (i < N && key0 < st.seen) {
            if constexpr (BIAS) {
              if (key0 + 63 - wb.first > bias_lo && key0 - wb.last < bias_hi) {
                near_bias<D>(wb, &table[0][0], st.sacc, key0);
                qk_tile<D, true>(kcur, st.qreg, st.sacc, w.kbase);
              } else {
                qk_tile<D>(kcur, st.qreg, st.sacc, w.kbase);
              }
            } else {
              qk_tile<D>(kcur, st.qreg, st.sacc, w.kbase);
            }
          }
        };
        auto v_phase = [&](int i) {
          const int key0 = 64 * (pc.ta + i);
          if (i >= 0 && i < N && key0 < st.seen) {
            if constexpr (BIAS) {
              const bool left = key0 + 63 - wb.first <= bias_lo, right = key0 - wb.last >= bias_hi;
              float shift[X::QT];
#pragma unroll
              for (int qt = 0; qt < X::QT; ++qt) {
                const float lo = wb.lo[qt], hi = wb.hi[qt];
                shift[qt] = left ? lo : (right ? hi : 0.f);
              }
              if (__builtin_expect(key0 >= key_open, 0)) mask_tile<D>(st.sacc, key0, 0, w);
              softmax_tile<D, true>(st.sacc, st.pb, st.oacc, st.m_run, st.l_run, w.scale_log2, shift);
            } else {
              if (__builtin_expect(key0 >= key_open, 0)) mask_tile<D>(st.sacc, key0, 0, w);
              softmax_tile<D>(st.sacc, st.pb, st.oacc, st.m_run, st.l_run, w.scale_log2);
            }
          }
        };
        auto iteration = [&](int i, unsigned char* sc, unsigned char* sp, unsigned char* sn) {
          if constexpr (!IS_G1) {
            m_phase(i, sc, sp);
            phase_barrier();
            v_phase(i);
            src.issue(sp);
          } else {
            v_phase(i - 1);
            src.issue(sn + VOFF);
            phase_barrier();
            m_phase(i, sc, sp);
          }
          src.wait();
          phase_barrier();
        };
        for (int i = 0;; i += 3) {
          iteration(i, s0, s2, s1);
          if (i + 1 > N) break;
          iteration(i + 1, s1, s0, s2);
          if (i + 2 > N) break;
          iteration(i + 2, s2, s1, s0);
          if (i + 3 > N) break;
        }
        const SeqArgs a = fresh_args();
        end_rows<D>(st, a.g, a.io, wk, pc, 2 * lambda, r_off, c, lg);
        // the loads behind the piece have landed before the next one's (or the end of the workgroup)
        __builtin_amdgcn_s_waitcnt(0);
      }
      const SeqArgs a = fresh_args();
      walk_on<CACHE>(a.g, wk, unit_end);
    }
  };
  if (wave >= 4) run(std::true_type{});
  else run(std::false_type{});
}

// The same with a bias for units of 128 rows: four waves of 32 rows and two stages of tiles, two workgroups to a CU,
// which cover each other's starts and ends, and a softmax by the other's products, without taking turns.  For short
// sequences (prompt_plan): 16 of 60 to 512 tokens, 16 heads, d 64, 21 us where units of 256 rows take 28.5, the
// next token of 8 over 500 to 1000 keys 13 instead of 17.  Long ones are 6 to 9 % faster by the larger units.
constexpr int kBiasThreads = 256;
template <int D>
__global__ __launch_bounds__(kBiasThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void bias_rows_kernel(SeqArgs) {
  using T = Tile<D>;
  using X = Mma<D>;
  __shared__ __attribute__((aligned(1024))) unsigned char ring[4 * T::BYTES];     // K of two stages, V of two
  __shared__ float table[kBiasHeads][kBiasPitch];
  const int P = gridDim.x;
  const int lambda = (blockIdx.x & 7) * (P >> 3) + (blockIdx.x >> 3);
  const int tid = threadIdx.x, lane = tid & 63;
  const int lw = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane % X::MR, lg = lane / X::MR;
  const int r_off = lw * QW;
  Walk wk;
  WaveCtx w;
  RowTiles<D, false> ks;
  RowTiles<D, true> vs;
  int bias_lo, bias_hi;
  {
    const SeqArgs a = fresh_args();
    if (a.g.cuts && tid == 0) a.io.cut[2 * lambda] = a.io.cut[2 * lambda + 1] = int4{0, 0, 0, 0};
    wk = start_walk<false>(a.g, lambda, P);
    if (!wk.more()) return;
    w.scale_log2 = a.io.scale_log2;
    bias_lo = a.bias.lo;
    bias_hi = a.bias.hi;
    ks.init(a.io, a.cg, lw, lane);
    vs.init(a.io, a.cg, lw, lane);
  }
  w.kbase = c * T::STRIDE + 16 * (lg ^ T::kswz(c));
  {
    const int vrow = 4 * lg + ((lane & 15) >> 2);
    w.vbase = vrow * T::STRIDE + 2 * X::MR * T::vswz(vrow) + (X::MR == 32 ? 2 * (lane & 16) : 0) + 8 * (lane & 3);
  }
  w.g4 = 4 * lg;
  PieceState<D> st;
  WaveBias<D> wb;
  int table_head = -1;
  while (wk.more()) {
    uint64_t unit_end;
    Piece pc;
    {
      const SeqArgs a = fresh_args();
      pc = walk_piece(a.g, wk, &unit_end);
    }
    const int N = pc.tb - pc.ta;
    if (N > 0) {
      int key_open;
      phase_barrier();                                 // the piece before is read
      {
        const SeqArgs a = fresh_args();
        ks.prime(a.io, wk, wk.kvh, pc.ta, pc.tb, ring, nullptr);
        vs.prime(a.io, wk, wk.kvh, pc.ta, pc.tb, ring + 2 * T::BYTES, nullptr);
        start_rows<D>(st, w, a.g, a.io, wk, r_off, c, lg);
        const int heads = unit_head0(a.g, wk);
        if (heads != table_head) fill_bias<kBiasThreads>(table, a, wk);
        table_head = heads;
        start_bias<D>(wb, a, wk, r_off, c, lg);
        const int open = a.g.causal ? max(0, wk.q.lk - wk.q.lq + wk.b * a.g.TB + 1) : wk.q.lk;
        key_open = min(open, wk.q.lk) - 63;
      }
      for (int i = 0; i < N; ++i) {
        __builtin_amdgcn_s_waitcnt(0);
        phase_barrier();
        if (i == 0) far_bias<D>(wb, &table[0][0], bias_hi - bias_lo, w.scale_log2);
        const unsigned char* kt = ring + (i & 1) * T::BYTES;
        const unsigned char* vt = kt + 2 * T::BYTES;
        if (i + 1 < N) {
          ks.issue(ring + (~i & 1) * T::BYTES);
          vs.issue(ring + (2 + (~i & 1)) * T::BYTES);
        }
        const int key0 = 64 * (pc.ta + i);
        if (key0 >= st.seen) continue;
        const bool left = key0 + 63 - wb.first <= bias_lo, right = key0 - wb.last >= bias_hi;
        if (!left && !right) {
          near_bias<D>(wb, &table[0][0], st.sacc, key0);
          qk_tile<D, true>(kt, st.qreg, st.sacc, w.kbase);
        } else {
          qk_tile<D>(kt, st.qreg, st.sacc, w.kbase);
        }
        float shift[X::QT];
#pragma unroll
        for (int qt = 0; qt < X::QT; ++qt) {
          const float lo = wb.lo[qt], hi = wb.hi[qt];
          shift[qt] = left ? lo : (right ? hi : 0.f);
        }
        if (__builtin_expect(key0 >= key_open, 0)) mask_tile<D>(st.sacc, key0, 0, w);
        softmax_tile<D, true>(st.sacc, st.pb, st.oacc, st.m_run, st.l_run, w.scale_log2, shift);
        pv_tile<D>(vt, st.pb, st.oacc, w.vbase);
      }
      const SeqArgs a = fresh_args();
      end_rows<D, kBiasRows>(st, a.g, a.io, wk, pc, 2 * lambda, r_off, c, lg);
    }
    const SeqArgs a = fresh_args();
    walk_on<false>(a.g, wk, unit_end);
  }
}

// Joins the pieces of a unit that several stretches share: o = sum 2^(m_s - m) O_s / sum 2^(m_s - m) l_s,
// over the pieces in the order of the stretches.  Workgroup (l, y) joins rows [RW y, RW y + RW) of
// the unit that stretch l starts and does not end, if there is one: its first piece lies in slot
// 2 l + 1, the others in the slots 2 l' of the stretches that follow.
// A unit of few rows is often one of many pieces (a long cache): NG groups of 256 threads take every
// NG-th batch of them and are joined in LDS.
template <int D, int R, int RW, int NG>
__global__ __launch_bounds__(256 * NG) void seq_merge_kernel(SeqIo io, int GH, int Hq, int P) {
  constexpr int TPR = 256 / RW;                       // threads of a row
  constexpr int W = D / TPR;
  const int l0 = blockIdx.x;
  const int lane = threadIdx.x & 63;
  const int4 u = io.cut[2 * l0 + 1];
  const int4 x0 = io.cut[2 * min(l0 + 1 + lane, P - 1)];
  if (u.w == 0) return;
  // pieces that follow: as long as slot 2 l' names the same unit
  int n = 0;
  for (;;) {
    const int l = l0 + 1 + n + lane;
    const int4 x = n == 0 ? x0 : io.cut[2 * min(l, P - 1)];
    const uint64_t other = ~__ballot(l < P && x.w != 0 && x.x == u.x && x.z == u.z);
    if (other) {
      n += __builtin_ctzll(other);
      break;
    }
    n += 64;
  }
  const int th = threadIdx.x & 255, grp = threadIdx.x >> 8;
  const int r = blockIdx.y * RW + th / TPR, part = th % TPR;
  const int token = r / GH, head = r - token * GH;    // as unit_row
  const bool ok = token < u.y && head < u.w;
  float m = -INFINITY, l = 0.f, acc[W];
#pragma unroll
  for (int e = 0; e < W; ++e) acc[e] = 0.f;
  constexpr int BATCH = 4;
  for (int i0 = grp * BATCH; i0 <= n && ok; i0 += NG * BATCH) {
    float pm[BATCH], pl[BATCH];
    f32x4 po[BATCH][W / 4];
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      const int i = min(i0 + j, n);                   // a repeated piece is left out below
      const size_t at = (size_t)(i == 0 ? 2 * l0 + 1 : 2 * (l0 + i)) * R + r;
      pm[j] = io.part_m[at];
      pl[j] = io.part_l[at];
#pragma unroll
      for (int e = 0; e < W / 4; ++e) po[j][e] = *(const f32x4*)(io.part_o + at * D + part * W + 4 * e);
    }
    float mx = m;
#pragma unroll
    for (int j = 0; j < BATCH; ++j) mx = fmaxf(mx, pm[j]);
    const float base = mx == -INFINITY ? 0.f : mx;
    const float keep = exp2f(m - base);
    l *= keep;
#pragma unroll
    for (int e = 0; e < W; ++e) acc[e] *= keep;
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      if (i0 + j > n) break;
      const float a = exp2f(pm[j] - base);
      l += a * pl[j];
#pragma unroll
      for (int e = 0; e < W; ++e) acc[e] += a * po[j][e / 4][e % 4];
    }
    m = mx;
  }
  if constexpr (NG > 1) {
    __shared__ float sm[NG - 1][256][W + 3];          // W + 2 values; the row stride is odd
    if (grp > 0) {
      float* p = sm[grp - 1][th];
#pragma unroll
      for (int e = 0; e < W; ++e) p[e] = acc[e];
      p[W] = m;
      p[W + 1] = l;
    }
    __syncthreads();
    if (grp > 0) return;
    float mx = m;
#pragma unroll
    for (int k = 0; k < NG - 1; ++k) mx = fmaxf(mx, sm[k][th][W]);
    const float base = mx == -INFINITY ? 0.f : mx;
    const float keep = exp2f(m - base);
    l *= keep;
#pragma unroll
    for (int e = 0; e < W; ++e) acc[e] *= keep;
#pragma unroll
    for (int k = 0; k < NG - 1; ++k) {
      const float* p = sm[k][th];
      const float a = exp2f(p[W] - base);
      l += a * p[W + 1];
#pragma unroll
      for (int e = 0; e < W; ++e) acc[e] += a * p[e];
    }
    m = mx;
  }
  if (!ok) return;
  const float inv = l > 0.f ? 1.0f / l : (l == 0.f ? 0.f : l);
  uint16_t* dst = io.o + (int64_t)(u.x + token) * io.o_tok + (int64_t)(u.z + head) * io.o_head + part * W;
  uint32_t y[W / 2];
#pragma unroll
  for (int e = 0; e < W / 2; ++e) y[e] = pack_bf16x2(acc[2 * e] * inv, acc[2 * e + 1] * inv);
#pragma unroll
  for (int e = 0; e < W / 4; ++e) *(u32x2*)(dst + 4 * e) = u32x2{y[2 * e], y[2 * e + 1]};
  if (io.lse && part == 0)
    io.lse[(int64_t)(u.x + token) * Hq + u.z + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

template <int D, int R>
void launch_merge(const SeqGeom& g, const SeqIo& io, int P, hipStream_t st) {
  constexpr int RW = R == 32 ? 32 : 16, NG = R <= 32 ? 4 : 1;
  hipLaunchKernelGGL((seq_merge_kernel<D, R, RW, NG>), dim3(P, R / RW), dim3(256 * NG), 0, st, io, g.GH, g.Hq, P);
}

}  // namespace

template <int D, bool CACHE, bool BIAS = false>
static hipError_t launch_rows(const SeqGeom& g, const SeqIo& io, const CacheGeom& cg, int P, hipStream_t st,
                              const SeqBias& bias = SeqBias{}) {
  hipLaunchKernelGGL((seq_attn_kernel<D, CACHE, BIAS>), dim3(P), dim3(kThreads), 0, st, SeqArgs{g, io, cg, bias});
  if (g.cuts) launch_merge<D, QR>(g, io, P, st);
  return hipGetLastError();
}

template <int D>
static hipError_t launch_bias_rows(const SeqGeom& g, const SeqIo& io, const SeqBias& bias, int P, hipStream_t st) {
  hipLaunchKernelGGL((bias_rows_kernel<D>), dim3(P), dim3(kBiasThreads), 0, st, SeqArgs{g, io, CacheGeom{}, bias});
  if (g.cuts) launch_merge<D, kBiasRows>(g, io, P, st);
  return hipGetLastError();
}

hipError_t launch_prompt_attn(const SeqGeom& g, const SeqIo& io, const SeqBias* bias, int d, int rows, int P,
                              hipStream_t st) {
  const CacheGeom none{};
  if (bias && rows == kBiasRows)
    return d == 128 ? launch_bias_rows<128>(g, io, *bias, P, st) : launch_bias_rows<64>(g, io, *bias, P, st);
  if (bias)
    return d == 128 ? launch_rows<128, false, true>(g, io, none, P, st, *bias)
                    : launch_rows<64, false, true>(g, io, none, P, st, *bias);
  return d == 128 ? launch_rows<128, false>(g, io, none, P, st) : launch_rows<64, false>(g, io, none, P, st);
}

hipError_t launch_cache_merge(const SeqGeom& g, const SeqIo& io, int d, int rows, int P, hipStream_t st) {
  if (d == 128) rows == 16 ? launch_merge<128, 16>(g, io, P, st) : launch_merge<128, 32>(g, io, P, st);
  else rows == 16 ? launch_merge<64, 16>(g, io, P, st) : launch_merge<64, 32>(g, io, P, st);
  return hipGetLastError();
}

hipError_t launch_cache_rows(const SeqGeom& g, const SeqIo& io, const CacheGeom& cg, int d, int P, hipStream_t st) {
  return d == 128 ? launch_rows<128, true>(g, io, cg, P, st) : launch_rows<64, true>(g, io, cg, P, st);
}

}  // namespace la
