// Gradients of the attention over packed sequences on gfx950, with recomputed probabilities.
//
// With x = scale q.k (+ bias), P = exp(x - lse), delta = do.o (- dlse), dP = do.v:
//   dS = P (dP - delta);  dV = P^T dO;  dK = scale dS^T Q;  dQ = scale dS K
// and the gradient of a bucket of the relative bias is the sum of dS over its pairs.
//
// Two walks over the pairs, so that no sum needs atomics and results repeat bit for bit: key_grad holds 128 keys of a
// key head and goes over the queries that see them (four products, dK and dV in registers), row_grad holds 128 packed
// query rows and goes over their keys (three, dQ in registers).  Seven products instead of five: dQ summed from the
// first walk would be one fp32 row for each of a head's runs of keys, and dS stored for a product of its own 2 bytes a
// pair, both more time in memory than the two products take.  Of a workgroup's four waves each has 32 of the 128 rows;
// two workgroups run on a CU, one of each walk, so that one's exponentials lie under the other's products without a
// barrier between them.  S and dP of a tile stay in registers, as they lie in them they are the operands of the
// products that follow; Q and dO, or K and V, come by asynchronous loads into two stages of LDS, one barrier a tile.
//
// P and dS are rounded to bf16 (by at most 2^-8 of themselves) as operands, which run at 16 times fp32's rate; dS is
// formed from P before its rounding, and the bias' gradient sums it unrounded.  Relative rms error against 64 bits
// 0.0024, of which the result's own rounding makes 0.0017.
//
// Bound, where sequences are long, by the card's power: 8192 causal tokens, 16 heads over 4, d 128, take 780 to
// 800 us from card to card, 1.20 to 1.23 PFLOP/s over seven products (0.86 to 0.88 over the five that are needed) where a
// large bf16 product of random data reaches 1.35 to 1.38 (the matrix pipeline is 54 % busy, as it is there); half the vector instructions in the
// loops, or fewer LDS conflicts, moved it by 1 to 3 %.  d 64 does the same vector work for half the products: 468 us,
// 1.03 PFLOP/s.  Short sequences: a unit costs 3.5 us beside its tiles (Q, dO or K, V, the first tile, the results), a
// tile of 64 by 128 pairs 2.1 us where two walks share a CU, and the start (finding the stretch) 2.5: 48 prompts of 1
// to 300 tokens, 16 heads over 4, d 64, 26 us.
#include <limits.h>
#include <math.h>

#include <type_traits>

#include "attn_core.h"
#include "grad_walk.h"

namespace la {
namespace {

// four words at any word's address
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

constexpr int kGradThreads = 256;        // four waves, each with 32 of a unit's 128 rows

// A tile of ROWS rows of D bf16 in LDS that is read both ways: as operands along d (16 bytes of MR rows) and
// transposed, as operands along the rows (chunks of 2 MR bytes of 4 rows a lane group).  The 16-byte slots of
// row r are permuted by an exclusive or with swz(r), for which both spread over all 64 banks.  (A 16-byte read takes
// lanes 0-3, 12-15 and 20-27 at once, then 4-11, 16-19 and 28-31, and so on: rows r and r + 8 of one 16-lane group
// never meet, so that three bits do.  With the row's fourth bit as the lowest there are 0.59 conflicts an access and
// 3 % more time.)
template <int D, int ROWS>
struct GradTile {
  static constexpr int STRIDE = D * 2;
  static constexpr int SLOTS = STRIDE / 16;
  static constexpr int BYTES = ROWS * STRIDE;
  static constexpr int PER = BYTES / 4096;             // 1 KiB loads of each of the four waves
  __device__ static constexpr int swz(int r) {
    return D == 128 ? (r & 7) << 1 : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
  }
};

// Global byte offset of lane `lane` of the i-th load of wave lw, less the immediate 1024 i (see slot_offset).
template <int D, int ROWS>
__device__ __forceinline__ uint32_t grad_slot(int lw, int i, int lane, uint32_t stride) {
  using T = GradTile<D, ROWS>;
  const int slot = 64 * i + lane;
  const int row = lw * (ROWS / 4) + slot / T::SLOTS;
  return (uint32_t)row * stride + (uint32_t)(((slot % T::SLOTS) ^ T::swz(row)) * 16 - 1024 * i);
}

// Asynchronous load of a wave's quarter of a tile; rows past nrec bytes come as zeros.
template <int D, int ROWS>
__device__ __forceinline__ void grad_issue(unsigned char* dst, const uint16_t* base, uint64_t off, uint32_t nrec,
                                           const uint32_t* lane_off) {
  // attn_core.h's, of as many bytes: 128 or 64 values a row stand for four or two loads
  issue_tile<GradTile<D, ROWS>::PER == 4 ? 128 : 64>(dst, base, off, nrec, lane_off);
}

// Asynchronous load of the statistics of up to 64 rows, by one wave: 16 bytes a lane, of which those behind nrec come
// as zeros, as does the second KiB.
constexpr int kStatBytes = 2048;
__device__ __forceinline__ void stat_issue(unsigned char* dst, const float2* base, uint64_t off, uint32_t nrec, int lane) {
  const uint32_t lane_off[2] = {16u * lane, 16u * lane};
  issue_tile<64>(dst, (const uint16_t*)base, off, nrec, lane_off);
}

// acc[t][c] = A B: A the first NT MR rows of a tile, B columns of the other operand in registers.
template <int D, int NT>
__device__ __forceinline__ void rows_product(const unsigned char* __restrict__ tile, const bf16x8 (*b)[Mma<D>::QT],
                                             typename Mma<D>::Acc (*acc)[Mma<D>::QT], int base) {
  using X = Mma<D>;
  constexpr int NO = NT * (D / X::KC);
  constexpr int AHEAD = NO < 4 ? NO : 4;
  bf16x8 a[NO];
#pragma unroll
  for (int i = 0; i < NO; ++i)
    a[i] = *(const bf16x8*)(tile + (base ^ (16 * X::NG * (i / NT))) + (i % NT) * X::MR * (2 * D));
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int c = 0; c < X::QT; ++c)
#pragma unroll
      for (int i = 0; i < X::AR; ++i) acc[t][c][i] = 0.f;
#pragma unroll
  for (int i = 0; i < NO; ++i)
#pragma unroll
    for (int c = 0; c < X::QT; ++c) acc[i % NT][c] = X::mma(a[i], b[i / NT][c], acc[i % NT][c]);
  __builtin_amdgcn_sched_group_barrier(kSgDsRead, AHEAD, 0);
#pragma unroll
  for (int i = 0; i < NO - AHEAD; ++i) {
    __builtin_amdgcn_sched_group_barrier(kSgMfma, X::QT, 0);
    __builtin_amdgcn_sched_group_barrier(kSgDsRead, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(kSgMfma, X::QT * AHEAD, 0);
}

// The same with B in LDS too, rows of `other` at bbase (32 of them, column c MR of the product).
template <int D, int NT>
__device__ __forceinline__ void tiles_product(const unsigned char* __restrict__ tile,
                                              const unsigned char* __restrict__ other,
                                              typename Mma<D>::Acc (*acc)[Mma<D>::QT], int base, int bbase) {
  using X = Mma<D>;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int c = 0; c < X::QT; ++c)
#pragma unroll
      for (int i = 0; i < X::AR; ++i) acc[t][c][i] = 0.f;
#pragma unroll
  for (int ks = 0; ks < D / X::KC; ++ks) {
    bf16x8 a[NT], b[X::QT];
#pragma unroll
    for (int c = 0; c < X::QT; ++c)
      b[c] = *(const bf16x8*)(other + (bbase ^ (16 * X::NG * ks)) + c * X::MR * (2 * D));
#pragma unroll
    for (int t = 0; t < NT; ++t) a[t] = *(const bf16x8*)(tile + (base ^ (16 * X::NG * ks)) + t * X::MR * (2 * D));
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int c = 0; c < X::QT; ++c) acc[t][c] = X::mma(a[t], b[c], acc[t][c]);
  }
}

// acc[dt][c] += A^T B over the rows of a tile: NS steps of KC rows, B columns [step][c] in registers, whose
// slot e of lane group g is row 4 g + e (e < 4) or KC / 2 + 4 g + e - 4 of the step, as accumulators lie.
template <int D, int NS>
__device__ __forceinline__ void columns_product(const unsigned char* __restrict__ tile, const bf16x8 (*b)[Mma<D>::QT],
                                                typename Mma<D>::Acc (*acc)[Mma<D>::QT], int base) {
  using X = Mma<D>;
  constexpr int DT = D / X::MR;
  constexpr int NO = NS * DT;
  constexpr int AHEAD = NO < 3 ? NO : (X::MR == 16 ? 3 : 2);
  // KC / 2 rows on, the permutation of d 128 is the same, that of d 64 (8 rows) differs by 2
  constexpr int HI = X::MR == 16 ? 0 : 32;
  bf16x8 a[NO];
#pragma unroll
  for (int i = 0; i < NO; ++i) {
    const int at = base ^ (2 * X::MR * (i % DT));
    const unsigned char* p = tile + (X::KC * (i / DT)) * (2 * D);
    const v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS v4i16*)(p + at));
    const v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS v4i16*)(p + (at ^ HI) + X::KC / 2 * (2 * D)));
    const v8i16 a8 = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    a[i] = __builtin_bit_cast(bf16x8, a8);
  }
#pragma unroll
  for (int i = 0; i < NO; ++i)
#pragma unroll
    for (int c = 0; c < X::QT; ++c) acc[i % DT][c] = X::mma(a[i], b[i / DT][c], acc[i % DT][c]);
  __builtin_amdgcn_sched_group_barrier(kSgDsRead, 2 * AHEAD, 0);
#pragma unroll
  for (int i = 0; i < NO - AHEAD; ++i) {
    __builtin_amdgcn_sched_group_barrier(kSgMfma, X::QT, 0);
    __builtin_amdgcn_sched_group_barrier(kSgDsRead, 2, 0);
  }
  __builtin_amdgcn_sched_group_barrier(kSgMfma, X::QT * AHEAD, 0);
}

// Bases of this lane for the two ways of reading a tile.
template <int D>
__device__ __forceinline__ int rows_base(int lane) {
  using X = Mma<D>;
  const int c = lane % X::MR, lg = lane / X::MR;
  return c * (2 * D) + 16 * (lg ^ GradTile<D, 64>::swz(c));
}
template <int D>
__device__ __forceinline__ int columns_base(int lane) {
  using X = Mma<D>;
  const int row = 4 * (lane / X::MR) + ((lane & 15) >> 2);
  const int slot = (X::MR == 32 ? 2 * ((lane >> 4) & 1) : 0) + ((lane & 3) >> 1);
  return row * (2 * D) + 16 * (slot ^ GradTile<D, 64>::swz(row)) + 8 * (lane & 1);
}

// Two products' accumulators of a step of KC rows as one bf16 operand: element e of the lane's 8.
template <int D, int NT>
__device__ __forceinline__ void as_operand(const typename Mma<D>::Acc (*acc)[Mma<D>::QT], bf16x8 (*b)[Mma<D>::QT]) {
  using X = Mma<D>;
#pragma unroll
  for (int s = 0; s < NT * X::MR / X::KC; ++s)
#pragma unroll
    for (int c = 0; c < X::QT; ++c) {
      u32x4 w;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int e = 8 * s + 2 * j;
        w[j] = pack_bf16x2(acc[e / X::AR][c][e % X::AR], acc[e / X::AR][c][e % X::AR + 1]);
      }
      b[s][c] = __builtin_bit_cast(bf16x8, w);
    }
}

// A wave's 32 rows of a result as bf16 (column c of `acc` is row MR c + lane % MR), or their fp32 partial sums.
template <int D>
__device__ __forceinline__ void store_rows(const typename Mma<D>::Acc (*acc)[Mma<D>::QT], int c, float factor, bool ok,
                                           uint16_t* dst, int lg) {
  using X = Mma<D>;
  u32x4 y[D / (8 * X::NG)];
  out_words<D>(acc, c, factor, y);
  if (!ok) return;
#pragma unroll
  for (int i = 0; i < D / (8 * X::NG); ++i) *(u32x4*)(dst + out_col<D>(i, lg)) = y[i];
}
template <int D>
__device__ __forceinline__ void store_part(const typename Mma<D>::Acc (*acc)[Mma<D>::QT], int c, float* dst, int lg) {
  using X = Mma<D>;
#pragma unroll
  for (int dt = 0; dt < D / X::MR; ++dt)
#pragma unroll
    for (int i = 0; i < X::AR; i += 4)
      *(f32x4*)(dst + X::MR * dt + X::acc_row(i) + 4 * lg) =
          f32x4{acc[dt][c][i], acc[dt][c][i + 1], acc[dt][c][i + 2], acc[dt][c][i + 3]};
}

struct GradArgs {
  GradGeom g;
  GradIo io;
  int P;                   // workgroups
};
struct GradBoth {
  GradArgs keys, rows;
};

// The arguments, read anew: the scalar registers that a unit needs at its ends must not be held over its loop.
template <bool KEYS>
__device__ __forceinline__ GradArgs grad_args() {
  typedef const __attribute__((address_space(4))) GradBoth CArgs;
  CArgs* p = (CArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return KEYS ? ((const GradBoth*)p)->keys : ((const GradBoth*)p)->rows;
}

// How the bias enters a wave's tile of pairs: every pair by its distance, or one number for all.
struct FarBias {
  int lo, hi;              // the first and last distance of the table
  float at_lo, at_hi;      // the bias there and beyond
  bool hides;              // some distance's bias is -inf
};
struct TileBias {
  bool near;
  float far;
};
__device__ __forceinline__ void far_bias(FarBias& b, const float* table) {
  b.at_lo = table[kBiasPad];
  b.at_hi = table[kBiasPad + b.hi - b.lo];
  b.hides = __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, table[0])) != 0;
}
__device__ __forceinline__ TileBias tile_bias(const FarBias& b, int least, int most) {
  if (most <= b.lo) return TileBias{false, b.at_lo};
  if (least >= b.hi) return TileBias{false, b.at_hi};
  return TileBias{true, 0.f};
}

// The compiler moves no access to LDS across (a wave's own come in order).
__device__ __forceinline__ void lds_order() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

// ------------------------------------------------------------------------------------------------
// dK and dV

template <int D>
constexpr int key_lds() {
  return 4 * 64 * 128 + 2 * GradTile<D, 64>::BYTES + 2 * kStatBytes;
}

// ROTATE: a unit's inner tiles start where those of the workgroups beside it are.  Bound by power and the products (see
// above); what it reads beside them is a tile of Q and dO for 128 keys, 16 KB for 4.2 MFLOP at d 128, which the L2
// has to serve: without a mask all units are alike, and with the walks out of step a 480P chunk over its context (16
// heads) read 8.6 GB from beyond the L2, in step 2.0.
template <int D, bool BIAS, bool ROTATE>
__device__ __forceinline__ void key_grad(unsigned char* lds, int block, int P) {
  using X = Mma<D>;
  constexpr int QT = D == 128 ? 32 : 64;               // query rows of a tile
  using T = GradTile<D, QT>;
  using TV = GradTile<D, 64>;
  constexpr int NT = QT / X::MR;
  static_assert(T::BYTES == 64 * 128);
  unsigned char* const ring = lds;                     // Q, dO of two stages
  unsigned char* const vtile = lds + 4 * T::BYTES;
  unsigned char* const stat = vtile + 2 * TV::BYTES;
  const int l = (block & 7) * (P >> 3) + (block >> 3);
  const int tid = threadIdx.x, lane = tid & 63;
  const int lw = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane % X::MR, lg = lane / X::MR;
  const int rbase = rows_base<D>(lane), cbase = columns_base<D>(lane);
  GradWalk wk;
  float scale_log2;
  uint32_t q_stride, do_stride;
  uint32_t q_off[T::PER], do_off[T::PER];
  FarBias far{0, 0, 0.f, 0.f, false};
  {
    const GradArgs a = grad_args<true>();
    if (a.g.cuts && tid == 0) a.io.cut[2 * l] = a.io.cut[2 * l + 1] = int4{0, 0, 0, 0};
    uint64_t share;
    wk = grad_start<QT>(a.g, l, P, &share);
    if (!wk.more()) return;
    scale_log2 = a.io.scale_log2;
    q_stride = (uint32_t)a.io.q_tok * 2u;
    do_stride = (uint32_t)a.io.do_tok * 2u;
    if constexpr (BIAS) {
      far.lo = a.io.bias_lo;
      far.hi = a.io.bias_hi;
    }
#pragma unroll
    for (int i = 0; i < T::PER; ++i) {
      q_off[i] = grad_slot<D, QT>(lw, i, lane, q_stride);
      do_off[i] = grad_slot<D, QT>(lw, i, lane, do_stride);
    }
  }
  const int w0 = 32 * lw;                              // the wave's first key of the unit
  uint32_t done = 0;                                   // tiles so far
  typename X::Acc dk[D / X::MR][X::QT], dv[D / X::MR][X::QT];
  bf16x8 kreg[D / X::KC][X::QT];

  while (wk.more()) {
    uint64_t unit_end;
    GradPiece pc;
    {
      const GradArgs a = grad_args<true>();
      pc = grad_piece<QT>(a.g, wk, &unit_end);
    }
    if (pc.tb > pc.ta) {
      const int lq = wk.q.lq, off = wk.q.lk - wk.q.lq;
      const int key0 = wk.b * kGradRows + w0;          // the wave's first key
      const int seen = __builtin_amdgcn_readfirstlane((int)(grad_seen(wk.line, wk.b) / QT));
      const int first = (lq + QT - 1) / QT - seen;     // first query tile that sees a key of the unit
      // the inner tiles are the `seen` tiles of each head in turn, from `begin` to the piece's end and then from its
      // start: workgroups that walk the same queries read the same tiles at the same time
      int64_t left = seen == 0 ? 0 : pc.tb - pc.ta;
      int64_t begin = pc.ta;
      if (ROTATE && left > 0 && left < (1 << 30)) {
        const int nq = seen + first;
        const uint64_t at = (uint64_t)done % ((uint64_t)nq * wk.line.mult);
        const int64_t i = (int64_t)(at / (uint32_t)nq) * seen + max((int)(at % (uint32_t)nq) - first, 0);
        if (i >= pc.ta && i < pc.tb) begin = i;
        done += (uint32_t)left;
      }
      const int seen1 = max(seen, 1);
      int head = __builtin_amdgcn_readfirstlane((int)(begin / seen1));              // of the present tile
      int tile = __builtin_amdgcn_readfirstlane((int)(begin % seen1));
      int to_end = begin == pc.ta ? 0 : (int)(pc.tb - begin);      // tiles to load before the piece's start, if that is due
      // the tile to load next, and where its rows are
      int next_head = head, next_tile = tile;
      uint64_t next_q, next_do, next_stat;
      auto seek = [&]() {
        const GradArgs a = grad_args<true>();
        const int64_t tok = (int64_t)wk.q.q0 + (first + next_tile) * QT;
        const int qh = wk.h * a.g.G + next_head;
        next_q = first_lane_u64((uint64_t)(uintptr_t)a.io.q + (uint64_t)(tok * a.io.q_tok + qh * a.io.q_head) * 2u);
        next_do = first_lane_u64((uint64_t)(uintptr_t)a.io.dout + (uint64_t)(tok * a.io.do_tok + qh * a.io.do_head) * 2u);
        next_stat = first_lane_u64((uint64_t)(uintptr_t)a.io.stat + ((uint64_t)qh * (uint32_t)a.g.Tq + (uint64_t)tok) * 8u);
      };
      auto issue = [&](int st) {
        const uint32_t rows = (uint32_t)min(lq - (first + next_tile) * QT, QT);
        unsigned char* dst = ring + st * (2 * T::BYTES) + lw * (T::BYTES / 4);
        grad_issue<D, QT>(dst, nullptr, first_lane_u64(next_q), __builtin_amdgcn_readfirstlane(rows * q_stride), q_off);
        grad_issue<D, QT>(dst + T::BYTES, nullptr, first_lane_u64(next_do),
                          __builtin_amdgcn_readfirstlane(rows * do_stride), do_off);
        // whole words of 16 bytes: the row behind an odd number of them is masked
        if (lw == 0)
          stat_issue(stat + st * kStatBytes, nullptr, first_lane_u64(next_stat),
                     __builtin_amdgcn_readfirstlane((rows + 1) / 2 * 16u), lane);
        ++next_tile;
        if (ROTATE && --to_end == 0) {
          next_head = (int)(pc.ta / seen1);
          next_tile = (int)(pc.ta % seen1);
          seek();
        } else if (next_tile < seen) {
          next_q += (uint64_t)QT * q_stride;
          next_do += (uint64_t)QT * do_stride;
          next_stat += QT * 8;
        } else {
          next_tile = 0;
          ++next_head;
          seek();
        }
      };
      phase_barrier();                                 // the piece before is read; its stores need not have landed
      const float* table = nullptr;                    // the bias of the present head
      {
        const GradArgs a = grad_args<true>();
        const Seq& q = wk.q;
        const int n0 = wk.b * kGradRows;
        const uint32_t v_stride = (uint32_t)a.io.v_tok * 2u;
        uint32_t v_off[TV::PER];
#pragma unroll
        for (int i = 0; i < TV::PER; ++i) v_off[i] = grad_slot<D, 64>(lw, i, lane, v_stride);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int k0 = n0 + 64 * half;
          const uint32_t nrec = __builtin_amdgcn_readfirstlane((uint32_t)min(max(q.lk - k0, 0), 64) * v_stride);
          const uint64_t at =
              first_lane_u64((uint64_t)(((int64_t)q.k0 + k0) * a.io.v_tok + (int64_t)wk.h * a.io.v_head) * 2u);
          grad_issue<D, 64>(vtile + half * TV::BYTES + lw * (TV::BYTES / 4), a.io.v, at, nrec, v_off);
        }
        if (left > 0) {
          seek();
          issue(0);
        }
        if constexpr (BIAS) {
          table = a.io.table + (int64_t)(wk.h * a.g.G + head) * a.io.bias_pitch;
          far_bias(far, table);
        }
#pragma unroll
        for (int kc = 0; kc < X::QT; ++kc) {
          const int n = key0 + X::MR * kc + c;
          const uint16_t* src = a.io.k + ((int64_t)q.k0 + n) * a.io.k_tok + (int64_t)wk.h * a.io.k_head + 8 * lg;
#pragma unroll
          for (int ks = 0; ks < D / X::KC; ++ks) {
            u32x4 w = u32x4{0u, 0u, 0u, 0u};
            if (n < q.lk) w = *(const u32x4*)(src + X::KC * ks);
            kreg[ks][kc] = __builtin_bit_cast(bf16x8, w);
          }
#pragma unroll
          for (int dt = 0; dt < D / X::MR; ++dt)
#pragma unroll
            for (int i = 0; i < X::AR; ++i) dk[dt][kc][i] = dv[dt][kc][i] = 0.f;
        }
      }
      // rows before this one see none of the wave's keys, those from it on all of them
      const bool causal = grad_args<true>().g.causal;
      const int from = key0 < wk.q.lk ? (causal ? key0 - off : 0) : 0x7fffffff;
      const int whole_from = causal ? key0 + 31 - off : 0;
      for (int st = 0, table_head = head; left > 0; --left, st ^= 1) {
        __builtin_amdgcn_s_waitcnt(0);
        phase_barrier();
        const int row0 = (first + tile) * QT;
        if constexpr (BIAS) {
          if (head != table_head) {
            table_head = head;
            const GradArgs a = grad_args<true>();
            table = a.io.table + (int64_t)(wk.h * a.g.G + head) * a.io.bias_pitch;
            far_bias(far, table);
          }
        }
        head = next_head;
        tile = next_tile;
        if (left > 1) issue(st ^ 1);
        if (row0 + (QT - 1) < from) continue;
        unsigned char* const qt = ring + st * (2 * T::BYTES);
        unsigned char* const dt = qt + T::BYTES;
        // Rows that see nothing take no part, whatever q and do hold there: 0 times NaN would.  They come from the mask or
        // from weights of -inf.  (Every wave clears them before it reads, all of them to the same zeros.)
        if (!ROTATE && __builtin_expect(far.hides || row0 + off < 0, 0)) {
          const float lse = *(const float*)(stat + st * kStatBytes + 8 * (lane & (QT - 1)));
          for (uint64_t none = __ballot(lse == INFINITY && lane < QT); none; none &= none - 1) {
            const int at = __builtin_ctzll(none) * T::STRIDE + 16 * lane;
            if (lane < T::SLOTS) *(u32x4*)(qt + at) = *(u32x4*)(dt + at) = u32x4{0u, 0u, 0u, 0u};
          }
          lds_order();
        }
        typename X::Acc s[NT][X::QT], dp[NT][X::QT];
        float to_log2 = scale_log2, shift = 0.f;
        rows_product<D, NT>(qt, kreg, s, rbase);
        if constexpr (BIAS) {
          const TileBias bias = tile_bias(far, key0 - (row0 + QT - 1 + off), key0 + 31 - (row0 + off));
          shift = bias.far;
          if (bias.near) {
            to_log2 = 1.0f;
            const float* at0 = table + (key0 + c - (row0 + 4 * lg + 3 + off) - far.lo + kBiasPad);
            f32x4u b[NT][X::QT][X::AR / 4];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int kc = 0; kc < X::QT; ++kc)
#pragma unroll
                for (int i = 0; i < X::AR; i += 4)
                  b[t][kc][i / 4] = *(const f32x4u*)(at0 + (X::MR * kc - X::MR * t - X::acc_row(i)));
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int kc = 0; kc < X::QT; ++kc)
#pragma unroll
                for (int i = 0; i < X::AR; ++i)
                  s[t][kc][i] = __builtin_fmaf(s[t][kc][i], scale_log2, b[t][kc][i / 4][3 - i % 4]);
          }
        }
        tiles_product<D, NT>(dt, vtile + (w0 >> 6) * TV::BYTES + (w0 & 63) * (2 * D), dp, rbase, rbase);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < X::AR; i += 4) {
            const int r = X::MR * t + X::acc_row(i) + 4 * lg;        // the first of four rows
            const f32x4 s01 = *(const f32x4*)(stat + st * kStatBytes + 8 * r);
            const f32x4 s23 = *(const f32x4*)(stat + st * kStatBytes + 8 * r + 16);
            const float lse[4] = {s01[0], s01[2], s23[0], s23[2]}, delta[4] = {s01[1], s01[3], s23[1], s23[3]};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float m = BIAS ? lse[j] - shift : lse[j];
#pragma unroll
              for (int kc = 0; kc < X::QT; ++kc) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][kc][i + j], to_log2, -m));
                s[t][kc][i + j] = p;
                dp[t][kc][i + j] = p * (dp[t][kc][i + j] - delta[j]);
              }
            }
          }
        if (__builtin_expect(row0 + QT > lq || row0 < whole_from, 0)) {
          // rows that do not exist, whatever their statistics are, and pairs that do not see each other
          const int end = lq - row0 - 4 * lg;
#pragma unroll
          for (int kc = 0; kc < X::QT; ++kc) {
            const int begin = causal ? key0 + X::MR * kc + c - off - row0 - 4 * lg : 0;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int i = 0; i < X::AR; ++i) {
                const int r = X::MR * t + X::acc_row(i);
                const bool none = (r >= end) | (causal & (r < begin));
                s[t][kc][i] = none ? 0.f : s[t][kc][i];
                dp[t][kc][i] = none ? 0.f : dp[t][kc][i];
              }
          }
        }
        bf16x8 op[QT / X::KC][X::QT];
        as_operand<D, NT>(s, op);
        columns_product<D, QT / X::KC>(dt, op, dv, cbase);
        as_operand<D, NT>(dp, op);
        columns_product<D, QT / X::KC>(qt, op, dk, cbase);
      }
      __builtin_amdgcn_s_waitcnt(0);                   // V, where nothing saw the unit
      const GradArgs a = grad_args<true>();
      const bool whole = pc.ta == 0 && pc.tb == pc.n;
      const int slot = 2 * l + (pc.ta == 0 ? 1 : 0);
      const int n0 = wk.b * kGradRows;
      if (!whole && tid == 0) a.io.cut[slot] = int4{wk.q.k0 + n0, min(kGradRows, wk.q.lk - n0), wk.h, 1};
#pragma unroll
      for (int kc = 0; kc < X::QT; ++kc) {
        const int r = w0 + X::MR * kc + c;
        if (whole) {
          const bool ok = n0 + r < wk.q.lk;
          const int64_t tok = (int64_t)wk.q.k0 + n0 + r;
          store_rows<D>(dk, kc, a.io.scale, ok, a.io.out0 + tok * a.io.out0_tok + (int64_t)wk.h * a.io.out0_head, lg);
          store_rows<D>(dv, kc, 1.0f, ok, a.io.out1 + tok * a.io.out1_tok + (int64_t)wk.h * a.io.out1_head, lg);
        } else {
          float* dst = a.io.part + ((size_t)slot * 2 * kGradRows + r) * D;
          store_part<D>(dk, kc, dst, lg);
          store_part<D>(dv, kc, dst + (size_t)kGradRows * D, lg);
        }
      }
    }
    const GradArgs a = grad_args<true>();
    grad_on<QT>(a.g, wk, unit_end);
  }
}

// ------------------------------------------------------------------------------------------------
// dQ, and the bias' gradient

// Blocks of 16 x 16 that are in LDS at once, of each wave: all five where there is room for two workgroups of a CU.
template <int D>
constexpr int diagonal_blocks() {
  return D == 128 ? 1 : 5;
}

// Sum over the lanes l, l ^ 16, l ^ 32 and l ^ 48, in all of them.
__device__ __forceinline__ float sum_quarters(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto s = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t v = __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, (uint32_t)s[0]) +
                                                      __builtin_bit_cast(float, (uint32_t)s[1]));
  const auto t = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return __builtin_bit_cast(float, (uint32_t)t[0]) + __builtin_bit_cast(float, (uint32_t)t[1]);
}

// Adds a wave's tile of dS to its sums by distance, `sums`, which start at distance lo - kBiasPad: x[t][c] is the
// product's accumulator, key rows by query columns; `first` is the place of distance 0 of the tile's first pair.
//
// The blocks of 16 keys by 16 queries whose keys are as far ahead of their queries are added first (block e has 16 e
// keys more than queries, from -1 to 3).  Each is laid into LDS row by row (a query's 16 keys) and its diagonals
// are summed: lane j of quarter h takes key (j + r) mod 16 of the queries r = 4 h .. 4 h + 3, which lie at distance
// j where j + r < 16, else j - 16.  So distance 16 m + j of the tile is what lies ahead in block m and behind in m + 1.
template <int D>
__device__ __forceinline__ void add_diagonals(const typename Mma<D>::Acc (*x)[Mma<D>::QT], float* block, float* sums,
                                              int first, int lane) {
  using X = Mma<D>;
  constexpr int NB = diagonal_blocks<D>();
  const int j = lane & 15, quarter = lane >> 4;
  float at[6] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f};        // distances 16 (m - 2) + j
#pragma unroll
  for (int e0 = -1; e0 < 4; e0 += NB) {
#pragma unroll
    for (int e = e0; e < 4 && e < e0 + NB; ++e) {
      float* to = block + 256 * (e - e0);
      if constexpr (X::MR == 16) {
        f32x4 y = e >= 0 ? x[e][0] : x[0][1];
        if (e >= 0 && e < 3) y += x[e + 1][1];
        *(f32x4*)(to + 16 * j + 4 * quarter) = y;
      } else {
        // lanes of even quarters hold the columns of the first 16 queries, the others those of the second; registers
        // 8 (kt & 1) + 4 u + v of accumulator kt / 2 hold key 8 u + 4 (lane / 32) + v of key block kt, which is
        // e for the first queries and e + 1 for the second
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          f32x4 y = f32x4{0.f, 0.f, 0.f, 0.f};
          const int k0 = e, k1 = e + 1;
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            if (k1 < 4) {
              const uint32_t z = __builtin_bit_cast(uint32_t, (float)x[(k1 & 3) >> 1][0][8 * (k1 & 1) + 4 * u + v]);
              const auto s = __builtin_amdgcn_permlane16_swap(z, z, false, false);
              y[v] = __builtin_bit_cast(float, (uint32_t)s[1]);          // the odd quarter's, in both
            }
            if (k0 >= 0) y[v] += x[(k0 & 3) >> 1][0][8 * (k0 & 1) + 4 * u + v];
          }
          if ((quarter & 1) == 0) *(f32x4*)(to + 16 * j + 8 * u + 4 * (lane >> 5)) = y;
        }
      }
    }
    lds_order();
#pragma unroll
    for (int e = e0; e < 4 && e < e0 + NB; ++e) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 4 * quarter + i;
        const float v = block[256 * (e - e0) + 16 * r + ((j + r) & 15)];
        at[e + 2] += j + r < 16 ? v : 0.f;
        at[e + 1] += j + r < 16 ? 0.f : v;
      }
    }
    lds_order();
  }
#pragma unroll
  for (int m = 0; m < 6; ++m) at[m] = sum_quarters(at[m]);
  // quarter h writes segments h and, for the last two, 4 + h
  const float a = quarter == 0 ? at[0] : quarter == 1 ? at[1] : quarter == 2 ? at[2] : at[3];
  const float b = quarter == 0 ? at[4] : at[5];
  float* p = sums + (first - 32 + lane);
  p[0] += a;
  if (quarter < 2) p[64] += b;
  lds_order();
}

template <int D, bool BIAS>
constexpr int row_lds() {
  return 4 * GradTile<D, KT>::BYTES + (BIAS ? 4 * (256 * diagonal_blocks<D>() + kBiasPitch) * 4 : 0);
}

// As key_grad, with 32 KB of K and V (d 128) for 6.3 MFLOP.
template <int D, bool BIAS, bool ROTATE>
__device__ __forceinline__ void row_grad(unsigned char* lds, int group, int P) {
  using X = Mma<D>;
  constexpr int NT = KT / X::MR;
  using T = GradTile<D, KT>;
  unsigned char* const ring = lds;                     // K, V of two stages
  constexpr int BLOCK = 256 * diagonal_blocks<D>();
  float(*const block)[BLOCK] = (float(*)[BLOCK])(lds + 4 * T::BYTES);
  float(*const sums)[kBiasPitch] = (float(*)[kBiasPitch])(lds + 4 * T::BYTES + 4 * BLOCK * 4);
  const int l = (group & 7) * (P >> 3) + (group >> 3);
  const int tid = threadIdx.x, lane = tid & 63;
  const int lw = __builtin_amdgcn_readfirstlane(tid >> 6);
  GradWalk wk;
  float scale_log2;
  FarBias far{0, 0, 0.f, 0.f, false};
  int sum_head = 0, last_head = 0;       // the heads whose sums this workgroup writes
  float far_lo = 0.f, far_hi = 0.f;      // the lane's sums of dS beyond the table's ends
  uint32_t k_stride, v_stride;
  {
    const GradArgs a = grad_args<false>();
    if (a.g.cuts && tid == 0) a.io.cut[2 * l] = a.io.cut[2 * l + 1] = int4{0, 0, 0, 0};
    uint64_t share;
    wk = grad_start<0>(a.g, l, P, &share);
    scale_log2 = a.io.scale_log2;
    k_stride = (uint32_t)a.io.k_tok * 2u;
    v_stride = (uint32_t)a.io.v_tok * 2u;
    if constexpr (BIAS) {
      if (group == 0 && tid == 0) {
        a.io.line[0] = wk.head;
        a.io.line[1] = share;
      }
      // a stretch that its borders' moving left empty still writes its heads' sums
      if ((uint64_t)(uint32_t)l * share >= wk.head * (uint32_t)a.g.NH) return;
      far.lo = a.io.bias_lo;
      far.hi = a.io.bias_hi;
      sum_head = (int)((uint64_t)(uint32_t)l * share / wk.head);
      last_head = (int)((wk.end - 1) / wk.head);
      for (int i = tid; i < 4 * kBiasPitch; i += kGradThreads) (&sums[0][0])[i] = 0.f;
      __syncthreads();
    } else if (!wk.more()) {
      return;
    }
  }
  // writes the sums of the heads before `until`
  auto flush = [&](int until) {
    if constexpr (BIAS) {
      if (sum_head >= until) return;
      const GradArgs a = grad_args<false>();
      const int pitch = a.io.bias_pitch;
      for (; sum_head < until; ++sum_head) {
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
          far_lo += __shfl_xor(far_lo, m);
          far_hi += __shfl_xor(far_hi, m);
        }
        if (lane == 0) {
          sums[lw][0] += far_lo;
          sums[lw][pitch - 1] += far_hi;
        }
        far_lo = far_hi = 0.f;
        __syncthreads();
        float* dst = a.io.dist + (size_t)(l + sum_head) * pitch;
        for (int i = tid; i < pitch; i += kGradThreads) {
          dst[i] = (sums[0][i] + sums[1][i]) + (sums[2][i] + sums[3][i]);
          sums[0][i] = sums[1][i] = sums[2][i] = sums[3][i] = 0.f;
        }
        __syncthreads();
      }
    }
  };
  const int c = lane % X::MR, lg = lane / X::MR;
  const int rbase = rows_base<D>(lane), cbase = columns_base<D>(lane);
  uint32_t k_off[T::PER], v_off[T::PER];
#pragma unroll
  for (int i = 0; i < T::PER; ++i) {
    k_off[i] = grad_slot<D, KT>(lw, i, lane, k_stride);
    v_off[i] = grad_slot<D, KT>(lw, i, lane, v_stride);
  }
  const int w0 = 32 * lw;
  uint32_t done = 0;                                   // tiles so far
  typename X::Acc dq[D / X::MR][X::QT];
  bf16x8 qreg[D / X::KC][X::QT], doreg[D / X::KC][X::QT];

  while (wk.more()) {
    uint64_t unit_end;
    GradPiece pc;
    {
      const GradArgs a = grad_args<false>();
      pc = grad_piece<KT>(a.g, wk, &unit_end);
    }
    if (pc.tb > pc.ta) {
      const int lk = wk.q.lk, off = wk.q.lk - wk.q.lq;
      const int keys = (int)grad_seen(wk.line, wk.b);  // keys that the unit's last token sees
      const int N = keys == 0 ? 0 : (int)(pc.tb - pc.ta);
      // as in key_grad: from `first` to the piece's end and then from its start
      int first = (int)pc.ta;
      if (ROTATE && N > 0) {
        const int at = (int)(done % (((uint32_t)lk + KT - 1) / KT));
        if (at >= pc.ta && at < pc.tb) first = at;
        done += (uint32_t)N;
      }
      first = __builtin_amdgcn_readfirstlane(first);
      int to_end = first == (int)pc.ta ? 0 : (int)pc.tb - first;   // tiles to load before the piece's start, if that is due
      if constexpr (BIAS) flush(wk.h);
      phase_barrier();                                 // the piece before is read; its stores need not have landed
      uint64_t next_k = 0, next_v = 0;                 // where the tile to load next starts
      int next_left = 0;                               // keys from it on
      auto issue = [&](int st) {
        const uint32_t rows = (uint32_t)min(next_left, KT);
        unsigned char* dst = ring + st * (2 * T::BYTES) + lw * (T::BYTES / 4);
        grad_issue<D, KT>(dst, nullptr, first_lane_u64(next_k), __builtin_amdgcn_readfirstlane(rows * k_stride), k_off);
        grad_issue<D, KT>(dst + T::BYTES, nullptr, first_lane_u64(next_v),
                          __builtin_amdgcn_readfirstlane(rows * v_stride), v_off);
        int tiles = 1;
        if (ROTATE && --to_end == 0) tiles = 1 - N;
        next_k += (uint64_t)((int64_t)tiles * KT * (int64_t)k_stride);
        next_v += (uint64_t)((int64_t)tiles * KT * (int64_t)v_stride);
        next_left -= tiles * KT;
      };
      float lse[X::QT], delta[X::QT];
      int limit[X::QT], wave_keys = 0, wave_open = 0x7fffffff;
      const float* table = nullptr;
      int least_pos = 0;                               // place of the wave's first query among the keys
      {
        const GradArgs a = grad_args<false>();
        const Seq& q = wk.q;
        const int kvh = wk.h / a.g.GS, head0 = wk.h % a.g.GS * a.g.GH;       // the unit's heads within the group
        const int heads = min(a.g.GH, a.g.G - head0);
        const int t0 = wk.b * a.g.TB, tokens = min(a.g.TB, q.lq - t0);
        if (N > 0) {
          const int64_t tok = (int64_t)q.k0 + 64 * (int64_t)first;
          next_k = first_lane_u64((uint64_t)(uintptr_t)a.io.k + (uint64_t)(tok * a.io.k_tok + kvh * a.io.k_head) * 2u);
          next_v = first_lane_u64((uint64_t)(uintptr_t)a.io.v + (uint64_t)(tok * a.io.v_tok + kvh * a.io.v_head) * 2u);
          next_left = lk - 64 * first;
          issue(0);
        }
        if constexpr (BIAS) {
          table = a.io.table + (int64_t)(kvh * a.g.G + head0) * a.io.bias_pitch;
          far_bias(far, table);
          least_pos = off + t0 + w0;
        }
#pragma unroll
        for (int qc = 0; qc < X::QT; ++qc) {
          const int r = w0 + X::MR * qc + c;
          const int t = (int)(((uint32_t)r * (uint32_t)a.g.gh_magic) >> 16), j = r - t * a.g.GH;
          const bool ok = t < tokens && j < heads;
          const int token = t0 + t, head = kvh * a.g.G + head0 + j;
          const int64_t tok = (int64_t)q.q0 + token;
          const uint16_t* qs = a.io.q + tok * a.io.q_tok + (int64_t)head * a.io.q_head + 8 * lg;
          const uint16_t* ds = a.io.dout + tok * a.io.do_tok + (int64_t)head * a.io.do_head + 8 * lg;
#pragma unroll
          for (int ks = 0; ks < D / X::KC; ++ks) {
            u32x4 w = u32x4{0u, 0u, 0u, 0u}, x = w;
            if (ok) {
              w = *(const u32x4*)(qs + X::KC * ks);
              x = *(const u32x4*)(ds + X::KC * ks);
            }
            qreg[ks][qc] = __builtin_bit_cast(bf16x8, w);
            doreg[ks][qc] = __builtin_bit_cast(bf16x8, x);
          }
          float2 z = float2{INFINITY, 0.f};
          if (ok) z = a.io.stat[(uint64_t)head * (uint32_t)a.g.Tq + (uint64_t)tok];
          lse[qc] = z.x;
          delta[qc] = z.y;
          // as in key_grad: rows that see nothing
          if (!ROTATE && __builtin_expect(far.hides || off + t0 < 0, 0) && z.x == INFINITY) {
#pragma unroll
            for (int ks = 0; ks < D / X::KC; ++ks) qreg[ks][qc] = doreg[ks][qc] = bf16x8{};
          }
          limit[qc] = ok ? (a.g.causal ? max(0, min(lk, off + token + 1)) : lk) : 0x7fffffff;
          wave_keys = max(wave_keys, ok ? limit[qc] : 0);
          wave_open = min(wave_open, limit[qc]);
#pragma unroll
          for (int dt = 0; dt < D / X::MR; ++dt)
#pragma unroll
            for (int i = 0; i < X::AR; ++i) dq[dt][qc][i] = 0.f;
        }
      }
#pragma unroll
      for (int m = 1; m < X::MR; m <<= 1) {
        wave_keys = max(wave_keys, __shfl_xor(wave_keys, m));
        wave_open = min(wave_open, __shfl_xor(wave_open, m));
      }
      wave_keys = __builtin_amdgcn_readfirstlane(wave_keys);       // keys that some row of the wave sees
      wave_open = __builtin_amdgcn_readfirstlane(wave_open);       // and that all of them see
      int next_key0 = 64 * first;
      for (int left = N, st = 0; left > 0; --left, st ^= 1) {
        __builtin_amdgcn_s_waitcnt(0);
        phase_barrier();
        const int key0 = next_key0;
        next_key0 = lk - next_left;
        if (left > 1) issue(st ^ 1);
        if (key0 >= wave_keys) continue;
        const unsigned char* kt = ring + st * (2 * T::BYTES);
        typename X::Acc s[NT][X::QT], dp[NT][X::QT];
        float to_log2 = scale_log2, shift = 0.f;
        bool near = false;
        rows_product<D, NT>(kt, qreg, s, rbase);
        if constexpr (BIAS) {
          const TileBias bias = tile_bias(far, key0 - (least_pos + 31), key0 + 63 - least_pos);
          shift = bias.far;
          near = bias.near;
          if (near) {
            to_log2 = 1.0f;
            const float* at = table + (key0 + 4 * lg - (least_pos + c) - far.lo + kBiasPad);
            f32x4u b[NT][X::QT][X::AR / 4];
#pragma unroll
            for (int qc = 0; qc < X::QT; ++qc)
#pragma unroll
              for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < X::AR; i += 4)
                  b[t][qc][i / 4] = *(const f32x4u*)(at + (X::MR * t + X::acc_row(i) - X::MR * qc));
#pragma unroll
            for (int qc = 0; qc < X::QT; ++qc)
#pragma unroll
              for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < X::AR; ++i)
                  s[t][qc][i] = __builtin_fmaf(s[t][qc][i], scale_log2, b[t][qc][i / 4][i % 4]);
          }
        }
        rows_product<D, NT>(kt + T::BYTES, doreg, dp, rbase);
#pragma unroll
        for (int qc = 0; qc < X::QT; ++qc) {
          const float m = BIAS ? lse[qc] - shift : lse[qc];
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < X::AR; ++i) {
              const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][qc][i], to_log2, -m));
              dp[t][qc][i] = p * (dp[t][qc][i] - delta[qc]);
            }
        }
        if (__builtin_expect(key0 + KT > wave_open, 0)) {
#pragma unroll
          for (int qc = 0; qc < X::QT; ++qc) {
            const int lim = limit[qc] - key0 - 4 * lg;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int i = 0; i < X::AR; ++i)
                if (X::MR * t + X::acc_row(i) >= lim) dp[t][qc][i] = 0.f;
          }
        }
        if constexpr (BIAS) {
          if (near) {
            add_diagonals<D>(dp, block[lw], sums[lw], key0 - least_pos - far.lo + kBiasPad, lane);
          } else {
            float x = 0.f;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int qc = 0; qc < X::QT; ++qc)
#pragma unroll
                for (int i = 0; i < X::AR; ++i) x += dp[t][qc][i];
            if (key0 + 63 - least_pos <= far.lo) far_lo += x;
            else far_hi += x;
          }
        }
        bf16x8 op[KT / X::KC][X::QT];
        as_operand<D, NT>(dp, op);
        columns_product<D, KT / X::KC>(kt, op, dq, cbase);
      }
      const GradArgs a = grad_args<false>();
      const bool whole = pc.ta == 0 && pc.tb == pc.n;
      const int slot = 2 * l + (pc.ta == 0 ? 1 : 0);
      const int kvh = wk.h / a.g.GS, head0 = wk.h % a.g.GS * a.g.GH;
      const int heads = min(a.g.GH, a.g.G - head0);
      const int t0 = wk.b * a.g.TB, tokens = min(a.g.TB, wk.q.lq - t0);
      if (!whole && tid == 0) a.io.cut[slot] = int4{wk.q.q0 + t0, tokens, kvh * a.g.G + head0, heads};
#pragma unroll
      for (int qc = 0; qc < X::QT; ++qc) {
        const int r = w0 + X::MR * qc + c;
        const int t = (int)(((uint32_t)r * (uint32_t)a.g.gh_magic) >> 16), j = r - t * a.g.GH;
        if (whole)
          store_rows<D>(dq, qc, a.io.scale, t < tokens && j < heads,
                        a.io.out0 + ((int64_t)wk.q.q0 + t0 + t) * a.io.out0_tok +
                            (int64_t)(kvh * a.g.G + head0 + j) * a.io.out0_head,
                        lg);
        else
          store_part<D>(dq, qc, a.io.part + ((size_t)slot * kGradRows + r) * D, lg);
      }
    }
    const GradArgs a = grad_args<false>();
    grad_on<0>(a.g, wk, unit_end);
  }
  if constexpr (BIAS) flush(last_head + 1);
}

// One launch for both walks, the workgroups of dK and dV, which take longer, in front: with as many of either as there
// are CUs every CU gets one of each (one after the other 836 us for 8192 tokens as above, together 780; one prompt of
// 77 tokens, 16 heads, d 64, 27 and 10).
template <int D, bool BIAS, bool ROTATE>
__global__ __launch_bounds__(kGradThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void grad_kernel(GradBoth) {
  constexpr int LDS = key_lds<D>() > row_lds<D, BIAS>() ? key_lds<D>() : row_lds<D, BIAS>();
  __shared__ __attribute__((aligned(1024))) unsigned char lds[LDS];
  const int keys_p = grad_args<true>().P;
  if ((int)blockIdx.x < keys_p) key_grad<D, BIAS, ROTATE>(lds, blockIdx.x, keys_p);
  else row_grad<D, BIAS, ROTATE>(lds, blockIdx.x - keys_p, gridDim.x - keys_p);
}

// ------------------------------------------------------------------------------------------------
// The gradient of the bias' weights: a workgroup adds the sums by distance of one bucket of a head, over the workgroups
// of dQ that met the head and the distances of the bucket (what lies beyond the ends belongs to them), in 64 bits and a
// fixed order, and then every `step`-th bucket from there.  A wave has every fourth workgroup, a lane every 64th distance.
// Where there are more buckets than distances it goes through those that some distance names; the others were set to 0 by
// the call's first launch (two prompts of 300 and 77 tokens, 16 heads, 2^20 buckets: 13.3 ms with each bucket's distances
// looked for, so 0.074; 4096 buckets 97 -> 61 us, but 513 49 -> 55).
struct DistArgs {
  const float* dist;
  const uint64_t* line;
  SeqBias bias;
  void* dweight;
  int pitch, Hq, P, empty;
  int groups;              // workgroups of a head
};
constexpr int kDistChunks = (kBiasMost + 2 * kBiasPad + 63) / 64;
constexpr int kDistGroups = 64;
bool by_name(const SeqBias& b) { return b.buckets > kBiasMost; }
// NAMED is a kernel of its own, as its registers would cost the joins of the pieces beside it a wave of a SIMD (48 prompts
// of 1 to 300 tokens 37.0 -> 37.6 us).
template <bool NAMED>
__device__ __forceinline__ void dist_merge(const DistArgs& a, int h, int first, int step) {
  __shared__ double part[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t head = a.empty ? 0 : a.line[0], share = a.empty ? 1 : a.line[1];
  const int l0 = (int)(head * (uint32_t)h / share);
  const int l1 = head == 0 ? l0 - 1 : min((int)((head * ((uint32_t)h + 1ull) - 1) / share), a.P - 1);
  int name[NAMED ? kDistChunks : 1];       // the buckets of the workgroup among the lane's distances
  if constexpr (NAMED) {
#pragma unroll
    for (int c = 0; c < kDistChunks; ++c) {
      const int b = a.bias.bucket[min(max(lane + 64 * c - kBiasPad, 0), a.bias.hi - a.bias.lo)];
      name[c] = b >= 0 && b < a.bias.buckets && b % step == first ? b : INT_MAX;
    }
  }
  // the one behind b
  auto next = [&](int b) {
    int x = b + step;
    if constexpr (NAMED) {
      x = INT_MAX;
#pragma unroll
      for (int c = 0; c < kDistChunks; ++c) x = min(x, name[c] > b ? name[c] : INT_MAX);
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) x = min(x, __shfl_xor(x, m));
      x = __builtin_amdgcn_readfirstlane(x);
    }
    return x;
  };
  for (int b = NAMED ? next(-1) : first; b < a.bias.buckets; b = next(b)) {
    double x = 0.0;
    uint32_t mine = 0;       // bit c: distance lane + 64 c is of the bucket (all loads at once, not one behind the other)
#pragma unroll
    for (int c = 0; c < kDistChunks; ++c) {
      const int i = lane + 64 * c;
      const bool hit = a.bias.bucket[min(max(i - kBiasPad, 0), a.bias.hi - a.bias.lo)] == b;
      mine |= hit && i < a.pitch ? 1u << c : 0;
    }
    for (; mine; mine &= mine - 1) {
      const float* at = a.dist + (size_t)h * a.pitch + lane + 64 * __builtin_ctz(mine);
#pragma unroll 16
      for (int l = l0 + wave; l <= l1; l += 4) x += at[(size_t)l * a.pitch];
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x += __shfl_xor(x, m);
    if (lane == 0) part[wave] = x;
    __syncthreads();
    if (threadIdx.x == 0) {
      const float y = (float)((part[0] + part[1]) + (part[2] + part[3]));
      const size_t at = (size_t)b * a.Hq + h;
      if (a.bias.bf16) ((uint16_t*)a.dweight)[at] = (uint16_t)(pack_bf16x2(y, 0.f) & 0xffffu);
      else ((float*)a.dweight)[at] = y;
    }
    __syncthreads();
  }
}

// Joins the pieces of a unit that several stretches share, in the order of the stretches (as seq_merge_kernel,
// but sums alone).  A workgroup joins 16 rows of an array (dK, dV or dQ) of the unit of one stretch.  In front of
// them (the longest chains) are those of the weights' gradient.
template <int D, bool NAMED>
__global__ __launch_bounds__(256) void grad_merge_kernel(GradIo keys, GradIo rows, DistArgs dist, int keys_p, int rows_p,
                                                         int rows_gh) {
  constexpr int TPR = 16, W = D / TPR;
  const int dists = dist.Hq * dist.groups;
  if ((int)blockIdx.x < dists) {
    dist_merge<NAMED>(dist, blockIdx.x / dist.groups, blockIdx.x % dist.groups, dist.groups);
    return;
  }
  const int block = blockIdx.x - dists;
  const bool of_keys = block < 16 * keys_p;
  const GradIo& io = of_keys ? keys : rows;
  const int y = of_keys ? block % 16 : block % 8, array = y / 8;
  const int l0 = of_keys ? block / 16 : (block - 16 * keys_p) / 8, P = of_keys ? keys_p : rows_p;
  const int A = of_keys ? 2 : 1, GH = of_keys ? 1 : rows_gh;
  const int lane = threadIdx.x & 63;
  const int4 u = io.cut[2 * l0 + 1];
  if (u.w == 0) return;
  int n = 0;
  for (;;) {
    const int l = l0 + 1 + n + lane;
    const int4 x = io.cut[2 * min(l, P - 1)];
    const uint64_t other = ~__ballot(l < P && x.w != 0 && x.x == u.x && x.z == u.z);
    if (other) {
      n += __builtin_ctzll(other);
      break;
    }
    n += 64;
  }
  const int r = y % 8 * 16 + threadIdx.x / TPR, part = threadIdx.x % TPR;
  const int token = r / GH, head = r - token * GH;
  if (token >= u.y || head >= u.w) return;
  float acc[W];
#pragma unroll
  for (int e = 0; e < W; ++e) acc[e] = 0.f;
  constexpr int BATCH = 4;
  for (int i0 = 0; i0 <= n; i0 += BATCH) {
    f32x4 x[BATCH][W / 4];
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      const int i = min(i0 + j, n);
      const size_t slot = i == 0 ? 2 * l0 + 1 : 2 * (l0 + i);
#pragma unroll
      for (int e = 0; e < W / 4; ++e)
        x[j][e] = *(const f32x4*)(io.part + ((slot * A + array) * kGradRows + r) * D + part * W + 4 * e);
    }
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      if (i0 + j > n) break;
#pragma unroll
      for (int e = 0; e < W; ++e) acc[e] += x[j][e / 4][e % 4];
    }
  }
  const bool second = array == 1;
  const float f = second ? 1.0f : io.scale;
  uint16_t* dst = (second ? io.out1 : io.out0) + (int64_t)(u.x + token) * (second ? io.out1_tok : io.out0_tok) +
                  (int64_t)(u.z + head) * (second ? io.out1_head : io.out0_head) + part * W;
#pragma unroll
  for (int e = 0; e < W; e += 4)
    *(u32x2*)(dst + e) = u32x2{pack_bf16x2(acc[e] * f, acc[e + 1] * f), pack_bf16x2(acc[e + 2] * f, acc[e + 3] * f)};
}

// ------------------------------------------------------------------------------------------------
// What both walks need of a row: lse in base 2, and delta; and the bias by distance, and zeros for its gradient where not
// every bucket is written later.  Bound by reading o and do: 67 MB
// (8192 tokens, 16 heads, d 128) in 12.2 us, 5.5 TB/s.
// More tokens take as long where there are many, and 1 us more where there are few.
constexpr int kPrepTokens = 4, kPrepHeads = 8;
struct PrepArgs {
  const uint16_t *o, *dout;
  const float *lse, *dlse;
  int64_t o_tok, o_head, do_tok, do_head;
  float2* stat;
  int Tq, Hq;
  int clears;                            // workgroups that clear the weights' gradient, in front
  int64_t zeros;                         // its values
  void* dweight;
  int tables;                            // workgroups that lay out the bias of a head each, behind them
  int64_t groups;                        // of kPrepTokens tokens by kPrepHeads heads
  SeqBias bias;
  int pitch;
  float* table;
};

template <int D>
__global__ __launch_bounds__(256) void grad_prep_kernel(PrepArgs a) {
  const int tid = threadIdx.x;
  if ((int)blockIdx.x < a.clears) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + tid; i < a.zeros; i += (int64_t)a.clears * 256) {
      if (a.bias.bf16) ((uint16_t*)a.dweight)[i] = 0;
      else ((float*)a.dweight)[i] = 0.f;
    }
    return;
  }
  const int block = blockIdx.x - a.clears, blocks = gridDim.x - a.clears;
  if (block < a.tables) {
    const int h = block;
    float* const table = a.table + (size_t)h * a.pitch;
    bool hides = false;
    for (int i = tid; i < a.pitch; i += 256) {
      const float x = bias_log2(a.bias, i - kBiasPad, a.Hq, h);
      hides |= x == -INFINITY;
      if (i > 0) table[i] = x;
    }
    const int any = __syncthreads_or(hides);
    if (tid == 0) table[0] = any ? 1.0f : 0.f;         // no tile reads the first three
    return;
  }
  constexpr int LPR = D / 8;             // lanes of a row
  constexpr int RPP = 256 / LPR;         // rows of a pass
  constexpr int ROWS = kPrepHeads * kPrepTokens;
  __shared__ float dots[ROWS];
  const int HB = (a.Hq + kPrepHeads - 1) / kPrepHeads;
  for (int64_t g = block - a.tables; g < a.groups; g += blocks - a.tables) {
    const int64_t t0 = g / HB * kPrepTokens;
    const int h0 = (int)(g % HB) * kPrepHeads;
#pragma unroll
    for (int p = 0; p < ROWS / RPP; ++p) {
      const int r = p * RPP + tid / LPR;
      const int64_t t = t0 + r / kPrepHeads;
      const int h = h0 + r % kPrepHeads;
      float x = 0.f;
      if (t < a.Tq && h < a.Hq) {
        const u32x4 u = *(const u32x4*)(a.o + t * a.o_tok + (int64_t)h * a.o_head + 8 * (tid % LPR));
        const u32x4 v = *(const u32x4*)(a.dout + t * a.do_tok + (int64_t)h * a.do_head + 8 * (tid % LPR));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x = __builtin_fmaf(__uint_as_float(u[i] << 16), __uint_as_float(v[i] << 16), x);
          x = __builtin_fmaf(__uint_as_float(u[i] & 0xffff0000u), __uint_as_float(v[i] & 0xffff0000u), x);
        }
      }
#pragma unroll
      for (int m = 1; m < LPR; m <<= 1) x += __shfl_xor(x, m);
      if (tid % LPR == 0) dots[r] = x;
    }
    __syncthreads();
    const int64_t t = t0 + tid % kPrepTokens;
    const int h = h0 + tid / kPrepTokens;
    if (tid < ROWS && t < a.Tq && h < a.Hq) {
      const float lse = a.lse[t * a.Hq + h];
      float delta = dots[tid % kPrepTokens * kPrepHeads + tid / kPrepTokens];
      if (a.dlse) delta -= a.dlse[t * a.Hq + h];
      // a row that sees nothing has no probabilities: exp2(x - inf) = 0
      const bool none = lse == -INFINITY;
      a.stat[(size_t)h * a.Tq + t] = float2{none ? INFINITY : lse * 1.4426950408889634f, none ? 0.f : delta};
    }
    __syncthreads();
  }
}

}  // namespace

template <int D>
static hipError_t launch_grad(const GradCall& c, hipStream_t st) {
  const int64_t zeros = c.has_bias && by_name(c.bias) ? (int64_t)c.bias.buckets * c.rows_g.Hq : 0;
  if (c.rows || zeros > 0) {
    const int64_t groups =
        c.rows ? ((int64_t)c.Tq + kPrepTokens - 1) / kPrepTokens * ceil_div(c.rows_g.Hq, kPrepHeads) : 0;
    const int tables = c.rows && c.has_bias ? c.rows_g.Hq : 0;
    const int clears = (int)(zeros < 1024 * 1024 ? (zeros + 1023) / 1024 : 1024);
    const PrepArgs p{c.o, c.rows_io.dout, c.lse, c.dlse, c.o_tok, c.o_head, c.rows_io.do_tok, c.rows_io.do_head,
                     const_cast<float2*>(c.rows_io.stat), c.Tq, c.rows_g.Hq, clears, zeros, c.dweight, tables, groups, c.bias,
                     c.rows_io.bias_pitch, const_cast<float*>(c.rows_io.table)};
    const int most = 1 << 20;
    hipLaunchKernelGGL((grad_prep_kernel<D>), dim3(clears + tables + (groups < most ? (int)groups : most)), dim3(256), 0, st, p);
  }
  const int keys_p = c.keys ? c.keys_p : 0, rows_p = c.rows ? c.rows_p : 0;
  if (keys_p + rows_p > 0) {
    const GradBoth a{{c.keys_g, c.keys_io, keys_p}, {c.rows_g, c.rows_io, rows_p}};
    const dim3 grid(keys_p + rows_p), block(kGradThreads);
    // the rotated walk is for calls without a mask and a bias: a 480P chunk over its context 1740 -> 1615 us; with a
    // mask it takes as long or 1.5 % longer, with a bias its variables cost more than it gains (d 128: 435 -> 486)
    if (c.has_bias) hipLaunchKernelGGL((grad_kernel<D, true, false>), grid, block, 0, st, a);
    else if (c.keys_g.causal) hipLaunchKernelGGL((grad_kernel<D, false, false>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((grad_kernel<D, false, true>), grid, block, 0, st, a);
  }
  const int keys_cut = c.keys_g.cuts ? keys_p : 0, rows_cut = c.rows_g.cuts ? rows_p : 0;
  const int groups = c.bias.buckets < kDistGroups ? c.bias.buckets : kDistGroups;
  const DistArgs d{c.rows_io.dist, c.rows_io.line, c.bias, c.dweight, c.rows_io.bias_pitch, c.has_bias ? c.rows_g.Hq : 0,
                   c.rows_p, !c.rows, groups};
  const int blocks = 16 * keys_cut + 8 * rows_cut + d.Hq * d.groups;
  if (blocks > 0) {
    const auto merge = c.has_bias && by_name(c.bias) ? grad_merge_kernel<D, true> : grad_merge_kernel<D, false>;
    hipLaunchKernelGGL(merge, dim3(blocks), dim3(256), 0, st, c.keys_io, c.rows_io, d, keys_cut, rows_cut, c.rows_g.GH);
  }
  return hipGetLastError();
}

hipError_t launch_prompt_bwd(const GradCall& c, int d, hipStream_t st) {
  return d == 128 ? launch_grad<128>(c, st) : launch_grad<64>(c, st);
}

}  // namespace la
